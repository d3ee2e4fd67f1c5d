"""The network operators where they can go wrong: rows without spread, tails of the activations, calls
between a pass and its backward pass, other streams, waits that run out."""
import numpy as np
import pytest

import paper_2608_27735_gb300 as ab

from . import _network as N
from .test_gpu_network import KINDS, TYPES, blank, close, f64, matrix

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    ab.build()
    return ab.Context(0)


# ---- layer norm

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cols", [7, 28, 63, 250, 1000, 4095, 9001, 17003])
@pytest.mark.parametrize("pad,lead", [(0, 0), (5, 3)])
def test_norm_of_constant_rows_at_any_width(ctx, kind, cols, pad, lead):
    """A row of one value has that value as its mean, whether the width's reciprocal and the row's sum are
    exact or not: y is the bias to the bit, and the weight gets no gradient."""
    values = np.array([[3.0], [37.5], [1000.0], [-0.1], [1000.1], [0.0]])
    x = matrix(np.repeat(values, cols, 1), kind, pad, lead)
    r = np.random.default_rng(cols)
    w = torch.as_tensor(r.normal(1, 0.3, cols)).to("cuda", TYPES[kind])
    b = torch.as_tensor(r.normal(0, 0.3, cols)).to("cuda", TYPES[kind])
    dy = matrix(r.normal(size=(6, cols)), kind, pad, lead)
    y, dx = blank(6, cols, kind, pad, lead), blank(6, cols, kind, pad, lead)
    mean, rstd = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    dw, db = torch.full_like(w, float("nan")), torch.full_like(b, float("nan"))
    ctx.reserve_network(6, cols)
    ab.abcd_layer_norm(ctx, x, w, b, 1e-5, y, mean, rstd)
    ab.abcd_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx, dw, db)
    ctx.sync()
    assert torch.equal(mean, x[:, 0].float())
    assert torch.equal(y, b.expand(6, cols))
    assert not dw.any()
    # the sums over the rows: 6 terms each, rounded to the type
    want = f64(dy).sum(0)
    mag = np.abs(f64(dy)).sum(0)
    close(db, want, 22 * N.EPS * mag + (np.abs(want) + 22 * N.EPS * mag) * N.UNIT[kind] + N.TINY[kind])
