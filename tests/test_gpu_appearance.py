"""The layer norm, feed-forward and dropout calls together with a block's render and its backward
pass: per-camera SH coefficients learned from photographs of different exposure."""
import numpy as np
import pytest

import paper_2608_27735_gb300 as ab
from paper_2608_27735_gb300 import scenegen as sg

from . import _network as N

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_layers_fit_exposures_that_one_colour_cannot():
    """Photographs differ by a gain of 0.4 to 1 per channel: one colour per Gaussian is left with the
    gains' spread, the layers with a fraction of it."""
    ab.build()
    from paper_2608_27735_gb300.appearance import appearance_experiment
    r = appearance_experiment()
    assert r["appearance"][0] == pytest.approx(r["one_colour"][0], rel=1e-6)   # they start as the identity
    assert r["appearance"][1] < 0.5 * r["one_colour"][1] < 0.5 * r["one_colour"][0]


def test_gradient_through_the_layers_is_the_formulas():
    """d sh and every weight's gradient of Appearance against the 64-bit formulas of its layers."""
    ab.build()
    from paper_2608_27735_gb300.appearance import Appearance
    ctx = ab.Context(0)
    n, cams = 200, 3
    app = Appearance(ctx, n, 1, cams, layers=2, embed=5, p=0.3, seed=4)
    r = np.random.default_rng(1)
    for b in app.blocks:
        b.w["w_down"].copy_(torch.from_numpy(r.normal(0, 0.1, b.w["w_down"].shape).astype(np.float32)))
    sh = torch.from_numpy(r.normal(size=(n, 4, 3)).astype(np.float32)).cuda()
    d = torch.from_numpy(r.normal(size=(n, 4, 3)).astype(np.float32)).cuda()
    got = app.forward(sh, 1)
    d_sh = app.backward(d, 1)
    ctx.sync()
    f = lambda t: t.double().cpu().numpy()
    x = [np.concatenate([f(sh).reshape(n, 12), np.tile(f(app.embed[1]), (n, 1))], 1)]
    kept = []
    for b in app.blocks:
        w = {k: f(t) for k, t in b.w.items()}
        nx, mean, rstd = N.norm(x[-1], w["norm_w"], w["norm_b"], b.eps)
        y, z, u = N.ff(nx, w["w_gate"], w["w_up"], w["w_down"], "silu")
        keep, s = N.kept(n, app.cols, 0.3, b.seed, b.drawn)
        kept.append((w, nx, mean, rstd, z, u, keep * s))
        x.append(x[-1] + y * keep * s)
    # sums of up to 200 terms of order one in 32 bits, through two layers
    tol = dict(rtol=2e-4, atol=2e-4)
    np.testing.assert_allclose(f(got), x[-1][:, :12].reshape(n, 4, 3), **tol)
    dx = np.concatenate([f(d).reshape(n, 12), np.zeros((n, 5))], 1)
    for k in (1, 0):
        w, nx, mean, rstd, z, u, mask = kept[k]
        dn, dwg, dwu, dwd = N.ff_grad(dx * mask, nx, w["w_gate"], w["w_up"], w["w_down"], "silu", z, u)
        dn, dw, db = N.norm_grad(dn, x[k], w["norm_w"], mean, rstd)
        g = app.blocks[k].grads
        for name, want in (("w_gate", dwg), ("w_up", dwu), ("w_down", dwd), ("norm_w", dw), ("norm_b", db)):
            assert np.linalg.norm(f(g[name]) - want) <= 2e-5 * np.linalg.norm(want), name
        dx = dx + dn
    np.testing.assert_allclose(f(d_sh), dx[:, :12].reshape(n, 4, 3), **tol)
    want = np.zeros((cams, 5))
    want[1] = dx[:, 12:].sum(0)
    np.testing.assert_allclose(f(app.d_embed), want, rtol=1e-3, atol=1e-3)


def test_adam_of_one_buffer_is_adam():
    ab.build()
    from paper_2608_27735_gb300.appearance import Adam
    ctx = ab.Context(0)
    r = np.random.default_rng(2)
    a = Adam(ctx, 100, 1e-2)
    x, m, v = r.normal(size=112), np.zeros(112), np.zeros(112)
    a.values.copy_(torch.from_numpy(x.astype(np.float32)))
    x = a.values.double().cpu().numpy()
    for t in range(1, 4):
        g = r.normal(size=112).astype(np.float32)
        a.grads.copy_(torch.from_numpy(g))
        a.step()
        m, v = 0.9 * m + 0.1 * g, 0.999 * v + 0.001 * g.astype(np.float64) ** 2
        x = x - 1e-2 / (1 - 0.9 ** t) * m / (np.sqrt(v / (1 - 0.999 ** t)) + 1e-8)
    ctx.sync()
    np.testing.assert_allclose(a.values.double().cpu().numpy(), x, rtol=1e-5, atol=1e-6)
