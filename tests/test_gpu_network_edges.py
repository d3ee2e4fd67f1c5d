"""The network operators where they can go wrong: rows without spread, tails of the activations, calls
between a pass and its backward pass, other streams, waits that run out."""
import math

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


# ---- gated feed-forward

def gelu_parts(z):
    """Phi(z), z phi(z) and what 32 bits may add to each, relative to itself.  z^2 / 2 is rounded three
    times on its way into an exponential (or into erfc, whose logarithm falls like it): 2^-24 z^2 / 2 each
    and so at most 0.7 z^2 EPS; the functions and products are good to 12 EPS."""
    cdf = 0.5 * np.vectorize(math.erfc)(-z / math.sqrt(2.0))
    return cdf, z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi), (0.7 * z * z + 12) * N.EPS


# 16-bit matrices: the tail's polynomial, 1.8e-5 of itself
TAIL = {"f32": 0.0, "f16": 1.8e-5, "bf16": 1.8e-5}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [5, 300, 3000])
def test_gelu_far_below_zero(ctx, kind, rows):
    """gelu of -8 ... -3 is as small as 1e-15, and as exact as elsewhere relative to itself: through
    unit matrices, so that y is the hidden matrix, whose up projection is large."""
    d = 64
    r = np.random.default_rng(rows)
    x = matrix(r.uniform(-8, -3, (rows, d)), kind)
    one = matrix(np.eye(d), kind)
    y = blank(rows, d, kind)
    ctx.reserve_network(rows, d, d, TYPES[kind])
    ab.abcd_gated_ff(ctx, x, one, matrix(1024 * np.eye(d), kind), one, "gelu", y)
    ctx.sync()
    z = f64(x)
    cdf, _, rel = gelu_parts(z)
    want = z * cdf * 1024 * z
    wide = np.abs(want) * (rel + TAIL[kind])
    # rounded to the type as the hidden matrix; as y it is a value of the type already
    close(y, want, wide + (np.abs(want) + wide) * N.UNIT[kind] + N.TINY[kind])


@pytest.mark.parametrize("kind", KINDS)
def test_gelu_far_below_zero_backward(ctx, kind):
    """The same for dG and dU, which unit matrices hand on as the weights' gradients."""
    d = 64
    r = np.random.default_rng(41)
    gate, up = matrix(r.uniform(-8, -3, (d, d)), kind), matrix(np.full((d, d), 2048.0), kind)
    one, dy = matrix(np.eye(d), kind), matrix(np.eye(d), kind)
    down = matrix(np.ones((d, d)), kind)
    dwg, dwu, dwd = (blank(d, d, kind) for _ in range(3))
    ctx.reserve_network(d, d, d, TYPES[kind])
    ab.abcd_gated_ff_backward(ctx, dy, one, one, one, down, "gelu", gate, up, None, dwg, dwu, dwd)
    ctx.sync()
    z = f64(gate)
    cdf, zphi, rel = gelu_parts(z)
    rel = rel + TAIL[kind]
    for got, want, mag in ((dwg.T, 2048 * (cdf + zphi), 2048 * (cdf + np.abs(zphi))), (dwu.T, z * cdf, np.abs(z) * cdf),
                           (dwd, 2048 * z * cdf, 2048 * np.abs(z) * cdf)):
        wide = mag * rel
        close(got, want, wide + (np.abs(want) + wide) * N.UNIT[kind] + N.TINY[kind])


# ---- the block

@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_block_evaluated_between_a_pass_and_its_backward_pass(ctx, kind):
    """The gradients are those of the last training pass, whatever was evaluated since."""
    r = np.random.default_rng(31)
    n, d, f = 60, 28, 112
    w = {"norm_w": torch.as_tensor(r.normal(1, 0.1, d)).to("cuda", TYPES[kind]),
         "norm_b": torch.as_tensor(r.normal(0, 0.1, d)).to("cuda", TYPES[kind]),
         "w_gate": matrix(r.normal(0, d ** -0.5, (f, d)), kind),
         "w_up": matrix(r.normal(0, d ** -0.5, (f, d)), kind),
         "w_down": matrix(r.normal(0, f ** -0.5, (d, f)), kind)}
    x, other, dy = (matrix(r.normal(size=(n, d)), kind) for _ in range(3))
    block = ab.FeedForwardBlock(ctx, w, n, p=0.2, seed=3)
    found = []
    for between in (False, True):
        y, dx, seen = (blank(n, d, kind) for _ in range(3))
        block.offset = 0                                # the same mask again
        block.forward(x, y)
        if between:
            block.forward(other, seen, train=False)
        block.backward(dy, x, dx)
        ctx.sync()
        found.append([t.clone() for t in (y, dx, *block.grads.values())])
    assert all(torch.equal(a, b) for a, b in zip(*found))


def test_appearance_evaluated_between_a_pass_and_its_backward_pass():
    from paper_2608_27735_gb300.appearance import Appearance
    ctx = ab.Context(0)
    app = Appearance(ctx, 150, 1, 3, layers=2, embed=5, p=0.3, seed=4)
    r = np.random.default_rng(1)
    for b in app.blocks:
        b.w["w_down"].copy_(torch.from_numpy(r.normal(0, 0.1, b.w["w_down"].shape).astype(np.float32)))
    sh, other, d = (torch.from_numpy(r.normal(size=(150, 4, 3)).astype(np.float32)).cuda() for _ in range(3))
    found = []
    for between in (False, True):
        for b in app.blocks:
            b.offset = 0
        seen = app.forward(sh, 1)
        if between:
            app.forward(other, 2, train=False)
        d_sh = app.backward(d, 1)
        ctx.sync()
        found.append((seen.clone(), d_sh.clone(), app.adam.grads.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*found))
    # and the evaluation is that of the layers: without dropout both are one
    plain = Appearance(ctx, 150, 1, 3, layers=2, embed=5, p=0.0, seed=4)
    plain.adam.values.copy_(app.adam.values)
    assert torch.equal(plain.forward(sh, 2, train=False), plain.forward(sh, 2))


# ---- streams

def pending(nbytes, value=255):
    """Queues a wait of some ten milliseconds on the current stream and, behind it, a kernel that fills
    nbytes with a value; gives the memory back at once.  Whoever gets it next has to wait for both."""
    torch.cuda.empty_cache()
    t = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    torch.cuda._sleep(40_000_000)
    t.fill_(value)
    return t.data_ptr()


@pytest.mark.parametrize("kind", KINDS)
def test_workspace_reserved_while_its_memory_is_written(kind):
    """A context on a stream of its own, whose workspace the allocator takes from memory that the
    current stream is still writing: the products' counters and sums are not written over."""
    from .test_gpu_network import everything, flat, make_everything
    n, d, f = 700, 264, 520
    args, out = make_everything(n, d, f, kind, 23)
    plain = ab.Context(0)
    plain.reserve_network(n, d, f, TYPES[kind])
    everything(plain, *args, out)
    plain.sync()
    want = flat(out)
    nbytes = plain.network_bytes + 256
    del plain
    for t in (*out[:-1], *out[-1]):
        t.fill_(float("nan"))
    torch.cuda.synchronize()
    side = ab.Context(0, torch.cuda.Stream())
    at = pending(nbytes)
    side.reserve_network(n, d, f, TYPES[kind])
    assert side.network_workspace.data_ptr() == at
    everything(side, *args, out)
    side.sync()
    assert all(torch.equal(a, b) for a, b in zip(flat(out), want))


def test_block_made_and_dropped_while_its_memory_is_in_use():
    """On a stream of the context's own: a block's buffers come from memory that the current stream
    still writes, and go back while the block's calls still run."""
    r = np.random.default_rng(33)
    n, d, f = 4000, 64, 256
    make = lambda: {"norm_w": torch.ones(d, device="cuda"), "norm_b": torch.zeros(d, device="cuda"),
                    **{k: matrix(r.normal(0, 0.1, s), "f32") for k, s in
                       (("w_gate", (f, d)), ("w_up", (f, d)), ("w_down", (d, f)))}}
    w, x, dy = make(), matrix(r.normal(size=(n, d)), "f32"), matrix(r.normal(size=(n, d)), "f32")

    def once(ctx, wait):
        y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
        torch.cuda.synchronize()
        if wait:
            pending(8 * n * f * 4)                      # more than the block takes
        block = ab.FeedForwardBlock(ctx, w, n, p=0.2, seed=3)
        if wait:
            with torch.cuda.stream(ctx.stream):
                torch.cuda._sleep(40_000_000)           # the calls have yet to run when the block goes
        block.forward(x, y)
        block.backward(dy, x, dx)
        del block
        if wait:
            others = [torch.full((n * d,), float("nan"), device="cuda") for _ in range(64)]
            del others
        ctx.sync()
        torch.cuda.synchronize()
        return y, dx

    y, dx = once(ab.Context(0), False)
    side = ab.Context(0, torch.cuda.Stream())
    side.reserve_network(n, d, f)
    y2, dx2 = once(side, True)
    assert torch.equal(y, y2) and torch.equal(dx, dx2)


# ---- waits

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,d,f", [(77, 64, 130), (3001, 72, 1032), (20000, 256, 1024)])
def test_waits_that_run_out_in_part(kind, n, d, f):
    """With few polls some waits of the products give up and others do not: the calls end, and once the
    limit is back and the status cleared they are right again.  (Which waits give up is a matter of
    chance, and so is whether the status says so.)"""
    from .test_gpu_network import everything, flat, make_everything
    args, out = make_everything(n, d, f, kind, 24)
    c = ab.Context(0)
    c.reserve_network(n, d, f, TYPES[kind])
    everything(c, *args, out)
    c.sync()
    want = flat(out)
    x, dy, w, wg, wu, wd = args
    for polls in (1, 2, 3, 5, 10, 30, 100, 300):
        assert ab.lib().abcd_set_wait_limit(c.h, polls) == ab.ABCD_OK
        ab.abcd_gated_ff(c, x, wg, wu, wd, "silu", out[0], out[1], out[2])
        ab.abcd_gated_ff_backward(c, dy, x, wg, wu, wd, "silu", out[1], out[2], out[5], *out[-1])
        try:
            c.sync()
        except ab.AbcdError as e:
            assert e.status == ab.ABCD_ERR_TIMEOUT
        c.clear_status()
    assert ab.lib().abcd_set_wait_limit(c.h, 1 << 20) == ab.ABCD_OK
    everything(c, *args, out)
    c.sync()
    assert all(torch.equal(a, b) for a, b in zip(flat(out), want))


# ---- refusals

@pytest.mark.parametrize("kind", KINDS)
def test_ff_refuses_outputs_that_overlap_in_part(ctx, kind):
    """An output that reaches into an operand or another output is refused wherever it starts; columns
    of one buffer next to each other are taken."""
    n, d, f = 20, 24, 40
    buf = torch.zeros(300, 400, dtype=TYPES[kind], device="cuda")
    at = lambda rows, cols, row, col: buf[row:row + rows, col:col + cols]
    x, wg, wu, wd = at(n, d, 0, 0), at(f, d, 0, 24), at(f, d, 0, 48), at(d, f, 0, 72)
    y, gate, up = at(n, d, 0, 112), at(n, f, 0, 136), at(n, f, 0, 176)
    dy, dx = at(n, d, 0, 216), at(n, d, 0, 240)
    dwg, dwu, dwd = at(f, d, 0, 264), at(f, d, 0, 288), at(d, f, 0, 312)
    ctx.reserve_network(n, d, f, TYPES[kind])
    forward = lambda y, gate, up: ab.abcd_gated_ff(ctx, x, wg, wu, wd, "silu", y, gate, up)
    backward = lambda *g: ab.abcd_gated_ff_backward(ctx, dy, x, wg, wu, wd, "silu", gate, up, *g)
    forward(y, gate, up)
    forward(x, gate, up)
    backward(dx, dwg, dwu, dwd)
    ctx.sync()
    x.zero_()
    for call, args in ((forward, (at(n, d, 3, 25), gate, up)),          # y in w_gate
                       (forward, (y, at(n, f, 19, 100), up)),           # gate's first row in w_down's
                       (forward, (y, gate, at(n, f, 1, 137))),          # up in gate
                       (forward, (y, at(n, f, 10, 111), up)),           # gate in y
                       (backward, (at(n, d, 19, 216), dwg, dwu, dwd)),  # dx's first row in dy's last
                       (backward, (at(n, d, 0, 239), dwg, dwu, dwd)),   # dx by one column
                       (backward, (dx, at(f, d, 39, 288), dwu, dwd)),   # dw_gate in dw_up
                       (backward, (dx, dwg, dwu, at(d, f, 0, 311)))):   # dw_down in dw_up by one column
        with pytest.raises(ab.AbcdError) as e:
            call(*args)
        assert e.value.status == ab.ABCD_ERR_INVALID_ARG
    backward(at(n, d, 20, 216), dwg, dwu, dwd)                          # right below dy
    ctx.sync()


def test_block_refuses_a_backward_pass_without_its_pass(ctx):
    r = np.random.default_rng(35)
    w = {"norm_w": torch.ones(24, device="cuda"), "norm_b": torch.zeros(24, device="cuda"),
         **{k: matrix(r.normal(size=s), "f32") for k, s in (("w_gate", (40, 24)), ("w_up", (40, 24)), ("w_down", (24, 40)))}}
    block = ab.FeedForwardBlock(ctx, w, 50)
    x, y = matrix(r.normal(size=(20, 24)), "f32"), blank(20, 24, "f32")
    with pytest.raises(ValueError):
        block.backward(x, x, y)
    block.forward(x, y, train=False)
    with pytest.raises(ValueError):
        block.backward(x, x, y)
    block.forward(x, y)
    with pytest.raises(ValueError):
        block.backward(x[:10], x[:10], y[:10])
    block.backward(x, x, y)
    ctx.sync()


# ---- long and many rows

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(900, 17003), (1000, 9001), (1500, 4097), (3000, 1100), (6000, 520), (20000, 59)])
@pytest.mark.parametrize("pad,lead", [(0, 0), (5, 3), (16, 8)])
def test_norm_of_many_rows(ctx, kind, rows, cols, pad, lead):
    """Several rows per CTA at every row length (rows ahead, barriers and sums used again), and dx over the
    residual's gradient."""
    r = np.random.default_rng(rows + cols)
    x = matrix(r.normal(0.5, 1, (rows, cols)), kind, pad, lead)
    dy = matrix(r.normal(0, 0.3, (rows, cols)), kind, pad, lead)
    res = matrix(r.normal(size=(rows, cols)), kind, pad, lead)
    w = torch.as_tensor(r.normal(1, 0.3, cols)).to("cuda", TYPES[kind])
    X, DY, R, W = f64(x), f64(dy), f64(res), f64(w)
    y = blank(rows, cols, kind, pad, lead)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dw, db = torch.full_like(w, float("nan")), torch.full_like(w, float("nan"))
    ctx.reserve_network(rows, cols)
    ab.abcd_layer_norm(ctx, x, w, None, 1e-5, y, mean, rstd)
    ab.abcd_layer_norm_backward(ctx, dy, x, w, mean, rstd, res, dw, db, res)
    ctx.sync()
    close(y, N.norm(X, W, 0 * W, 1e-5)[0], N.norm_bound(X, W, 0 * W, 1e-5, kind))
    m32, r32 = f64(mean)[:, None], f64(rstd)[:, None]
    bounds = N.norm_grad_bounds(DY, X, W, m32, r32, kind, kind, R)
    want = N.norm_grad(DY, X, W, m32, r32)
    for got, exact, bound in zip((res, dw, db), (want[0] + R, *want[1:]), bounds):
        close(got, exact, bound)
