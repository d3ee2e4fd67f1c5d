"""The network operators on the GPU against their 64-bit formulas, within forward error bounds that
are computed from the inputs (tests/_network.py)."""
import numpy as np
import pytest

import paper_2608_27735_gb300 as ab

from . import _network as N

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
KINDS = ["f32", "f16", "bf16"]


@pytest.fixture(scope="module")
def ctx():
    ab.build()
    return ab.Context(0)


def matrix(a, kind, pad=0, lead=0):
    """A CUDA matrix with the values of a, rows `pad` elements further apart than they are long and
    the first one `lead` elements into its buffer; what lies between is NaN."""
    rows, cols = a.shape
    buf = torch.full((rows * (cols + pad) + lead,), float("nan"), dtype=TYPES[kind], device="cuda")
    t = buf[lead:].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.as_tensor(np.ascontiguousarray(a)))
    return t


def blank(rows, cols, kind, pad=0, lead=0):
    return matrix(np.full((rows, cols), np.nan), kind, pad, lead)


def f64(t):
    return t.double().cpu().numpy()


def gaps_untouched(t):
    """Whether the elements between the rows of a matrix() are still NaN."""
    base = t._base if t._base is not None else t
    rows, cols = t.shape
    full = base.reshape(-1)[t.storage_offset():].view(rows, -1)
    return bool(torch.isnan(full[:, cols:]).all()) and bool(torch.isnan(base.reshape(-1)[:t.storage_offset()]).all())


def close(got, want, bound):
    got = f64(got)
    assert got.shape == want.shape
    assert np.isfinite(got).all()
    bad = np.abs(got - want) > bound
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], bound[bad][:4])


# ---- layer norm

NORM_SHAPES = [(1, 1), (1, 8), (3, 59), (5, 64), (2, 250), (7, 256), (33, 257), (2, 1000),
               (1, 1024), (1201, 16), (700, 59), (3, 4096), (2, 5001), (1, 33000)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("pad,lead", [(0, 0), (5, 3), (16, 8)])
def test_norm(ctx, kind, rows, cols, pad, lead):
    r = np.random.default_rng(rows * 7 + cols)
    wkind = "f32" if pad == 16 else kind
    x = matrix(r.normal(0.5, 1, (rows, cols)) * np.exp(r.normal(0, 1, (rows, 1))), kind, pad, lead)
    dy = matrix(r.normal(0, 0.3, (rows, cols)), kind, pad, lead)
    w = torch.as_tensor(r.normal(1, 0.3, cols)).to("cuda", TYPES[wkind])
    b = torch.as_tensor(r.normal(0, 0.3, cols)).to("cuda", TYPES[wkind])
    y, dx = blank(rows, cols, kind, pad, lead), blank(rows, cols, kind, pad, lead)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dw, db = torch.full_like(w, float("nan")), torch.full_like(b, float("nan"))
    ctx.reserve_network(rows, cols)
    ab.abcd_layer_norm(ctx, x, w, b, 1e-5, y, mean, rstd)
    ab.abcd_layer_norm_backward(ctx, dy, x, w, mean, rstd, dx, dw, db)
    ctx.sync()
    X, W, B, DY = f64(x), f64(w), f64(b), f64(dy)
    want, m64, r64 = N.norm(X, W, B, 1e-5)
    close(y, want, N.norm_bound(X, W, B, 1e-5, kind))
    k = (cols + 8) * N.EPS
    mag = np.abs(X).mean(1)
    assert (np.abs(f64(mean) - m64[:, 0]) <= k * mag + 1e-30).all()
    assert (np.abs(f64(rstd) / r64[:, 0] - 1) <= k * (2 + 4 * (mag * r64[:, 0]) ** 2)).all()
    # the backward pass from the statistics that it was given
    m32, r32 = f64(mean)[:, None], f64(rstd)[:, None]
    bounds = N.norm_grad_bounds(DY, X, W, m32, r32, kind, wkind)
    for got, exact, bound in zip((dx, dw, db), N.norm_grad(DY, X, W, m32, r32), bounds):
        close(got, exact, bound)
    assert gaps_untouched(y) and gaps_untouched(dx)


@pytest.mark.parametrize("cols", [59, 64, 1024])
def test_norm_without_weights_in_place_and_with_a_residual(ctx, cols):
    r = np.random.default_rng(3)
    x = matrix(r.normal(size=(40, cols)), "f32")
    X = f64(x)
    mean, rstd = torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
    dy, res = matrix(r.normal(size=(40, cols)), "f32"), matrix(r.normal(size=(40, cols)), "f32")
    DY, R = f64(dy), f64(res)
    y = blank(40, cols, "f32")
    ctx.reserve_network(40, cols)
    ab.abcd_layer_norm(ctx, x, None, None, 1e-5, y, mean, rstd)
    close(y, N.norm(X, 1.0, 0.0, 1e-5)[0], N.norm_bound(X, np.ones(cols), np.zeros(cols), 1e-5, "f32"))
    one = np.ones(cols)
    m32, r32 = f64(mean)[:, None], f64(rstd)[:, None]
    want = N.norm_grad(DY, X, one, m32, r32)
    bounds = N.norm_grad_bounds(DY, X, one, m32, r32, "f32", "f32", R)
    dw = torch.empty(cols, device="cuda")
    ab.abcd_layer_norm_backward(ctx, dy, x, None, mean, rstd, None, dw)          # the sums alone
    close(dw, want[1], bounds[1])
    ab.abcd_layer_norm_backward(ctx, dy, x, None, mean, rstd, res, d_residual=res)   # over its residual
    close(res, want[0] + R, bounds[0])
    ab.abcd_layer_norm_backward(ctx, dy, x, None, mean, rstd, dy)                # over dy
    close(dy, want[0], bounds[0])
    ab.abcd_layer_norm(ctx, x, None, None, 1e-5, x)                              # over x
    close(x, N.norm(X, 1.0, 0.0, 1e-5)[0], N.norm_bound(X, one, 0 * one, 1e-5, "f32"))


def test_norm_of_constant_rows_and_far_from_zero(ctx):
    """A row without spread is its bias; a mean of 1000 spreads costs no digits of the variance."""
    r = np.random.default_rng(5)
    x = matrix(np.concatenate([np.full((2, 96), 3.0), r.normal(1000, 1, (2, 96))]), "f32")
    w, b = torch.full((96,), 2.0, device="cuda"), torch.full((96,), 0.25, device="cuda")
    y = blank(4, 96, "f32")
    ab.abcd_layer_norm(ctx, x, w, b, 1e-5, y)
    assert (f64(y)[:2] == 0.25).all()
    X = f64(x)
    close(y, N.norm(X, f64(w), f64(b), 1e-5)[0], N.norm_bound(X, f64(w), f64(b), 1e-5, "f32"))


def test_norm_of_constant_rows_backward(ctx):
    """Without spread xh is zero, whatever the rows' values: the weight gets no gradient."""
    x = matrix(np.repeat([[1000.0], [-37.5], [0.0]], 64, 1), "f32")
    dy = matrix(np.random.default_rng(15).normal(size=(3, 64)), "f32")
    mean, rstd, y = torch.empty(3, device="cuda"), torch.empty(3, device="cuda"), blank(3, 64, "f32")
    dw, dx = torch.full((64,), float("nan"), device="cuda"), blank(3, 64, "f32")
    ctx.reserve_network(3, 64)
    ab.abcd_layer_norm(ctx, x, None, None, 1e-5, y, mean, rstd)
    ab.abcd_layer_norm_backward(ctx, dy, x, None, mean, rstd, dx, dw)
    ctx.sync()
    assert not y.any() and not dw.any()


def test_norm_keeps_a_bad_row_to_itself(ctx):
    x = matrix(np.random.default_rng(6).normal(size=(6, 64)), "f32")
    want = blank(6, 64, "f32")
    ab.abcd_layer_norm(ctx, x, None, None, 1e-5, want)
    x[2, 5], x[4, 0] = float("nan"), float("inf")
    y = blank(6, 64, "f32")
    ab.abcd_layer_norm(ctx, x, None, None, 1e-5, y)
    good = [0, 1, 3, 5]
    assert torch.equal(y[good], want[good]) and torch.isnan(y[[2, 4]]).all()


# ---- gated feed-forward

FF_SHAPES = [(1, 1, 1), (1, 64, 128), (2, 59, 77), (7, 64, 256), (129, 64, 128), (130, 250, 999),
             (300, 33, 513), (257, 256, 64), (64, 520, 136), (16, 1024, 512), (1500, 8, 16),
            (3001, 72, 1032), (2900, 136, 1100)]


def ff_weights(r, d, f, kind, pad, lead):
    return (matrix(r.normal(0, d ** -0.5, (f, d)), kind, pad, lead),
            matrix(r.normal(0, d ** -0.5, (f, d)), kind, pad, lead),
            matrix(r.normal(0, f ** -0.5, (d, f)), kind, pad, lead))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,d,f", FF_SHAPES)
@pytest.mark.parametrize("pad,lead", [(0, 0), (5, 3), (16, 8)])
def test_ff(ctx, kind, rows, d, f, pad, lead):
    r = np.random.default_rng(rows + 3 * d + 5 * f)
    name = ("silu", "gelu", "relu")[(rows + d + f + pad) % 3]
    x = matrix(r.normal(size=(rows, d)), kind, pad, lead)
    wg, wu, wd = ff_weights(r, d, f, kind, pad, lead)
    y = blank(rows, d, kind, pad, lead)
    gate, up = blank(rows, f, kind, pad, lead), blank(rows, f, kind, pad, lead)
    ctx.reserve_network(rows, d, f, TYPES[kind])
    ab.abcd_gated_ff(ctx, x, wg, wu, wd, name, y, gate, up)
    alone = blank(rows, d, kind, pad, lead)
    ab.abcd_gated_ff(ctx, x, wg, wu, wd, name, alone)
    ctx.sync()
    A = [f64(t) for t in (x, wg, wu, wd)]
    for got, want, bound in zip((y, gate, up), N.ff(*A, name), N.ff_bounds(*A, name, kind)):
        close(got, want, bound)
        assert gaps_untouched(got)
    assert torch.equal(alone, y)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,d,f", FF_SHAPES)
@pytest.mark.parametrize("pad,lead", [(0, 0), (5, 3), (16, 8)])
def test_ff_backward(ctx, kind, rows, d, f, pad, lead):
    r = np.random.default_rng(rows + 3 * d + 5 * f + 1)
    name = ("silu", "gelu", "relu")[(rows + d + f + pad + 1) % 3]
    x, dy = matrix(r.normal(size=(rows, d)), kind, pad, lead), matrix(r.normal(size=(rows, d)), kind, pad, lead)
    wg, wu, wd = ff_weights(r, d, f, kind, pad, lead)
    # the projections that the forward pass leaves, as values of the type
    _, z, u = N.ff(f64(x), f64(wg), f64(wu), f64(wd), name)
    gate, up = matrix(z, kind, pad, lead), matrix(u, kind, pad, lead)
    dx = blank(rows, d, kind, pad, lead)
    dwg, dwu, dwd = blank(f, d, kind, pad, lead), blank(f, d, kind, pad, lead), blank(d, f, kind, pad, lead)
    ctx.reserve_network(rows, d, f, TYPES[kind])
    ab.abcd_gated_ff_backward(ctx, dy, x, wg, wu, wd, name, gate, up, dx, dwg, dwu, dwd)
    ctx.sync()
    args = [f64(dy), f64(x), f64(wg), f64(wu), f64(wd), name, f64(gate), f64(up)]
    for got, want, bound in zip((dx, dwg, dwu, dwd), N.ff_grad(*args), N.ff_grad_bounds(*args, kind)):
        close(got, want, bound)
        assert gaps_untouched(got)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("want", [(1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (0, 1, 0, 1)])
def test_ff_backward_of_some(ctx, kind, want):
    """The gradients that are asked for are the ones of the whole call."""
    r = np.random.default_rng(8)
    x, dy = matrix(r.normal(size=(150, 72)), kind), matrix(r.normal(size=(150, 72)), kind)
    wg, wu, wd = ff_weights(r, 72, 200, kind, 0, 0)
    gate, up = matrix(r.normal(size=(150, 200)), kind), matrix(r.normal(size=(150, 200)), kind)
    ctx.reserve_network(150, 72, 200, TYPES[kind])
    shapes = [(150, 72), (200, 72), (200, 72), (72, 200)]
    every = [blank(*s, kind) for s in shapes]
    some = [blank(*s, kind) if k else None for s, k in zip(shapes, want)]
    ab.abcd_gated_ff_backward(ctx, dy, x, wg, wu, wd, "silu", gate, up, *every)
    ab.abcd_gated_ff_backward(ctx, dy, x, wg, wu, wd, "silu", gate, up, *some)
    ctx.sync()
    for a, b in zip(every, some):
        assert b is None or torch.equal(a, b)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [5, 300])
def test_ff_over_its_input(ctx, kind, rows):
    r = np.random.default_rng(14)
    x = matrix(r.normal(size=(rows, 64)), kind)
    wg, wu, wd = ff_weights(r, 64, 130, kind, 0, 0)
    ctx.reserve_network(rows, 64, 130, TYPES[kind])
    y = blank(rows, 64, kind)
    ab.abcd_gated_ff(ctx, x, wg, wu, wd, "silu", y)
    ab.abcd_gated_ff(ctx, x, wg, wu, wd, "silu", x)
    ctx.sync()
    assert torch.equal(x, y)


@pytest.mark.parametrize("kind", KINDS)
def test_without_rows(ctx, kind):
    e = torch.empty(0, 24, dtype=TYPES[kind], device="cuda")
    h = torch.empty(0, 40, dtype=TYPES[kind], device="cuda")
    r = np.random.default_rng(1)
    wg, wu, wd = ff_weights(r, 24, 40, kind, 0, 0)
    ctx.reserve_network(1, 24, 40, TYPES[kind])
    ab.abcd_gated_ff(ctx, e, wg, wu, wd, "silu", e.clone(), h, h.clone())
    g = [blank(40, 24, kind), blank(40, 24, kind), blank(24, 40, kind)]
    ab.abcd_gated_ff_backward(ctx, e, e, wg, wu, wd, "silu", h, h, e.clone(), *g)
    w = torch.ones(24, dtype=TYPES[kind], device="cuda")
    s = torch.empty(0, device="cuda")
    dw, db = torch.full_like(w, 7.0), torch.full_like(w, 7.0)
    ab.abcd_layer_norm(ctx, e, w, w, 1e-5, e.clone(), s, s)
    ab.abcd_layer_norm_backward(ctx, e, e, w, s, s, e.clone(), dw, db)
    ab.abcd_dropout(ctx, e, 0.5, 1, 2, e.clone())
    ctx.sync()
    assert all((t == 0).all() for t in (*g, dw, db))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,d,f", [(3, 64, 96), (300, 256, 640)])
def test_ff_keeps_a_bad_token_to_itself(ctx, kind, rows, d, f):
    """NaN and infinity in one token reach that token's outputs alone (and, backward, its dx)."""
    r = np.random.default_rng(9)
    x, dy = matrix(r.normal(size=(rows, d)), kind), matrix(r.normal(size=(rows, d)), kind)
    wg, wu, wd = ff_weights(r, d, f, kind, 0, 0)
    ctx.reserve_network(rows, d, f, TYPES[kind])
    outs = []
    for bad in (False, True):
        if bad:
            x[1, 3], dy[1, 5] = float("nan"), float("inf")
        y, gate, up, dx = (blank(rows, c, kind) for c in (d, f, f, d))
        ab.abcd_gated_ff(ctx, x, wg, wu, wd, "silu", y, gate, up)
        ab.abcd_gated_ff_backward(ctx, dy, x, wg, wu, wd, "silu", gate, up, dx)
        outs.append((y, dx))
    ctx.sync()
    others = [k for k in range(rows) if k != 1]
    for a, b in zip(*outs):
        assert torch.equal(a[others], b[others]) and torch.isnan(b[1]).all()


@pytest.mark.parametrize("kind", KINDS)
def test_results_are_the_same_every_time(ctx, kind):
    """No result depends on the order in which CTAs run."""
    r = np.random.default_rng(10)
    n, d, f = 5000, 72, 96
    x, dy = matrix(r.normal(size=(n, d)), kind), matrix(r.normal(size=(n, d)), kind)
    wg, wu, wd = ff_weights(r, d, f, kind, 0, 0)
    w = torch.ones(d, dtype=TYPES[kind], device="cuda")
    ctx.reserve_network(n, d, f, TYPES[kind])
    first = None
    for _ in range(4):
        y, gate, up, dx, nx, dn = (blank(n, c, kind) for c in (d, f, f, d, d, d))
        g = [blank(f, d, kind), blank(f, d, kind), blank(d, f, kind)]
        mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        dw, db = torch.empty_like(w), torch.empty_like(w)
        ab.abcd_layer_norm(ctx, x, w, w, 1e-5, nx, mean, rstd)
        ab.abcd_gated_ff(ctx, nx, wg, wu, wd, "gelu", y, gate, up)
        ab.abcd_gated_ff_backward(ctx, dy, nx, wg, wu, wd, "gelu", gate, up, dx, *g)
        ab.abcd_layer_norm_backward(ctx, dx, x, w, mean, rstd, dn, dw, db)
        ctx.sync()
        got = [y, dx, dn, dw, db, *g]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


# ---- dropout

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 1024), (3, 59), (40, 64), (17, 250), (2, 7), (1001, 3)])
@pytest.mark.parametrize("pad,lead", [(0, 0), (5, 3), (16, 8)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(ctx, kind, rows, cols, pad, lead, p):
    r = np.random.default_rng(rows + cols)
    seed, offset = 0x1234567890ABCDEF, (1 << 32) - 3
    x = matrix(r.choice([-1, 1], (rows, cols)) * r.uniform(0.5, 2, (rows, cols)), kind, pad, lead)
    res = matrix(r.normal(size=(rows, cols)), kind, pad, lead)
    y, z, dx = (blank(rows, cols, kind, pad, lead) for _ in range(3))
    ab.abcd_dropout(ctx, x, p, seed, offset, y)
    ab.abcd_dropout(ctx, x, p, seed, offset, z, res)
    ab.abcd_dropout_backward(ctx, x, p, seed, offset, dx)
    ctx.sync()
    keep, s = N.kept(rows, cols, p, seed, offset)
    X, R = f64(x), f64(res)
    assert ((f64(y) != 0) == keep).all()
    # the scale and the product are rounded to 32 bits, the sum once more
    bound = lambda v, mag: 3 * N.EPS * mag + (np.abs(v) + 3 * N.EPS * mag) * N.UNIT[kind] + N.TINY[kind]
    want = keep * X * s
    close(y, want, bound(want, np.abs(want)))
    close(z, want + R, bound(want + R, np.abs(want) + np.abs(R)))
    assert torch.equal(y, dx)
    assert gaps_untouched(y) and gaps_untouched(z)


def test_dropout_in_place_and_of_bad_values(ctx):
    """y over x or over the residual; a dropped NaN or infinity is dropped."""
    r = np.random.default_rng(2)
    x, res = matrix(r.normal(size=(9, 64)), "f32"), matrix(r.normal(size=(9, 64)), "f32")
    y = blank(9, 64, "f32")
    ab.abcd_dropout(ctx, x, 0.5, 11, 0, y, res)
    a, b = x.clone(), res.clone()
    ab.abcd_dropout(ctx, a, 0.5, 11, 0, a, res)
    ab.abcd_dropout(ctx, x, 0.5, 11, 0, b, b)
    assert torch.equal(a, y) and torch.equal(b, y)
    keep, _ = N.kept(9, 64, 0.5, 11, 0)
    x[torch.as_tensor(~keep).cuda()] = float("nan")
    ab.abcd_dropout(ctx, x, 0.5, 11, 0, a, res)
    assert torch.equal(a, y)


def test_dropout_of_consecutive_offsets_is_one_stream(ctx):
    """Rows whose length is a multiple of eight: the mask of a part is the part of the mask."""
    x = torch.ones(32, 64, device="cuda")
    whole, part = torch.empty_like(x), torch.empty_like(x)
    ab.abcd_dropout(ctx, x, 0.3, 5, 100, whole)
    ab.abcd_dropout(ctx, x[:12], 0.3, 5, 100, part[:12])
    ab.abcd_dropout(ctx, x[12:], 0.3, 5, 100 + 12 * 8, part[12:])
    assert torch.equal(whole, part)


# ---- long matrices

def far(rows, cols, kind, pad=0):
    """A CUDA matrix of normal numbers."""
    buf = torch.empty(rows, cols + pad, dtype=TYPES[kind], device="cuda")
    return buf.normal_(0, 1)[:, :cols]


def some_rows(rows, width):
    """Rows at both ends and around the ones that start at elements 2^31 and 2^32 of rows `width` long."""
    near = [0, 1, rows - 2, rows - 1] + [e // width + k for e in (2 ** 31, 2 ** 32) for k in (0, 1)]
    return sorted({k for k in near if k < rows})


def only(rows, cols, kind, chosen):
    """Zeros but in the chosen rows."""
    t = torch.zeros(rows, cols, dtype=TYPES[kind], device="cuda")
    t[chosen] = torch.randn(len(chosen), cols, device="cuda").to(t.dtype)
    return t


@pytest.fixture
def roomy():
    """A context of its own, whose workspace is given back, and room for large matrices."""
    torch.cuda.empty_cache()
    torch.manual_seed(4)
    c = ab.Context(0)
    yield c
    c.sync()
    del c
    torch.cuda.empty_cache()


@pytest.mark.parametrize("pad", [0, 3])
def test_norm_past_32_bits(roomy, pad):
    rows, cols, kind = 4_300_007, 1000, "f16"
    chosen = some_rows(rows, cols + pad)
    x, dy = far(rows, cols, kind, pad), only(rows, cols, kind, chosen)
    w = torch.randn(cols, device="cuda")
    y, dx = torch.full_like(dy, float("nan")), torch.full_like(dy, float("nan"))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dw, db = torch.empty_like(w), torch.empty_like(w)
    roomy.reserve_network(rows, cols)
    ab.abcd_layer_norm(roomy, x, w, None, 1e-5, y, mean, rstd)
    ab.abcd_layer_norm_backward(roomy, dy, x, w, mean, rstd, dx, dw, db)
    roomy.sync()
    assert torch.isfinite(y.sum(1, dtype=torch.float32)).all()
    X, DY, W = f64(x[chosen]), f64(dy[chosen]), f64(w)
    close(y[chosen], N.norm(X, W, 0 * W, 1e-5)[0], N.norm_bound(X, W, 0 * W, 1e-5, kind))
    m32, r32 = f64(mean[chosen])[:, None], f64(rstd[chosen])[:, None]
    bounds = N.norm_grad_bounds(DY, X, W, m32, r32, kind, "f32")     # the other rows add zeros
    for got, want, bound in zip((dx[chosen], dw, db), N.norm_grad(DY, X, W, m32, r32), bounds):
        close(got, want, bound)
    dx[chosen] = 0
    assert not dx.any()


@pytest.mark.parametrize("kind,rows,d,f", [("f16", 4_300_007, 64, 1000), ("f32", 2_200_003, 40, 1000)])
def test_ff_past_32_bits(roomy, kind, rows, d, f):
    chosen = some_rows(rows, f)
    x, dy = far(rows, d, kind), only(rows, d, kind, chosen)
    wg, wu, wd = ff_weights(np.random.default_rng(2), d, f, kind, 0, 0)
    y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    gate, up = (torch.empty(rows, f, dtype=x.dtype, device="cuda") for _ in range(2))
    grads = [torch.full_like(t, float("nan")) for t in (wg, wu, wd)]
    roomy.reserve_network(rows, d, f, TYPES[kind])
    ab.abcd_gated_ff(roomy, x, wg, wu, wd, "silu", y, gate, up)
    ab.abcd_gated_ff_backward(roomy, dy, x, wg, wu, wd, "silu", gate, up, dx, *grads)
    roomy.sync()
    assert torch.isfinite(y.sum(1, dtype=torch.float32)).all()
    weights = [f64(t) for t in (wg, wu, wd)]
    X, DY = f64(x[chosen]), f64(dy[chosen])
    for got, want, bound in zip((y, gate, up), N.ff(X, *weights, "silu"), N.ff_bounds(X, *weights, "silu", kind)):
        close(got[chosen], want, bound)
    args = [DY, X, *weights, "silu", f64(gate[chosen]), f64(up[chosen])]
    for got, want, bound in zip((dx[chosen], *grads), N.ff_grad(*args), N.ff_grad_bounds(*args, kind)):
        close(got, want, bound)
    dx[chosen] = 0
    assert not dx.any()


@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_ff_of_rows_far_apart(roomy, kind):
    """Rows so far apart that a matrix reaches past 2^31 elements, all matrices in one buffer."""
    rows, d, f = 300, 40, 72
    stride = 2 ** 31 // 256
    buf = torch.zeros(rows, stride, dtype=TYPES[kind], device="cuda")
    place = iter(range(0, stride, 128))
    matrices = lambda *shapes: [buf[:n, a:a + c] for (n, c), a in zip(shapes, place)]
    x, dy, wg, wu, wd = matrices((rows, d), (rows, d), (f, d), (f, d), (d, f))
    for t, s in zip((x, dy, wg, wu, wd), (1, 1, d ** -0.5, d ** -0.5, f ** -0.5)):
        t.normal_(0, s)
    y, gate, up, dx, *grads = matrices((rows, d), (rows, f), (rows, f), (rows, d), (f, d), (f, d), (d, f))
    roomy.reserve_network(rows, d, f, TYPES[kind])
    ab.abcd_gated_ff(roomy, x, wg, wu, wd, "gelu", y, gate, up)
    ab.abcd_gated_ff_backward(roomy, dy, x, wg, wu, wd, "gelu", gate, up, dx, *grads)
    roomy.sync()
    A = [f64(t) for t in (x, wg, wu, wd)]
    for got, want, bound in zip((y, gate, up), N.ff(*A, "gelu"), N.ff_bounds(*A, "gelu", kind)):
        close(got, want, bound)
    args = [f64(dy), *A, "gelu", f64(gate), f64(up)]
    for got, want, bound in zip((dx, *grads), N.ff_grad(*args), N.ff_grad_bounds(*args, kind)):
        close(got, want, bound)


@pytest.mark.parametrize("cols,pad", [(1000, 0), (1000, 8), (999, 0), (1000, 3)])
def test_dropout_past_32_bits(roomy, cols, pad):
    rows, kind, offset = 4_300_008, "f16", 77
    x = far(rows, cols, kind, pad)
    y = torch.empty_like(x)
    ab.abcd_dropout(roomy, x, 0.25, 5, offset, y, x)
    roomy.sync()
    chosen = sorted({8 * (k // 8) for k in some_rows(rows, cols + pad)})    # eight rows from each: whole blocks
    for k in chosen:
        keep, s = N.kept(8, cols, 0.25, 5, offset + k * cols // 8)
        X = f64(x[k:k + 8])
        want = keep * X * s + X
        close(y[k:k + 8], want, 3 * N.EPS * (s + 1) * np.abs(X) + np.abs(want) * 2 * N.UNIT[kind] + N.TINY[kind])
    ratio = (y / x).nan_to_num_(1.0)
    share = float((ratio > 1.5).sum(1, dtype=torch.int32).double().mean() / cols)
    assert abs(share - 0.75) < 1e-3                     # of 4e9 elements


# ---- refusals

def status(f, *a, **k):
    with pytest.raises(ab.AbcdError) as e:
        f(*a, **k)
    return e.value.status


def test_refusals(ctx):
    t = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    x, y, w = t(4, 8), t(4, 8), t(8)
    bad = ab.ABCD_ERR_INVALID_ARG
    assert status(ab.abcd_layer_norm, ctx, x, w, w, 1e-5, t(4, 9)) == bad
    assert status(ab.abcd_layer_norm, ctx, x, w, w, 1e-5, t(4, 8, dt=torch.float16)) == bad
    assert status(ab.abcd_layer_norm, ctx, x, w, w, -1.0, y) == bad
    assert status(ab.abcd_layer_norm, ctx, x, w, w, float("nan"), y) == bad
    assert status(ab.abcd_layer_norm, ctx, x, w, w, 1e-5, y, t(4), None) == bad
    assert status(ab.abcd_layer_norm_backward, ctx, y, x, w, None, None, y) == bad
    assert status(ab.abcd_layer_norm_backward, ctx, y, x, w, t(4), t(4), None, w, w, y) == bad
    assert status(ab.abcd_dropout, ctx, x, 1.5, 0, 0, y) == bad
    assert status(ab.abcd_dropout, ctx, x, float("nan"), 0, 0, y) == bad
    assert status(ab.abcd_dropout, ctx, x, 0.1, 0, 0, y, t(3, 8)) == bad
    wg, wd = t(6, 8), t(8, 6)
    ctx.reserve_network(4, 8, 6)
    assert status(ab.abcd_gated_ff, ctx, x, wg, t(5, 8), wd, "silu", y) == bad
    assert status(ab.abcd_gated_ff, ctx, x, wg, wg, wg, "silu", y) == bad
    assert status(ab.abcd_gated_ff, ctx, x, wg, wg, wd, "silu", t(4, 6)) == bad
    assert status(ab.abcd_gated_ff, ctx, x, wg, wg, wd, "silu", y, t(4, 6), None) == bad
    assert status(ab.abcd_gated_ff, ctx, x.half(), wg, wg, wd, "silu", y) == bad
    g = t(4, 6)
    assert status(ab.abcd_gated_ff_backward, ctx, y, x, wg, wg, wd, "silu", g, t(4, 5), t(4, 8)) == bad
    assert status(ab.abcd_gated_ff_backward, ctx, y, x, wg, wg, wd, "silu", g, g, t(4, 8), t(6, 9)) == bad
    # outputs that are operands or other outputs; the forward pass's y may be x
    up = t(4, 6)
    assert status(ab.abcd_gated_ff, ctx, x, wg, wg, wd, "silu", y, g, g) == bad
    assert status(ab.abcd_gated_ff, ctx, x, wg, wg, wd, "silu", wg[:4]) == bad
    assert status(ab.abcd_gated_ff_backward, ctx, y, x, wg, wg, wd, "silu", g, up, y) == bad
    assert status(ab.abcd_gated_ff_backward, ctx, y, x, wg, wg, wd, "silu", g, up, x) == bad
    assert status(ab.abcd_gated_ff_backward, ctx, y, x, wg, wg, wd, "silu", g, up, None, t(6, 8), wg) == bad
    same = t(6, 8)
    assert status(ab.abcd_gated_ff_backward, ctx, y, x, wg, wg, wd, "silu", g, up, None, same, same) == bad
    with pytest.raises(ValueError):
        ab.abcd_gated_ff(ctx, x, wg, wg, wd, "tanh", y)
    with pytest.raises(ValueError):
        ab.abcd_layer_norm(ctx, x, t(7), None, 1e-5, y)
    with pytest.raises(ValueError):
        ab.abcd_layer_norm(ctx, x, w.half(), None, 1e-5, y)
    with pytest.raises(ValueError):
        ab.abcd_dropout(ctx, t(8, 4).T, 0.1, 0, 0, y)
    with pytest.raises(ValueError):
        ab.abcd_dropout(ctx, x.double(), 0.1, 0, 0, y)
    with pytest.raises(ValueError):
        ab.abcd_dropout(ctx, x.cpu(), 0.1, 0, 0, y)
    fresh = ab.Context(0)
    assert status(ab.abcd_gated_ff, fresh, x, wg, wg, wd, "silu", y) == ab.ABCD_ERR_WORKSPACE
    assert status(ab.abcd_layer_norm_backward, fresh, y, x, w, t(4), t(4), t(4, 8)) == ab.ABCD_ERR_WORKSPACE
    fresh.reserve_network(4, 8, 6)
    ab.abcd_gated_ff(fresh, x, wg, wg, wd, "silu", y)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,d,f", [(1, 1, 1), (9, 3, 5), (77, 59, 130), (130, 250, 999), (64, 520, 136)])
def test_the_reserved_workspace_is_enough(kind, rows, d, f):
    """A context that reserved for these very sizes takes them, whatever the rows' starts."""
    c = ab.Context(0)
    c.reserve_network(rows, d, f, TYPES[kind])
    r = np.random.default_rng(1)
    for pad, lead in ((0, 0), (3, 1)):
        x = matrix(r.normal(size=(rows, d)), kind, pad, lead)
        wg, wu, wd = ff_weights(r, d, f, kind, pad, lead)
        gate, up = blank(rows, f, kind, pad, lead), blank(rows, f, kind, pad, lead)
        ab.abcd_gated_ff(c, x, wg, wu, wd, "relu", x.clone(), gate, up)
        ab.abcd_gated_ff_backward(c, x, x, wg, wu, wd, "relu", gate, up, x.clone(), wg.clone(), wu.clone(), wd.clone())
        ab.abcd_layer_norm_backward(c, x, x, None, torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda"),
                                    x.clone(), torch.zeros(d, dtype=x.dtype, device="cuda"))
    c.sync()


# ---- streams, graphs, waits

def everything(ctx, x, dy, w, wg, wu, wd, out):
    """Every call once, on the context's stream."""
    y, gate, up, nx, dn, dx, mean, rstd, dw, db, g = out
    ab.abcd_layer_norm(ctx, x, w, w, 1e-5, nx, mean, rstd)
    ab.abcd_gated_ff(ctx, nx, wg, wu, wd, "silu", y, gate, up)
    ab.abcd_dropout(ctx, y, 0.25, 9, 4, y, x)
    ab.abcd_dropout_backward(ctx, dy, 0.25, 9, 4, dn)
    ab.abcd_gated_ff_backward(ctx, dn, nx, wg, wu, wd, "silu", gate, up, dx, *g)
    ab.abcd_layer_norm_backward(ctx, dx, x, w, mean, rstd, dx, dw, db, dy)


def make_everything(n, d, f, kind, seed):
    r = np.random.default_rng(seed)
    x, dy = matrix(r.normal(size=(n, d)), kind), matrix(r.normal(size=(n, d)), kind)
    w = torch.as_tensor(r.normal(1, 0.2, d)).to("cuda", TYPES[kind])
    weights = ff_weights(r, d, f, kind, 0, 0)
    out = (blank(n, d, kind), blank(n, f, kind), blank(n, f, kind), blank(n, d, kind), blank(n, d, kind),
           blank(n, d, kind), torch.empty(n, device="cuda"), torch.empty(n, device="cuda"),
           torch.empty_like(w), torch.empty_like(w), [blank(f, d, kind), blank(f, d, kind), blank(d, f, kind)])
    return (x, dy, w, *weights), out


def flat(out):
    return [t.clone() for t in (*out[:-1], *out[-1])]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,d,f", [(1, 64, 128), (77, 59, 130), (700, 264, 520)])
def test_other_streams_and_captured_graphs(ctx, kind, n, d, f):
    """The same results on a stream of the context's own, and from a captured graph replayed on other
    inputs."""
    args, out = make_everything(n, d, f, kind, 20)
    ctx.reserve_network(n, d, f, TYPES[kind])
    everything(ctx, *args, out)
    ctx.sync()
    want = flat(out)
    stream = torch.cuda.Stream()
    side = ab.Context(0, stream)
    side.reserve_network(n, d, f, TYPES[kind])
    with torch.cuda.stream(stream):
        stream.wait_stream(torch.cuda.default_stream())
        for t in (*out[:-1], *out[-1]):
            t.fill_(float("nan"))
        everything(side, *args, out)
    side.sync()
    assert all(torch.equal(a, b) for a, b in zip(flat(out), want))
    other, _ = make_everything(n, d, f, kind, 21)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        everything(side, *args, out)
    everything(ctx, *other, out)
    ctx.sync()
    want = flat(out)
    torch.cuda.synchronize()
    for a, b in zip(args, other):
        a.copy_(b)
    for t in (*out[:-1], *out[-1]):
        t.fill_(float("nan"))
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(flat(out), want))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,d,f", [(77, 64, 130), (3001, 72, 1032)])
def test_a_wait_that_runs_out_is_reported(kind, n, d, f):
    """With no polls allowed every wait of the products gives up at once: the calls end, the status
    says so, and once it is cleared the calls are right again."""
    args, out = make_everything(n, d, f, kind, 22)
    c = ab.Context(0)
    c.reserve_network(n, d, f, TYPES[kind])
    everything(c, *args, out)
    c.sync()
    want = flat(out)
    assert ab.lib().abcd_set_wait_limit(c.h, 0) == ab.ABCD_OK
    x, dy, w, wg, wu, wd = args
    ab.abcd_gated_ff(c, x, wg, wu, wd, "silu", out[0], out[1], out[2])
    ab.abcd_gated_ff_backward(c, dy, x, wg, wu, wd, "silu", out[1], out[2], out[5], *out[-1])
    assert status(c.sync) == ab.ABCD_ERR_TIMEOUT
    assert ab.lib().abcd_set_wait_limit(c.h, 1 << 20) == ab.ABCD_OK
    c.clear_status()
    everything(c, *args, out)
    c.sync()
    assert all(torch.equal(a, b) for a, b in zip(flat(out), want))


# ---- the block

@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_block_gradient_against_differences(ctx, kind):
    """The directional derivative of sum(y c) through the whole block, from the forward calls at
    x +- h v and at the weights +- h v, against the backward calls.  With f32 and h = 2^-6 the
    quotient's own error is of order h^2 = 2.4e-4 of the third derivatives, and 2^-24 / h of the
    values; 1% of the gradient's size covers both.  bf16 rounds the block's input to 2^-9 of itself,
    far above h, so there the gradients are compared with f32's: five roundings of 2^-9 each in
    sequence stay below 2% of the norm."""
    r = np.random.default_rng(12)
    n, d, f = 300, 64, 160
    make = lambda kind: {"norm_w": torch.as_tensor(1 + 0.1 * v[0]).to("cuda", TYPES[kind]),
                         "norm_b": torch.as_tensor(0.1 * v[1]).to("cuda", TYPES[kind]),
                         "w_gate": matrix(v[2] * d ** -0.5, kind), "w_up": matrix(v[3] * d ** -0.5, kind),
                         "w_down": matrix(v[4] * f ** -0.5, kind)}
    v = [r.normal(size=s) for s in (d, d, (f, d), (f, d), (d, f))]
    xs, cs = r.normal(size=(n, d)), r.normal(size=(n, d))

    def grads(kind):
        w = make(kind)
        block = ab.FeedForwardBlock(ctx, w, n, p=0.2, seed=3)
        x, c = matrix(xs, kind), matrix(cs, kind)
        y, dx = blank(n, d, kind), blank(n, d, kind)
        block.forward(x, y)
        block.backward(c, x, dx)
        ctx.sync()
        return w, x, c, dx, block

    w, x, c, dx, block = grads("f32")
    if kind == "bf16":
        _, _, _, dx16, b16 = grads("bf16")
        for a, b in [(dx, dx16)] + [(block.grads[k], b16.grads[k]) for k in block.grads]:
            assert np.linalg.norm(f64(a) - f64(b)) <= 0.02 * np.linalg.norm(f64(a))
        return
    h = 2.0 ** -6

    def value(x):
        block.offset = 0                                # the same mask again
        y = blank(n, d, "f32")
        block.forward(x, y)
        ctx.sync()
        return float((y.double() * c.double()).sum())

    for t, g in [(x, dx)] + [(w[k], block.grads[k]) for k in w]:
        g = g.clone()
        dirn = torch.as_tensor(r.normal(size=tuple(t.shape))).to("cuda", torch.float32)
        old = t.clone()
        t.copy_(old + h * dirn)
        a = value(x)
        t.copy_(old - h * dirn)
        b = value(x)
        t.copy_(old)
        want = (a - b) / (2 * h)
        size = float(g.double().norm() * dirn.double().norm()) / g.numel() ** 0.5
        assert abs(want - float((g.double() * dirn.double()).sum())) <= 0.01 * size + 0.01 * abs(want)


def test_block_evaluates_without_dropping(ctx):
    r = np.random.default_rng(13)
    w = {"norm_w": torch.ones(24, device="cuda"), "norm_b": torch.zeros(24, device="cuda"),
         **dict(zip(("w_gate", "w_up", "w_down"), ff_weights(r, 24, 40, "f32", 0, 0)))}
    block = ab.FeedForwardBlock(ctx, w, 50, p=0.5, seed=1)
    x = matrix(r.normal(size=(20, 24)), "f32")
    y = blank(20, 24, "f32")
    block.forward(x, y, train=False)
    X = f64(x)
    nx = N.norm(X, 1.0, 0.0, 1e-5)[0]
    want = X + N.ff(nx, f64(w["w_gate"]), f64(w["w_up"]), f64(w["w_down"]), "silu")[0]
    np.testing.assert_allclose(f64(y), want, rtol=0, atol=2e-4)    # (24 + 40 + 50) EPS of values below 10
    drawn = [block.offset]
    for _ in range(2):
        block.forward(x, y)
        drawn.append(block.offset)
    assert drawn == [0, 60, 120]                        # 20 * 24 / 8 counters a pass
