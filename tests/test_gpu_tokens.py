"""The token operators on the GPU against their 64-bit formulas, within forward error bounds that are
computed from the inputs (tests/_tokens.py)."""
import numpy as np
import pytest

import paper_2608_27735_gb300 as ab

from . import _network as N
from . import _tokens as K
from .test_gpu_network import KINDS, TYPES, blank, close, f64, gaps_untouched, matrix

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    ab.build()
    return ab.Context(0)


def vector(a, kind):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda", TYPES[kind])


# ---- 8 bits

PACK_SHAPES = [(1, 1), (1, 32), (3, 59), (5, 64), (2, 250), (33, 257), (700, 31), (2, 5001), (1201, 16)]


def values_to_pack(r, rows, cols):
    x = r.normal(size=(rows, cols)) * np.exp(3 * r.normal(size=(rows, 1)))
    x[r.random((rows, cols)) < 0.02] = 0.0
    if rows > 4:
        x[1] = 0.0
        x[2] = 2.0 ** -13 * np.sign(x[2])
        x[3] *= 127.6 / 128 / max(1e-9, np.abs(x[3]).max())         # near the end of the codes' range
    return x


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", PACK_SHAPES)
@pytest.mark.parametrize("pad,lead", [(0, 0), (5, 3), (16, 8)])
def test_pack(ctx, kind, rows, cols, pad, lead):
    """Codes and powers are the definition's, what is read back is exact (in fp16: rounded once)."""
    x = matrix(values_to_pack(np.random.default_rng(rows + cols), rows, cols), kind, pad, lead)
    q = ab.Packed8(rows, cols)
    q.codes.fill_(77)
    ab.abcd_pack8(ctx, x, q)
    y = blank(rows, cols, kind, pad, lead)
    ab.abcd_unpack8(ctx, q, y)
    ctx.sync()
    codes, powers = K.packed(f64(x))
    assert (q.codes[:, :cols].cpu().numpy() == codes).all() and (q.powers.cpu().numpy() == powers).all()
    assert (q.codes[:, cols:] == 77).all()
    want = torch.as_tensor(K.unpacked(codes, powers)).to(TYPES[kind])
    assert torch.equal(y.cpu(), want) and gaps_untouched(y)


@pytest.mark.parametrize("kind", KINDS)
def test_pack_of_what_is_not_finite_and_of_the_smallest(ctx, kind):
    """An infinity or NaN makes its group of 32 NaN and no other; the largest values stay finite."""
    x = np.random.default_rng(1).normal(size=(6, 100))
    top = {"f32": 3.4e38, "f16": 65504.0, "bf16": 3.38e38}[kind]
    x[0, 40], x[1, 99], x[2, 0] = np.inf, -np.inf, np.nan
    x[3] = top * np.sign(x[3])
    x[4] = {"f32": 1e-45, "f16": 6e-8, "bf16": 1e-40}[kind]
    t = matrix(x, kind)
    q, y = ab.Packed8(6, 100), blank(6, 100, kind)
    ab.abcd_pack8(ctx, t, q)
    ab.abcd_unpack8(ctx, q, y)
    ctx.sync()
    codes, powers = K.packed(f64(t))
    assert (q.codes[:, :100].cpu().numpy() == codes).all() and (q.powers.cpu().numpy() == powers).all()
    want = torch.as_tensor(K.unpacked(codes, powers)).to(TYPES[kind])
    assert torch.equal(torch.nan_to_num(y.cpu(), 5.0, 7.0, 9.0), torch.nan_to_num(want, 5.0, 7.0, 9.0))
    assert np.isfinite(f64(y)[3]).all() and (np.abs(f64(y)[3]) > 0.99 * top).all()
    assert np.isnan(f64(y)[0, 32:64]).all() and np.isfinite(np.delete(f64(y)[0], range(32, 64))).all()


def test_pack_of_part_of_the_rows(ctx):
    """The first rows of a packed matrix; the others stay."""
    x = matrix(np.random.default_rng(2).normal(size=(50, 96)), "bf16")
    q = ab.Packed8(50, 96)
    q.codes.fill_(5)
    q.powers.fill_(9)
    ab.abcd_pack8(ctx, x[:20], q.head(20))
    ctx.sync()
    assert (q.codes[20:] == 5).all() and (q.powers[20:] == 9).all()
    assert (q.codes[:20].cpu().numpy() == K.packed(f64(x[:20]))[0]).all()
    with pytest.raises(ValueError):
        q.head(51)


@pytest.mark.parametrize("kind,pad", [("f32", 0), ("bf16", 0), ("f16", 3)])
def test_pack_with_powers_between_the_rows_of_codes(ctx, kind, pad):
    from paper_2608_27735_gb300 import network
    rows, cols = 130, 70
    x = matrix(values_to_pack(np.random.default_rng(4), rows, cols), kind, pad)
    apart, together, buf = ab.Packed8(rows, cols), ab.Packed8(rows, cols), torch.full((rows, 128), 55, dtype=torch.int8, device="cuda")
    together.c = network._pack_packed(buf.data_ptr(), buf.data_ptr() + 100, rows, cols, 128, 128)
    back = [blank(rows, cols, kind, pad) for _ in range(2)]
    for q, y in zip((apart, together), back):
        ab.abcd_pack8(ctx, x, q)
        ab.abcd_unpack8(ctx, q, y)
    ctx.sync()
    assert torch.equal(buf[:, :cols], apart.codes[:, :cols]) and torch.equal(buf[:, 100:103], apart.powers.view(torch.int8))
    assert (buf[:, cols:100] == 55).all() and (buf[:, 103:] == 55).all() and torch.equal(*back)


PACKED_FF = [(1, 8, 16), (9, 59, 40), (200, 64, 256), (300, 250, 129), (1100, 256, 512), (9000, 64, 700)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols,ff", PACKED_FF)
@pytest.mark.parametrize("name,pad", [("silu", 0), ("gelu", 3), ("relu", 8)])
def test_feed_forward_backward_from_packed(ctx, kind, rows, cols, ff, name, pad):
    """The gradients are those of what the packed matrices stand for."""
    r = np.random.default_rng(rows + ff)
    x, dy = matrix(r.normal(size=(rows, cols)), kind), matrix(0.1 * r.normal(size=(rows, cols)), kind, pad)
    wg, wu = (matrix(r.normal(size=(ff, cols)) / cols ** 0.5, kind, pad) for _ in range(2))
    wd = matrix(r.normal(size=(cols, ff)) / ff ** 0.5, kind, pad)
    z, u = (matrix(r.normal(size=(rows, ff)), kind) for _ in range(2))
    saved = [ab.Packed8(rows, cols), ab.Packed8(rows, ff), ab.Packed8(rows, ff)]
    for t, q in zip((x, z, u), saved):
        ab.abcd_pack8(ctx, t, q)
    ctx.reserve_packed8(rows, cols, ff, TYPES[kind])
    out = [blank(rows, cols, kind, pad), blank(ff, cols, kind, pad), blank(ff, cols, kind, pad), blank(cols, ff, kind, pad)]
    ab.abcd_gated_ff_backward_packed8(ctx, dy, saved[0], wg, wu, wd, name, saved[1], saved[2], *out)
    ctx.sync()
    X, Z, U = (K.unpacked(*K.packed(f64(t))) for t in (x, z, u))
    if kind == "f16":                                   # operands are held in the matrices' type
        X, Z, U = (v.astype(np.float16).astype(np.float64) for v in (X, Z, U))
    args = f64(dy), X, f64(wg), f64(wu), f64(wd), name, Z, U
    for got, want, bound in zip(out, N.ff_grad(*args), N.ff_grad_bounds(*args, kind)):
        close(got, want, bound)
        assert gaps_untouched(got)
    # one gradient alone is the same
    for k in range(4):
        one = blank(*out[k].shape, kind, pad)
        ab.abcd_gated_ff_backward_packed8(ctx, dy, saved[0], wg, wu, wd, name, saved[1], saved[2], *[one if i == k else None for i in range(4)])
        assert torch.equal(one, out[k])


# ---- embedding

EMBED_SHAPES = [(1, 1, 1), (1, 10, 64), (5, 3, 59), (300, 7, 33), (1000, 1000, 16), (2500, 1, 20), (5000, 300, 257), (6000, 2000, 8),
                (70000, 40000, 4), (30, 5, 2100)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,table_rows,cols", EMBED_SHAPES)
@pytest.mark.parametrize("pad,lead,wide", [(0, 0, True), (5, 3, False), (16, 8, True)])
def test_embedding(ctx, kind, rows, table_rows, cols, pad, lead, wide):
    r = np.random.default_rng(rows + cols)
    index = (r.random(rows) ** 3 * table_rows).astype(np.int64)
    index[r.random(rows) < 0.1] = -3
    at = torch.as_tensor(index).to("cuda", torch.int64 if wide else torch.int32)
    table, dy = matrix(r.normal(size=(table_rows, cols)), kind, pad, lead), matrix(r.normal(size=(rows, cols)), kind, pad, lead)
    add = matrix(r.normal(size=(rows, cols)), kind, pad, lead) if pad else None
    y, d = blank(rows, cols, kind, pad, lead), blank(table_rows, cols, kind, pad, lead)
    ctx.reserve_embedding(rows, table_rows, cols)
    scale = float(np.float32(1.7))
    ab.abcd_embedding(ctx, table, at, scale, y, add)
    ab.abcd_embedding_backward(ctx, dy, at, scale, d)
    ctx.sync()
    args = f64(table), index, scale, None if add is None else f64(add)
    close(y, K.embed(*args), K.embed_bound(*args, kind))
    close(d, K.embed_grad(f64(dy), index, scale, table_rows), K.embed_grad_bound(f64(dy), index, scale, table_rows, kind))
    assert gaps_untouched(y) and gaps_untouched(d)
    again = torch.empty_like(d)
    ab.abcd_embedding_backward(ctx, dy, at, scale, again)
    assert torch.equal(again, d)                        # the same in every run


@pytest.mark.parametrize("rows", [1, 255, 256, 257, 513, 4096, 4097, 20000, 200000])
def test_embedding_gradient_of_one_row_and_of_long_runs(ctx, rows):
    """All tokens on one row; two rows that meet at every place; all on none.  Whole numbers: exact."""
    dy = torch.randint(-4, 5, (rows, 12), device="cuda").float()
    d = torch.empty(9, 12, device="cuda")
    ctx.reserve_embedding(rows, 9, 12)
    want = torch.zeros(9, 12, device="cuda")
    at = torch.full((rows,), 4, device="cuda")
    ab.abcd_embedding_backward(ctx, dy, at, 1.0, d)
    want[4] = dy.double().sum(0).float()
    assert torch.equal(d, want)
    for cut in sorted({1, rows // 3, rows // 2 + 1, rows - 1}):
        at = torch.where(torch.arange(rows, device="cuda") < cut, 7, 2)
        ab.abcd_embedding_backward(ctx, dy, at, 1.0, d)
        want.zero_()
        want[7], want[2] = dy[:cut].double().sum(0).float(), dy[cut:].double().sum(0).float()
        assert torch.equal(d, want)
    d.fill_(float("nan"))
    ab.abcd_embedding_backward(ctx, dy, torch.full((rows,), -1, device="cuda"), 1.0, d)
    assert (d == 0).all()
    ctx.sync()


def test_embedding_without_tokens_and_over_its_sum(ctx):
    table = matrix(np.random.default_rng(3).normal(size=(6, 40)), "f32")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    d = blank(6, 40, "f32")
    ctx.reserve_embedding(1, 6, 40)
    ab.abcd_embedding(ctx, table, none, 1.0, torch.empty(0, 40, device="cuda"))
    ab.abcd_embedding_backward(ctx, torch.empty(0, 40, device="cuda"), none, 1.0, d)
    assert (d == 0).all()
    at = torch.tensor([3, -1, 0], device="cuda")
    y = torch.ones(3, 40, device="cuda")
    ab.abcd_embedding(ctx, table, at, 0.5, y, y)
    ctx.sync()
    want = 1 + 0.5 * table[[3, 0, 0]]
    want[1] = 1
    assert torch.equal(y, want)


def test_index_past_the_table_is_reported(ctx):
    """It names no row, and sync says so until the status is cleared."""
    c = ab.Context(0)
    c.reserve_embedding(4, 5, 8)
    table, y, d = torch.ones(5, 8, device="cuda"), torch.empty(4, 8, device="cuda"), torch.empty(5, 8, device="cuda")
    for bad in (5, 2 ** 31 - 1, 2 ** 40 + 1):
        at = torch.tensor([0, bad, 4, 1], device="cuda")
        ab.abcd_embedding(c, table, at, 2.0, y)
        with pytest.raises(ab.AbcdError) as e:
            c.sync()
        assert e.value.status == ab.ABCD_ERR_INVALID_ARG
        c.clear_status()
        assert (y[[0, 2, 3]] == 2).all() and (y[1] == 0).all()
        ab.abcd_embedding_backward(c, y, at, 1.0, d)
        with pytest.raises(ab.AbcdError):
            c.sync()
        c.clear_status()
        assert (d.sum(1) == torch.tensor([16.0, 16, 0, 0, 16], device="cuda")).all()
    c.sync()


# ---- linear layer

LINEAR_SHAPES = [(1, 1, 1), (1, 64, 48), (7, 59, 33), (8, 1024, 96), (9, 64, 64), (130, 250, 257), (500, 64, 1000), (1000, 700, 16),
                 (3000, 256, 256), (40, 2000, 300), (300, 8, 700), (5000, 300, 1100)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols,out", LINEAR_SHAPES)
@pytest.mark.parametrize("name,pad,lead", [("none", 0, 0), ("gelu", 5, 3), ("silu", 8, 8), ("relu", 0, 0)])
def test_linear(ctx, kind, rows, cols, out, name, pad, lead):
    r = np.random.default_rng(rows + cols + out)
    bkind = "f32" if pad == 8 else kind
    x, dy = matrix(r.normal(size=(rows, cols)), kind, pad, lead), matrix(r.normal(size=(rows, out)), kind, pad, lead)
    w = matrix(r.normal(size=(out, cols)) / cols ** 0.5, kind, pad, lead)
    b = vector(r.normal(size=out), bkind) if name != "relu" else None
    res = matrix(r.normal(size=(rows, out)), kind, pad, lead) if name != "silu" else None
    y = blank(rows, out, kind, pad, lead)
    z = blank(rows, out, kind, pad, lead) if name != "none" else None
    dx, dw, db = blank(rows, cols, kind, pad, lead), blank(out, cols, kind, pad, lead), vector(np.full(out, np.nan), bkind)
    ctx.reserve_linear(rows, cols, out, TYPES[kind])
    ab.abcd_linear(ctx, x, w, b, name, y, res, z)
    ab.abcd_linear_backward(ctx, dy, x, w, name, z, dx, dw, db)
    ctx.sync()
    B, R = f64(b) if b is not None else np.zeros(out), f64(res) if res is not None else np.zeros((rows, out))
    args = f64(x), f64(w), B, name, R
    bounds = K.linear_bounds(*args, kind)
    want = K.linear(*args)
    close(y, want[0], bounds[0])
    if z is not None:
        close(z, want[1], bounds[1])
    args = f64(dy), f64(x), f64(w), name, want[1] if z is None else f64(z)
    for got, exact, bound in zip((dx, dw, db), K.linear_grad(*args), K.linear_grad_bounds(*args, kind, bkind)):
        close(got, exact, bound)
    for t in (y, z, dx, dw):
        assert t is None or gaps_untouched(t)
    # without z the result is the same, and one gradient alone too
    again = blank(rows, out, kind, pad, lead)
    ab.abcd_linear(ctx, x, w, b, name, again, res)
    assert torch.equal(again, y)
    for k, want in enumerate((dx, dw, db)):
        one = torch.full_like(want, float("nan"))
        ab.abcd_linear_backward(ctx, dy, x, w, name, z, *[one if i == k else None for i in range(3)])
        assert torch.equal(one, want)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols,out", [(300, 59, 67), (5000, 64, 515), (9000, 59, 1067), (50000, 8, 515), (9000, 64, 1065), (20000, 16, 1022)])
@pytest.mark.parametrize("more", [0, 8])
def test_linear_writes_nothing_behind_its_rows(ctx, kind, rows, cols, out, more):
    """Rows on 16-byte boundaries whose last 16 bytes reach past them, in tiles of every size: what lies there is
    someone else's (the next columns of a wider matrix)."""
    r = np.random.default_rng(out)
    pad = -out % 8 + more
    x, w = matrix(r.normal(size=(rows, cols)), kind, -cols % 8), matrix(r.normal(size=(out, cols)) / cols ** 0.5, kind, -cols % 8)
    b = vector(r.normal(size=out), "f32")
    ctx.reserve_linear(rows, cols, out, TYPES[kind])
    res = matrix(r.normal(size=(rows, out)), kind, pad)
    args = f64(x), f64(w), f64(b), "silu", f64(res)
    want, bounds = K.linear(*args), K.linear_bounds(*args, kind)
    for pads in ((pad, pad), (pad, pad + 1), (pad + 1, pad)):
        y, z = (blank(rows, out, kind, p) for p in pads)
        ab.abcd_linear(ctx, x, w, b, "silu", y, res, z)
        ctx.sync()
        for got, exact, bound in zip((y, z), want, bounds):
            close(got, exact, bound)
            assert gaps_untouched(got)
    ab.abcd_linear(ctx, x, w, b, "silu", res, res)
    ctx.sync()
    close(res, want[0], bounds[0])
    assert gaps_untouched(res)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols,ff", [(300, 59, 67), (5000, 16, 1067), (7536, 64, 515), (9000, 35, 1001)])
@pytest.mark.parametrize("more", [0, 8])
def test_feed_forward_writes_nothing_behind_its_rows(ctx, kind, rows, cols, ff, more):
    """The same of the result, gate and up of the gated feed-forward layer and its gradients."""
    r = np.random.default_rng(ff)
    new = lambda rows, cols, scale=1.0: matrix(scale * r.normal(size=(rows, cols)), kind, -cols % 8 + more)
    out = lambda rows, cols: blank(rows, cols, kind, -cols % 8 + more)
    x, dy, wg, wu, wd = new(rows, cols), new(rows, cols, 0.1), new(ff, cols, cols ** -0.5), new(ff, cols, cols ** -0.5), new(cols, ff, ff ** -0.5)
    y, gate, up, grads = out(rows, cols), out(rows, ff), out(rows, ff), [out(rows, cols), out(ff, cols), out(ff, cols), out(cols, ff)]
    ctx.reserve_network(rows, cols, ff, TYPES[kind])
    ab.abcd_gated_ff(ctx, x, wg, wu, wd, "silu", y, gate, up)
    ab.abcd_gated_ff_backward(ctx, dy, x, wg, wu, wd, "silu", gate, up, *grads)
    ctx.sync()
    args = f64(x), f64(wg), f64(wu), f64(wd), "silu"
    for got, exact, bound in zip((y, gate, up), N.ff(*args), N.ff_bounds(*args, kind)):
        close(got, exact, bound)
    args = f64(dy), *args, f64(gate), f64(up)
    for got, exact, bound in zip(grads, N.ff_grad(*args), N.ff_grad_bounds(*args, kind)):
        close(got, exact, bound)
    assert all(gaps_untouched(t) for t in (y, gate, up, *grads))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [5, 300])
def test_linear_gelu_far_below_zero(ctx, kind, rows):
    """gelu and its slope at -9 ... 3 are as exact as elsewhere relative to themselves, through unit matrices.
    The exponential's argument z^2 / 2 is rounded twice and its factor once (0.7 z^2 EPS), the functions,
    products and, of 16-bit matrices, the polynomial (1.8e-5) add what tests/test_gpu_network_edges.py says; the
    products through unit matrices are sums of up to three terms that are not zero (less than that again), and
    dz is rounded to its type before dx is."""
    from .test_gpu_network_edges import TAIL, gelu_parts
    d = 64
    r = np.random.default_rng(rows)
    x, one = matrix(r.uniform(-9, 3, (rows, d)), kind), matrix(np.eye(d), kind)
    y, z, dx = (blank(rows, d, kind) for _ in range(3))
    ctx.reserve_linear(rows, d, d, TYPES[kind])
    ab.abcd_linear(ctx, x, one, None, "gelu", y, None, z)
    ab.abcd_linear_backward(ctx, matrix(np.ones((rows, d)), kind), x, one, "gelu", z, dx)
    ctx.sync()
    v = f64(x)
    assert (f64(z) == v).all()
    cdf, zphi, rel = gelu_parts(v)
    rel = rel + TAIL[kind]
    for got, want, mag in ((y, v * cdf, np.abs(v) * cdf), (dx, cdf + zphi, cdf + np.abs(zphi))):
        wide = mag * rel
        close(got, want, 2 * wide + 2 * (np.abs(want) + wide) * N.UNIT[kind] + N.TINY[kind])


def test_linear_gelu_of_few_tokens_is_that_of_many(ctx):
    """The activation of a value does not depend on how many rows lie beside it: in 32 bits one form of gelu, whatever
    the product.  Through a unit matrix z is x; the exponentials are the same, and the polynomial, whose ten steps a
    compiler may round once or twice each, is within 3.5 units of 2^-23 of itself in both kernels (as its coefficients
    were fitted)."""
    d = 64
    x, one = matrix(np.random.default_rng(3).uniform(-12, 3, (300, d)), "f32"), matrix(np.eye(d), "f32")
    ctx.reserve_linear(300, d, d)
    y = torch.empty_like(x)
    ab.abcd_linear(ctx, x, one, None, "gelu", y)
    for rows in (1, 3, 8, 9):
        few, z = torch.empty(rows, d, device="cuda"), torch.empty(rows, d, device="cuda")
        for at in range(0, 300 - rows, 8):
            ab.abcd_linear(ctx, x[at:at + rows], one, None, "gelu", few, None, z)
            assert torch.equal(z, x[at:at + rows])
            want = y[at:at + rows].double()
            assert ((few.double() - want).abs() <= 7 * 2.0 ** -23 * want.abs()).all()
    ctx.sync()


@pytest.mark.parametrize("rows,cols,out", [(50, 64, 96), (5000, 256, 1024)])
def test_linear_with_matrices_of_different_starts(ctx, rows, cols, out):
    """Each of residual, y and z on 16-byte boundaries or not."""
    r = np.random.default_rng(8)
    x, w = matrix(r.normal(size=(rows, cols)), "bf16"), matrix(r.normal(size=(out, cols)) / cols ** 0.5, "bf16")
    values = r.normal(size=(rows, out))
    ctx.reserve_linear(rows, cols, out, torch.bfloat16)
    want = None
    for pads in np.ndindex(2, 2, 2):
        res, y, z = matrix(values, "bf16", 3 * pads[0]), blank(rows, out, "bf16", 3 * pads[1]), blank(rows, out, "bf16", 3 * pads[2])
        ab.abcd_linear(ctx, x, w, None, "gelu", y, res, z)
        ctx.sync()
        if want is None:
            want = y.clone(), z.clone()
            args = f64(x), f64(w), np.zeros(out), "gelu", f64(res)
            for got, exact, bound in zip(want, K.linear(*args), K.linear_bounds(*args, "bf16")):
                close(got, exact, bound)
        assert torch.equal(y, want[0]) and torch.equal(z, want[1])
        assert gaps_untouched(y) and gaps_untouched(z)
        ab.abcd_linear(ctx, x, w, None, "gelu", res, res)
        assert torch.equal(res, want[0]) and gaps_untouched(res)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,out", [(300, 201), (5000, 131), (20001, 259), (40003, 515)])
def test_linear_over_residuals_that_start_anywhere(ctx, kind, rows, out):
    """In tiles of every width, whose warps take their columns in several turns: the residual's columns of a turn
    and the results of the one before go through the same shared memory.  Whole numbers: exact."""
    r = np.random.default_rng(rows)
    whole = lambda shape, most, pad=0: matrix(r.integers(-most, most + 1, shape).astype(float), kind, pad)
    x, w, res, b = whole((rows, 16), 1), whole((out, 16), 1), whole((rows, out), 9, 3), whole((1, out), 3)[0]
    want = (x.float() @ w.float().T + b.float() + res.float()).to(TYPES[kind])          # up to 28
    ctx.reserve_linear(rows, 16, out, TYPES[kind])
    for pad in (0, 3):
        y = blank(rows, out, kind, pad)
        ab.abcd_linear(ctx, x, w, b, "none", y, res)
        assert torch.equal(y, want) and gaps_untouched(y)
    ab.abcd_linear(ctx, x, w, b, "none", res, res)
    assert torch.equal(res, want) and gaps_untouched(res)
    ctx.sync()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [3, 300])
def test_linear_over_its_residual_and_without_rows(ctx, kind, rows):
    r = np.random.default_rng(6)
    x, w = matrix(r.normal(size=(rows, 96)), kind), matrix(0.1 * r.normal(size=(200, 96)), kind)
    res = matrix(r.normal(size=(rows, 200)), kind)
    y = torch.empty_like(res)
    ctx.reserve_linear(rows, 96, 200, TYPES[kind])
    ab.abcd_linear(ctx, x, w, None, "gelu", y, res)
    ab.abcd_linear(ctx, x, w, None, "gelu", res, res)
    assert torch.equal(res, y)
    dw, db = torch.ones_like(w), torch.ones(200, dtype=TYPES[kind], device="cuda")
    ab.abcd_linear_backward(ctx, y[:0], x[:0], w, "none", None, None, dw, db)
    ab.abcd_linear(ctx, x[:0], w, None, "none", y[:0])
    ctx.sync()
    assert (dw == 0).all() and (db == 0).all()


# ---- the norms around a residual sum

CLOSE_SHAPES = [(1, 1), (1, 8), (3, 59), (5, 64), (2, 250), (33, 257), (1, 1024), (1201, 16), (700, 59), (3, 4096), (2, 5001), (1, 9000),
                (40, 130), (1500, 500)]
NORM_KINDS = [("layer", "layer"), ("rms", "rms"), ("rms", "layer"), (None, "rms"), ("layer", None), (None, None)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", CLOSE_SHAPES)
@pytest.mark.parametrize("after,before", NORM_KINDS)
@pytest.mark.parametrize("pad,lead", [(0, 0), (5, 3), (16, 8)])
def test_residual_norm(ctx, kind, rows, cols, after, before, pad, lead):
    r = np.random.default_rng(rows * 7 + cols)
    wkind = "f32" if pad == 16 else kind
    x, dy, dn = (matrix(r.normal(size=(rows, cols)), kind, pad, lead) for _ in range(3))
    f = matrix(r.normal(0.5, 1, (rows, cols)) * np.exp(r.normal(0, 1, (rows, 1))), kind, pad, lead)
    v = {k: vector(r.normal(a, 0.3, cols), wkind) for k, a in (("gate", 0.7), ("aw", 1.0), ("ab", 0.0), ("bw", 1.0), ("bb", 0.0))}
    if pad == 5:
        v["gate"] = v["ab"] = v["bw"] = None
    scale = float(np.float32(0.6))
    if before is None:
        dn = None
    stat = torch.full((4, rows), float("nan"), device="cuda")
    norms = [None if k is None else ab.Norm(k, v[n + "w"], v[n + "b"], 1e-5, stat[2 * i], stat[2 * i + 1])
             for i, (k, n) in enumerate(((after, "a"), (before, "b")))]
    y, n = blank(rows, cols, kind, pad, lead), blank(rows, cols, kind, pad, lead) if before else None
    ctx.reserve_residual_norm(rows, cols)
    ab.abcd_residual_norm(ctx, x, f, *norms, v["gate"], scale, y, n)
    dx, df = blank(rows, cols, kind, pad, lead), blank(rows, cols, kind, pad, lead)
    g = {k: vector(np.full(cols, np.nan), wkind) if k == "gate" or (after if k[0] == "a" else before) else None for k in v}
    ab.abcd_residual_norm_backward(ctx, dy, dn, x, f, *norms, v["gate"], scale, dx, df, *[g[k] for k in ("gate", "aw", "ab", "bw", "bb")])
    ctx.sync()
    h = {k: None if t is None else f64(t) for k, t in v.items()}
    C = K.Close(cols, after and (after, h["aw"], h["ab"]), before and (before, h["bw"], h["bb"]), h["gate"], scale)
    X, F = f64(x), f64(f)
    want_y, want_n, _ = C.forward(X, F)
    bound_y, bound_n = C.forward_bounds(X, F, kind)
    close(y, want_y, bound_y)
    if before:
        close(n, want_n, bound_n)
    # the backward pass from the statistics that it was given
    s = [np.zeros((rows, 1)), np.ones((rows, 1))] * 2
    for i, k in enumerate((after, before)):
        if k:
            s[2 * i + 1] = f64(stat[2 * i + 1])[:, None]
            if k == "layer":
                s[2 * i] = f64(stat[2 * i])[:, None]
    args = f64(dy), None if dn is None else f64(dn), X, F, s
    got = (dx, df, g["gate"], g["aw"], g["ab"], g["bw"], g["bb"])
    for t, want, bound in zip(got, C.backward(*args), C.backward_bounds(*args, kind, wkind)):
        if t is not None:
            close(t, want, bound)
    for t in (y, n, dx, df):
        assert t is None or gaps_untouched(t)


@pytest.mark.parametrize("cols", [59, 64, 1024, 6000])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_residual_norm_in_place_and_in_part(ctx, cols, kind):
    """Outputs over inputs, gradients by themselves, no statistics."""
    r = np.random.default_rng(4)
    new = lambda: matrix(r.normal(size=(50, cols)), kind)
    x, f, dy, dn = new(), new(), new(), new()
    stat = torch.empty(4, 50, device="cuda")
    w = vector(r.normal(1, 0.3, cols), "f32")
    norms = ab.Norm("rms", w, None, 1e-5, None, stat[1]), ab.Norm("layer", w, None, 1e-5, stat[2], stat[3])
    bare = ab.Norm("rms", w), ab.Norm("layer", w)
    y, n, dx, df = (torch.empty_like(x) for _ in range(4))
    ctx.reserve_residual_norm(50, cols)
    ab.abcd_residual_norm(ctx, x, f, *norms, w, 0.5, y, n)
    d = [torch.empty(cols, device="cuda") for _ in range(3)]
    ab.abcd_residual_norm_backward(ctx, dy, dn, x, f, *norms, w, 0.5, dx, df, d[0], d[1], None, d[2])
    # without dy
    dx0, zero = torch.empty_like(x), torch.zeros_like(x)
    ab.abcd_residual_norm_backward(ctx, None, dn, x, f, *norms, w, 0.5, dx0)
    dx1 = torch.empty_like(x)
    ab.abcd_residual_norm_backward(ctx, zero, dn, x, f, *norms, w, 0.5, dx1)
    assert torch.equal(dx0, dx1)
    # the vectors alone, the rows alone
    for k in range(3):
        one = torch.empty(cols, device="cuda")
        ab.abcd_residual_norm_backward(ctx, dy, dn, x, f, *norms, w, 0.5, None, None, *[one if i == j else None for i, j in ((k, 0), (k, 1), (-1, 0), (k, 2))])
        assert torch.equal(one, d[k])
    df1 = torch.empty_like(x)
    ab.abcd_residual_norm_backward(ctx, dy, dn, x, f, *norms, w, 0.5, None, df1)
    assert torch.equal(df1, df)
    a, b = dy.clone(), dn.clone()
    ab.abcd_residual_norm_backward(ctx, a, b, x, f, *norms, w, 0.5, a, b)
    assert torch.equal(a, dx) and torch.equal(b, df)
    a, b = x.clone(), f.clone()
    ab.abcd_residual_norm_backward(ctx, dy, dn, a, b, *norms, w, 0.5, b, a)
    assert torch.equal(b, dx) and torch.equal(a, df)
    a, b = x.clone(), f.clone()
    ab.abcd_residual_norm(ctx, a, b, *bare, w, 0.5, a, b)
    assert torch.equal(a, y) and torch.equal(b, n)
    a, b = x.clone(), f.clone()
    ab.abcd_residual_norm(ctx, a, b, *bare, w, 0.5, b, a)
    assert torch.equal(b, y) and torch.equal(a, n)
    ctx.sync()


def test_residual_norm_of_rows_without_spread(ctx):
    """Rows of one value normalise to zero, whatever it is; zero rows of an rms norm too."""
    for cols in (28, 64, 250, 1000, 1024):
        f = torch.full((6, cols), 1000.0, device="cuda")
        x, y, n = torch.full_like(f, 3.0), torch.empty_like(f), torch.empty_like(f)
        ab.abcd_residual_norm(ctx, x, f, ab.Norm("layer"), ab.Norm("layer"), None, 1.0, y, n)
        assert (y == 3).all() and (n == 0).all()
        f.zero_()
        x.zero_()
        ab.abcd_residual_norm(ctx, x, f, ab.Norm("rms"), ab.Norm("rms"), None, 1.0, y, n)
        assert (y == 0).all() and (n == 0).all()
    ctx.sync()


@pytest.mark.parametrize("cols", [59, 60, 200, 1000, 1001])
@pytest.mark.parametrize("kind", KINDS)
def test_residual_norm_of_rows_of_one_great_value(ctx, kind, cols):
    """Such a row deviates by nothing, and its mean times rstd is beyond 32 bits: nothing of what a thread holds
    past the row's end may come of that.  (Powers of two, so that the sums are exact; fp16 has no such values.)"""
    level = 2.0 ** 9 if kind == "f16" else 2.0 ** 117
    eps = 1e-30 if kind == "f16" else 1e-7
    dtype = TYPES[kind]
    m = 5
    x, zero, y, n, dx, df = (torch.zeros(m, cols, device="cuda", dtype=dtype) for _ in range(6))
    f = torch.full((m, cols), level, device="cuda", dtype=dtype)
    x[:, ::2], x[:, 1::2] = 1.0, -1.0
    one, b = torch.ones(cols, device="cuda"), torch.full((cols,), 0.25, device="cuda")
    ctx.reserve_residual_norm(m, cols)
    s = torch.empty(4, m, device="cuda")
    # the norm that closes the block: its rows are its bias
    after, before = ab.Norm("layer", one, b, eps, s[0], s[1]), ab.Norm("rms", one, None, 1e-5, None, s[3])
    ab.abcd_residual_norm(ctx, x, f, after, before, None, 1.0, y, n)
    assert torch.equal(y, x + 0.25)
    want = (x + 0.25).double()
    want = want / (want.square().mean(1, keepdim=True) + 1e-5).sqrt()
    assert ((n.double() - want).abs() <= (N.UNIT[kind] + 16 * N.EPS) * want.abs()).all()     # the sums of squares are exact
    ab.abcd_residual_norm_backward(ctx, zero, zero, x, f, after, before, None, 1.0, dx, df)
    assert (dx == 0).all() and (df == 0).all()
    # the next block's norm
    after, before = None, ab.Norm("layer", one, b, eps, s[2], s[3])
    ab.abcd_residual_norm(ctx, f, zero, after, before, None, 1.0, y, n)
    assert torch.equal(y, f) and (n == 0.25).all()
    w = [torch.empty(cols, device="cuda") for _ in range(2)]
    ab.abcd_residual_norm_backward(ctx, x, zero, f, zero, after, before, None, 1.0, dx, df, None, None, None, *w)
    assert torch.equal(dx, x) and torch.equal(df, x) and not any(v.any() for v in w)


@pytest.mark.parametrize("cols", [12, 59, 60, 64, 100, 101])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [33, 9731, 20011])
def test_residual_norm_of_great_values_and_groups_without_a_row(ctx, kind, cols, rows):
    """Rows share a warp and are taken in several turns, the last of which some groups of threads have no row in:
    what statistics of an earlier row would make of nothing, here infinities, is in no sum.  (fp16 has no such
    values.)  Powers of two and whole numbers of rows: the sums are exact."""
    dtype = TYPES[kind]
    x, dy, dn, dx, df = (torch.zeros(rows, cols, device="cuda", dtype=dtype) for _ in range(5))
    f = torch.full((rows, cols), 2.0 ** 117, device="cuda", dtype=dtype)
    x[:, ::2], x[:, 1::2] = 1.0, -1.0
    dy.fill_(1.0)
    dn.fill_(0.5)
    three, b, s = torch.full((cols,), 3.0, device="cuda"), torch.full((cols,), 0.25, device="cuda"), torch.empty(4, rows, device="cuda")
    ctx.reserve_residual_norm(rows, cols)
    after, before = ab.Norm("layer", three, b, 1e-6, s[0], s[1]), ab.Norm("rms", three, None, 0.0, None, s[3])
    y, n = torch.empty_like(x), torch.empty_like(x)
    ab.abcd_residual_norm(ctx, x, f, after, before, None, 1.0, y, n)
    assert torch.equal(y, x + 0.25)
    d = [torch.full((cols,), float("nan"), device="cuda") for _ in range(4)]
    ab.abcd_residual_norm_backward(ctx, dy, dn, x, f, after, before, None, 1.0, dx, df, None, *d)
    ctx.sync()
    assert all(torch.isfinite(t).all() for t in (dx, df, *d))
    assert (d[0] == 0).all() and (d[3] == 0.5 * rows).all()           # the rows normalise to zero
    # dbefore_weight: rows of one value, (1.25 or -0.75) rstd; sums of `rows` equal terms in 32 bits
    yh = (x[0].double() + 0.25) * s[3, 0].double()
    assert ((d[2].double() - 0.5 * rows * yh).abs() <= (rows + 24) * N.EPS * 0.5 * rows * yh.abs()).all()


def test_residual_norm_without_rows(ctx):
    w, d = torch.ones(40, device="cuda"), [torch.ones(40, device="cuda") for _ in range(5)]
    e = torch.empty(0, 40, device="cuda")
    norms = ab.Norm("layer", w, w), ab.Norm("rms", w, w)
    ctx.reserve_residual_norm(1, 40)
    ab.abcd_residual_norm(ctx, e, e, *norms, w, 1.0, e, e)
    ab.abcd_residual_norm_backward(ctx, e, e, e, e, *norms, w, 1.0, e, e, *d)
    ctx.sync()
    assert all((t == 0).all() for t in d)
