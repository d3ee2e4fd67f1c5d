"""The token operators together: stacks of blocks with norms before and after, tokens of a block's
Gaussians, against their 64-bit formulas; other streams, captured graphs, workspaces, long offsets."""
import numpy as np
import pytest

import paper_2608_27735_gb300 as ab

from . import _network as N
from . import _tokens as K
from .test_gpu_network import TYPES, blank, close, f64, matrix
from .test_gpu_tokens import vector

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    ab.build()
    return ab.Context(0)


def block_weights(r, cols, ff, kind="f32", depth=2):
    return [{"before_w": vector(r.normal(1, 0.1, cols), kind), "before_b": vector(r.normal(0, 0.1, cols), kind),
             "after_w": vector(r.normal(1, 0.1, cols), kind), "gate": vector(r.normal(0.5, 0.1, cols), kind),
             "w_gate": matrix(r.normal(0, cols ** -0.5, (ff, cols)), kind),
             "w_up": matrix(r.normal(0, cols ** -0.5, (ff, cols)), kind),
             "w_down": matrix(r.normal(0, ff ** -0.5, (cols, ff)), kind)} for _ in range(depth)]


def stack_formula(weights, x, dy, scale=1.0, eps=1e-5):
    """y, dx and the blocks' gradients of a NormedStack in 64 bits."""
    w = [{k: f64(t) for k, t in b.items()} for b in weights]
    nx, mean, rstd = N.norm(x, w[0]["before_w"], w[0]["before_b"], eps)
    kept, first = [], (x, mean, rstd)
    for k, b in enumerate(w):
        f, z, u = N.ff(nx, b["w_gate"], b["w_up"], b["w_down"], "silu")
        before = None if k + 1 == len(w) else ("layer", w[k + 1]["before_w"], w[k + 1]["before_b"])
        C = K.Close(x.shape[1], ("rms", b["after_w"], None), before, b["gate"], scale, eps)
        y, n, s = C.forward(x, f)
        kept.append((C, x, f, s, nx, z, u))
        x, nx = y, n
    grads = [{} for _ in w]
    d, dn = dy, None
    for k in reversed(range(len(w))):
        C, xk, f, s, nk, z, u = kept[k]
        d, df, dgate, daw, _, dbw, dbb = C.backward(d, dn, xk, f, s)
        grads[k].update(gate=dgate, after_w=daw)
        if k + 1 < len(w):
            grads[k + 1].update(before_w=dbw, before_b=dbb)
        dn, *g = N.ff_grad(df, nk, w[k]["w_gate"], w[k]["w_up"], w[k]["w_down"], "silu", z, u)
        grads[k].update(zip(("w_gate", "w_up", "w_down"), g))
    dx, dw, db = N.norm_grad(dn, first[0], w[0]["before_w"], first[1], first[2])
    grads[0].update(before_w=dw, before_b=db)
    return x, dx + d, grads


@pytest.mark.parametrize("rows,cols,ff,depth", [(7, 16, 24, 1), (200, 28, 112, 2), (300, 64, 96, 3)])
def test_stack_is_its_formulas(ctx, rows, cols, ff, depth):
    """Sums of up to 300 terms of order one in 32 bits, through up to three blocks: a few hundred roundings of
    2^-24 in the norm of each result."""
    r = np.random.default_rng(rows)
    w = block_weights(r, cols, ff, depth=depth)
    stack = ab.NormedStack(ctx, w, rows + 5, "silu", scale=0.8)
    x, dy = matrix(r.normal(size=(rows, cols)), "f32"), matrix(r.normal(size=(rows, cols)), "f32")
    y, dx, seen = (blank(rows, cols, "f32") for _ in range(3))
    stack.forward(x, y)
    stack.forward(dy, seen, train=False)                # what was kept stays
    stack.forward(x, seen, train=False)
    stack.backward(dy, dx)
    ctx.sync()
    assert torch.equal(y, seen)
    want, want_dx, grads = stack_formula(w, f64(x), f64(dy), 0.8)
    near = lambda got, exact: np.linalg.norm(f64(got) - exact) <= 300 * 2.0 ** -24 * np.linalg.norm(exact)
    assert near(y, want) and near(dx, want_dx)
    for g, exact in zip(stack.grads, grads):
        for name in exact:
            assert near(g[name], exact[name]), name
    with pytest.raises(ValueError):
        stack.backward(dy[:3], dx[:3])
    in_place = x.clone()
    stack.forward(in_place, in_place, train=False)
    d = dy.clone()
    stack.backward(d, d)
    ctx.sync()
    assert torch.equal(in_place, y) and torch.equal(d, dx)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_packed_stack_is_one_that_kept_what_the_packed_matrices_stand_for(ctx, kind):
    r = np.random.default_rng(5)
    rows, cols, ff = 150, 40, 100
    w = block_weights(r, cols, ff, kind)
    x, dy = matrix(r.normal(size=(rows, cols)), kind), matrix(r.normal(size=(rows, cols)), kind)
    found = []
    for packed in (False, True):
        stack = ab.NormedStack(ctx, w, rows, "silu", packed=packed)
        y, dx = blank(rows, cols, kind), blank(rows, cols, kind)
        stack.forward(x, y)
        if not packed:
            for k in range(2):
                for t in (stack.normed[k], stack.gate[k], stack.up[k]):
                    q = ab.Packed8(rows, t.shape[1])
                    ab.abcd_pack8(ctx, t, q)
                    ab.abcd_unpack8(ctx, q, t)
        stack.backward(dy, dx)
        ctx.sync()
        found.append([f64(t) for t in (y, dx, *(g for b in stack.grads for g in b.values()))])
    # the same sums; in 32 bits with the zero terms of what eight bits hold left out: sums in another order
    for a, b in zip(*found):
        assert np.linalg.norm(a - b) <= (0.0 if kind == "bf16" else 100 * 2.0 ** -24) * np.linalg.norm(a) + 0.0


def test_tokens_of_an_appearance_are_the_formulas():
    """d sh and every weight's gradient of TokenAppearance, and what it does between a pass and its
    backward pass."""
    from paper_2608_27735_gb300.appearance import TokenAppearance
    ctx = ab.Context(0)
    n, cams = 200, 3
    r = np.random.default_rng(1)
    means = r.uniform(-2, 2, (n, 3)).astype(np.float32)
    app = TokenAppearance(ctx, means, 1, cams, layers=2, width=20, cells=3, seed=4)
    app.w["w_out"].copy_(torch.from_numpy(r.normal(0, 0.2, app.w["w_out"].shape).astype(np.float32)))
    app.w["b_in"].copy_(torch.from_numpy(r.normal(0, 0.2, 20).astype(np.float32)))
    assert len(set(app.cell.cpu().numpy())) > 20
    sh = torch.from_numpy(r.normal(size=(n, 4, 3)).astype(np.float32)).cuda()
    d = torch.from_numpy(r.normal(size=(n, 4, 3)).astype(np.float32)).cuda()
    got = app.forward(sh, 1)
    assert torch.equal(app.forward(sh, 1, train=False), got)
    app.forward(sh, 2, train=False)
    d_sh = app.backward(d, 1)
    ctx.sync()
    w = {k: f64(t) for k, t in app.w.items()}
    X, D, cell = f64(sh).reshape(n, 12), f64(d).reshape(n, 12), app.cell.cpu().numpy()
    tokens = X @ w["w_in"].T + w["b_in"] + w["cameras"][1] + w["cells"][cell]
    d_result = D @ w["w_out"]
    result, d_tokens, grads = stack_formula(app.stack.w, tokens, d_result)
    want = {"w_out": D.T @ result, "b_out": D.sum(0), "cells": K.embed_grad(d_tokens, cell, 1.0, 27),
            "cameras": K.embed_grad(d_tokens, np.full(n, 1), 1.0, cams), "w_in": d_tokens.T @ X, "b_in": d_tokens.sum(0)}
    near = lambda got, exact: np.linalg.norm(f64(got) - exact) <= 300 * 2.0 ** -24 * np.linalg.norm(exact)
    assert near(got, (X + result @ w["w_out"].T + w["b_out"]).reshape(n, 4, 3))
    assert near(d_sh, (D + d_tokens @ w["w_in"]).reshape(n, 4, 3))
    for name, exact in want.items():
        assert near(app.g[name], exact), name
    for g, exact in zip(app.stack.grads, grads):
        for name in exact:
            assert near(g[name], exact[name]), name


@pytest.mark.parametrize("packed", [False, True])
def test_tokens_train_with_a_render(packed):
    """A few steps of a stage with tokens run, change the weights and leave everything finite."""
    from paper_2608_27735_gb300.appearance import AppearanceStage
    from paper_2608_27735_gb300 import scenegen as sg
    s = sg.grid_scene((1, 1, 1), 5.0, 300, 1, seed=3)
    cams = sg.ring_cameras(2, 1.5 * sg.half_diagonal(s.grid), np.zeros(3), 48, 48, seed=3, height_jitter=1.0)
    photos = np.random.default_rng(2).uniform(0, 1, (2, 48, 48, 3)).astype(np.float32)
    run = AppearanceStage(s.gaussians, cams, photos, appearance="tokens", width=24, packed=packed)
    before = run.appearance.adam.values.clone()
    for _ in range(3):
        run.step()
    assert np.isfinite(run.eval_loss())
    after = run.appearance.adam.values
    assert torch.isfinite(after).all() and not torch.equal(after, before)


# ---- streams, graphs, workspaces

@pytest.mark.parametrize("packed", [False, True])
def test_stack_on_a_stream_of_its_own(packed):
    """Two training passes, called while the current stream is another one: each takes its input as the
    context's stream leaves it, after the pass before has read its own."""
    r = np.random.default_rng(12)
    rows, cols, ff = 3000, 64, 128
    w = block_weights(r, cols, ff)
    inputs = [[matrix(r.normal(size=(rows, cols)), "f32") for _ in range(2)] for _ in range(2)]

    def passes(ctx):
        stack = ab.NormedStack(ctx, w, rows, packed=packed)
        out = [[torch.full_like(inputs[0][0], float("nan")) for _ in range(2)] + [{k: torch.zeros_like(t) for k, t in g.items()} for g in stack.grads]
               for _ in range(2)]
        x = torch.full_like(inputs[0][0], float("nan"))
        torch.cuda.synchronize()
        for (given, dy), (y, dx, *grads) in zip(inputs, out):
            with torch.cuda.stream(ctx.stream):
                torch.cuda._sleep(10_000_000)
                x.copy_(given)
            stack.forward(x, y)
            stack.backward(dy, dx)
            with torch.cuda.stream(ctx.stream):
                for a, b in zip(grads, stack.grads):
                    for k in a:
                        a[k].copy_(b[k])
        ctx.sync()
        torch.cuda.synchronize()
        return [t for y, dx, *grads in out for t in (y, dx, *(v for g in grads for v in g.values()))]

    want = passes(ab.Context(0))
    assert torch.isfinite(want[0]).all() and not torch.equal(want[0], want[len(want) // 2])
    assert all(torch.equal(a, b) for a, b in zip(passes(ab.Context(0, torch.cuda.Stream())), want))


def every_call(ctx, t):
    """Each token operator once, over the tensors of operands()."""
    ab.abcd_embedding(ctx, t["table"], t["at"], 0.7, t["tokens"], t["x"])
    ab.abcd_linear(ctx, t["tokens"], t["w"], t["b"], "gelu", t["y"], t["x"], t["z"])
    norms = ab.Norm("rms", t["b"], None, 1e-5, None, t["stat"][1]), ab.Norm("layer", t["b"], t["b"], 1e-5, t["stat"][2], t["stat"][3])
    ab.abcd_residual_norm(ctx, t["x"], t["y"], *norms, t["b"], 0.5, t["r"], t["n"])
    ab.abcd_residual_norm_backward(ctx, t["n"], t["r"], t["x"], t["y"], *norms, t["b"], 0.5, t["dx"], t["df"], *t["dv"][:2], None, *t["dv"][2:4])
    ab.abcd_linear_backward(ctx, t["df"], t["tokens"], t["w"], "gelu", t["z"], t["dt"], t["dw"], t["dv"][4])
    ab.abcd_embedding_backward(ctx, t["dt"], t["at"], 0.7, t["dtable"])
    ab.abcd_pack8(ctx, t["dt"], t["packed"])
    ab.abcd_unpack8(ctx, t["packed"], t["back"])
    ab.abcd_gated_ff_backward_packed8(ctx, t["df"], t["packed"], t["w"], t["w"], t["w"], "silu", t["packed"], t["packed"], t["g"][0], t["g"][1], t["g"][2], t["g"][3])


OUTPUTS = ("tokens", "y", "z", "r", "n", "dx", "df", "dt", "dw", "dtable", "back")


def operands(seed, rows=300, cols=64, kind="bf16"):
    r = np.random.default_rng(seed)
    new = lambda *s: matrix(r.normal(size=s), kind)
    t = {k: blank(rows, cols, kind) for k in ("tokens", "y", "z", "r", "n", "dx", "df", "dt", "back")}
    t.update(table=new(50, cols), x=new(rows, cols), w=matrix(r.normal(size=(cols, cols)) / 8, kind), dw=blank(cols, cols, kind),
             dtable=blank(50, cols, kind), b=vector(r.normal(1, 0.2, cols), kind),
             at=torch.as_tensor(r.integers(-1, 50, rows)).cuda(), stat=torch.empty(4, rows, device="cuda"),
             dv=[torch.empty(cols, dtype=TYPES[kind], device="cuda") for _ in range(5)],
             g=[blank(rows, cols, kind)] + [blank(cols, cols, kind) for _ in range(3)], packed=ab.Packed8(rows, cols))
    return t


def reserve(ctx, rows=300, cols=64, kind="bf16"):
    ctx.reserve_embedding(rows, 50, cols)
    ctx.reserve_linear(rows, cols, cols, TYPES[kind])
    ctx.reserve_residual_norm(rows, cols)
    ctx.reserve_packed8(rows, cols, cols, TYPES[kind])


def outputs(t):
    return [t[k] for k in OUTPUTS] + t["dv"] + t["g"] + [t["packed"].codes, t["packed"].powers]


@pytest.mark.parametrize("layers", ["layers", "tokens", "packed tokens"])
def test_appearance_on_a_stream_of_its_own(layers):
    """Training and other passes, called while the current stream is another one, whose memory they take."""
    from paper_2608_27735_gb300.appearance import Appearance, TokenAppearance
    n, cams = 2000, 3
    r = np.random.default_rng(13)
    means = r.uniform(-2, 2, (n, 3)).astype(np.float32)
    inputs = [[torch.from_numpy(r.normal(size=(n, 4, 4)).astype(np.float32)).cuda()[:, :, :3] for _ in range(2)] for _ in range(3)]

    def passes(ctx):
        if layers == "layers":
            app = Appearance(ctx, n, 1, cams, p=0.1, seed=4)
            last = app.blocks[-1].w["w_down"]
        else:
            app = TokenAppearance(ctx, means, 1, cams, width=24, packed=layers == "packed tokens", seed=4)
            last = app.w["w_out"]
        given = torch.full_like(inputs[0][0], float("nan"))
        kept = []
        torch.cuda.synchronize()
        for ci, (sh, d) in enumerate(inputs):
            with torch.cuda.stream(ctx.stream):
                torch.cuda._sleep(10_000_000)
                given.copy_(sh)
                last.add_(0.01)
            kept.append(app.forward(given, ci))
            other = app.forward(given, 0, train=False)
            del other                                   # its memory is the current stream's to use again
            spoiled = [torch.full((n, 12), float("nan"), device="cuda") for _ in range(8)]
            del spoiled
            kept.append(app.backward(d, ci))
            app.step()
        ctx.sync()
        torch.cuda.synchronize()
        return [*kept, app.adam.values.clone()]

    want = passes(ab.Context(0))
    assert all(torch.isfinite(t).all() for t in want)
    assert all(torch.equal(a, b) for a, b in zip(passes(ab.Context(0, torch.cuda.Stream())), want))


def test_captured_and_replayed_with_other_inputs(ctx):
    """A graph of every call takes what its inputs hold when it runs."""
    stream = torch.cuda.Stream()
    c = ab.Context(0, stream)
    reserve(c)
    reserve(ctx)
    t = operands(1)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        every_call(c, t)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            every_call(c, t)
    for seed in (2, 3):
        other = operands(seed)
        for k in ("table", "x", "w", "b", "at"):
            t[k].copy_(other[k])
        for o in outputs(t):
            o.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        every_call(ctx, other)
        ctx.sync()
        for a, b in zip(outputs(t), outputs(other)):
            assert torch.equal(a, b)
    c.sync()


def test_two_contexts_at_once():
    """Contexts on streams of their own, each with its workspace, side by side."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    contexts = [ab.Context(0, s) for s in streams]
    sets = [operands(k) for k in range(2)]
    for c in contexts:
        reserve(c)
    torch.cuda.synchronize()
    for _ in range(20):
        for c, t in zip(contexts, sets):
            every_call(c, t)
    torch.cuda.synchronize()
    for k, c in enumerate(contexts):
        c.sync()
        alone = operands(k)
        every_call(c, alone)
        torch.cuda.synchronize()
        c.sync()
        for a, b in zip(outputs(sets[k]), outputs(alone)):
            assert torch.equal(a, b)


def test_workspaces_as_reserved_and_too_small():
    """Each call runs with exactly what its size function says for it, for more, and is refused below."""
    rows, cols = 700, 72
    r = np.random.default_rng(2)
    new = lambda *s: matrix(r.normal(size=s), "f32", 1)
    x, y, z, w, at = new(rows, cols), new(rows, 40), new(rows, 40), new(40, cols), torch.as_tensor(r.integers(0, 9, rows)).cuda()
    dx, dw, db, table = torch.empty_like(x), torch.empty_like(w), torch.empty(40, device="cuda"), new(9, cols)
    stat, v = torch.empty(4, rows, device="cuda"), torch.empty(cols, device="cuda")
    norms = ab.Norm("rms", None, None, 1e-5, None, stat[1]), ab.Norm("layer", None, None, 1e-5, stat[2], stat[3])
    ff = new(40, cols), new(40, cols), new(cols, 40)
    saved = ab.Packed8(rows, cols), ab.Packed8(rows, 40), ab.Packed8(rows, 40)
    c = ab.Context(0)
    for t, q in zip((x, y, z), saved):
        ab.abcd_pack8(c, t, q)
    calls = {"reserve_linear": ((rows, cols, 40), lambda c: (ab.abcd_linear(c, x, w, None, "silu", y, None, z),
                                                            ab.abcd_linear_backward(c, y, x, w, "silu", z, dx, dw, db))),
             "reserve_embedding": ((rows, 9, cols), lambda c: (ab.abcd_embedding(c, table, at, 1.0, dx), ab.abcd_embedding_backward(c, dx, at, 1.0, table))),
             "reserve_residual_norm": ((rows, cols), lambda c: (ab.abcd_residual_norm(c, x, x, *norms, None, 1.0, dx, torch.empty_like(dx)),
                                                                ab.abcd_residual_norm_backward(c, None, x, x, x, *norms, None, 1.0, dx, dbefore_weight=v))),
             "reserve_packed8": ((rows, cols, 40), lambda c: ab.abcd_gated_ff_backward_packed8(c, x, saved[0], *ff, "silu", saved[1], saved[2], dx,
                                                                                               *(torch.empty_like(t) for t in ff)))}
    for name, (sizes, run) in calls.items():
        c = ab.Context(0)
        with pytest.raises(ab.AbcdError) as e:
            run(c)
        assert e.value.status == ab.ABCD_ERR_WORKSPACE
        getattr(c, name)(*sizes)
        run(c)
        c.sync()
        more = ab.Context(0)
        getattr(more, name)(*(3 * s for s in sizes))
        run(more)
        more.sync()


@pytest.mark.parametrize("limit", [1, 2, 3, 10, 100, 300])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_products_whose_waits_run_out_say_so(limit, kind):
    """With few polls a wait the products give up or not: never a hang, always a status, and the context
    works again once that is cleared."""
    c = ab.Context(0)
    rows, cols, out = 3000, 256, 512
    c.reserve_linear(rows, cols, out, TYPES[kind])
    r = np.random.default_rng(9)
    x, w, res = matrix(r.normal(size=(rows, cols)), kind), matrix(r.normal(size=(out, cols)) / 16, kind), matrix(r.normal(size=(rows, out)), kind)
    y, z, want = torch.empty_like(res), torch.empty_like(res), torch.empty_like(res)
    ab.abcd_linear(c, x, w, None, "silu", want, res, z)
    c.sync()
    c.check(ab.lib().abcd_set_wait_limit(c.h, limit))
    for _ in range(3):
        ab.abcd_linear(c, x, w, None, "silu", y, res, z)
        try:
            c.sync()
            assert torch.equal(y, want)
        except ab.AbcdError as e:
            assert e.status == ab.ABCD_ERR_TIMEOUT
            c.clear_status()
    c.check(ab.lib().abcd_set_wait_limit(c.h, 1 << 20))
    ab.abcd_linear(c, x, w, None, "silu", y, res, z)
    c.sync()
    assert torch.equal(y, want)


# ---- what is not finite, and offsets past 32 bits

def test_what_is_not_finite_stays_in_its_row(ctx):
    r = np.random.default_rng(7)
    rows, cols = 40, 96
    x, f, dy, dn = (matrix(r.normal(size=(rows, cols)), "f32") for _ in range(4))
    x[3, 5], f[7, 0], dy[9, 1], dn[11, 2] = float("inf"), float("nan"), float("nan"), float("inf")
    stat = torch.empty(4, rows, device="cuda")
    norms = ab.Norm("rms", None, None, 1e-5, None, stat[1]), ab.Norm("layer", None, None, 1e-5, stat[2], stat[3])
    y, n, dx, df = (torch.empty_like(x) for _ in range(4))
    ctx.reserve_residual_norm(rows, cols)
    ab.abcd_residual_norm(ctx, x, f, *norms, None, 1.0, y, n)
    ab.abcd_residual_norm_backward(ctx, dy, dn, x, f, *norms, None, 1.0, dx, df)
    ctx.sync()
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[[3, 7]] = True
    assert torch.equal(~torch.isfinite(n).all(1), bad)
    bad[[9, 11]] = True
    assert torch.equal(~torch.isfinite(df).all(1), bad) and torch.isfinite(dx[~bad]).all()
    at = torch.arange(rows, device="cuda") // 4
    d = torch.empty(10, cols, device="cuda")
    ctx.reserve_embedding(rows, 10, cols)
    ab.abcd_embedding_backward(ctx, dy, at, 1.0, d)
    ctx.sync()
    where = torch.zeros_like(d, dtype=torch.bool)
    where[2, 1] = True
    assert torch.equal(~torch.isfinite(d), where)


def test_rows_past_32_bit_offsets(ctx):
    """Tables and matrices of more than 2^32 bytes and 2^31 elements."""
    cols, apart = 40, 1 << 26
    rows = 2 ** 31 // apart + 3                        # 35 rows, 67 million elements apart
    buf = torch.zeros(rows * apart, dtype=torch.bfloat16, device="cuda")
    far = buf.view(rows, apart)[:, :cols]
    near = matrix(np.random.default_rng(8).normal(size=(rows, cols)), "bf16")
    far.copy_(near)
    at = torch.arange(rows, device="cuda").flip(0)
    ctx.reserve_embedding(rows, rows, cols)
    ctx.reserve_residual_norm(rows, cols)
    y, back = torch.empty_like(near), torch.empty_like(near)
    ab.abcd_embedding(ctx, far, at, 1.0, y)
    assert torch.equal(y, near.flip(0))
    ab.abcd_embedding_backward(ctx, far, at, 1.0, y)
    assert torch.equal(y, near.flip(0))
    q = ab.Packed8(rows, cols), ab.Packed8(rows, cols)
    ab.abcd_pack8(ctx, far, q[0])
    ab.abcd_pack8(ctx, near, q[1])
    assert torch.equal(q[0].codes[:, :cols], q[1].codes[:, :cols]) and torch.equal(q[0].powers, q[1].powers)
    ab.abcd_unpack8(ctx, q[1], back)
    found = []
    for t in (near, far):
        stat = torch.empty(4, rows, device="cuda")
        norms = ab.Norm("rms", None, None, 1e-5, None, stat[1]), ab.Norm("layer", None, None, 1e-5, stat[2], stat[3])
        n, dx, df = (torch.empty_like(near) for _ in range(3))
        ab.abcd_residual_norm(ctx, t, t, *norms, None, 1.0, y, n)
        ab.abcd_residual_norm_backward(ctx, t, t, t, t, *norms, None, 1.0, dx, df)
        found.append([y.clone(), n, dx, df])
    assert all(torch.equal(a, b) for a, b in zip(*found))
    norms = ab.Norm("rms"), ab.Norm("layer")
    ab.abcd_residual_norm(ctx, near, near, *norms, None, 1.0, far, y)
    assert torch.equal(far, found[0][0])
    ab.abcd_unpack8(ctx, q[1], far)
    assert torch.equal(far, back)
    ab.abcd_embedding(ctx, near, at, 1.0, far)
    assert torch.equal(far, near.flip(0))
    ab.abcd_embedding_backward(ctx, near, at, 1.0, far)
    assert torch.equal(far, near.flip(0))
    w = matrix(np.eye(cols), "bf16")
    ctx.reserve_linear(rows, cols, cols, torch.bfloat16)
    ab.abcd_linear(ctx, near, w, None, "none", far)
    assert torch.equal(far, near)
    ab.abcd_linear(ctx, far, w, None, "none", y, far)
    assert torch.equal(y, 2 * near)
    ctx.sync()


@pytest.mark.parametrize("tokens", [9000, 700000, 1500000])
def test_sort_of_tokens_in_tiles_of_every_size(ctx, tokens):
    """Whole numbers: exact sums, whatever the order."""
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    for rows in (3, 1023, 1024, 200000):
        at = torch.randint(-1, rows, (tokens,), generator=g, device="cuda")
        dy = torch.randint(-3, 4, (tokens, 4), generator=g, device="cuda").float()
        d = torch.empty(rows, 4, device="cuda")
        ctx.reserve_embedding(tokens, rows, 4)
        ab.abcd_embedding_backward(ctx, dy, at, 1.0, d)
        ctx.sync()
        want = torch.zeros(rows, 4, dtype=torch.float64, device="cuda").index_add_(0, at.clamp(min=0), torch.where(at[:, None] >= 0, dy, 0.0).double())
        assert torch.equal(d.double(), want)
