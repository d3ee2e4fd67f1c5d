"""More operators of a network over the Gaussians of a block, as cases that can be timed and compared.

Tokens are made by lookups in learned tables (a row per camera, per cell, per material) and by products
with bias, activation and residual; blocks are closed by a norm, a gate and the residual sum, whose
result the next block's norm takes; and what the backward pass needs of a block is kept in 8 bits.
`run` is either the plain form (elementary torch operations in 32 bits, rounded once) or the package's
calls; `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


# ---------------------------------------------------------------------------------------
# the cases.  rows: tokens; cols: width of a token; pad: columns between the rows of the token matrices
# beyond their width (a token matrix that is a slice of a wider one).
# emb: table: rows of the table; spread: how the tokens name them; linear: out: width of the result;
# close: after, before: the norms around the sum; ffkeep: ff: hidden width.

def listed():
    return [
        # the row of one camera for one token: the call's latency
        {"name": "emb_1x1024_bf16", "op": "emb", "train": False, "rows": 1, "table": 1000,
         "cols": 1024, "pad": 0, "index": "i32", "spread": "even", "add": False, "type": "bf16"},
        # a partition's Gaussians name 1,000 materials, a few of them most of the time; odd width, rows
        # that are a slice of a wider matrix
        {"name": "emb_20000x59_f16", "op": "emb", "train": True, "rows": 20000, "table": 1000,
         "cols": 59, "pad": 5, "index": "i64", "spread": "skewed", "add": True, "type": "f16"},
        # a large scene with a code for each of 100,000 cells
        {"name": "emb_1000000x64_f32", "op": "emb", "train": True, "rows": 1000000,
         "table": 100000, "cols": 64, "pad": 0, "index": "i64", "spread": "even", "add": False,
         "type": "f32"},
        # one token through a wide product: the weights are read once, latency counts
        {"name": "linear_1x1024x4096_bf16", "op": "linear", "train": False, "rows": 1,
         "cols": 1024, "out": 4096, "act": "silu", "bias": True, "residual": False, "pad": 0,
         "type": "bf16"},
        # the 59 parameters of a partition's SH-3 Gaussians to tokens, trained in 32 bits
        {"name": "linear_20000x59x256_f32", "op": "linear", "train": True, "rows": 20000,
         "cols": 59, "out": 256, "act": "gelu", "bias": True, "residual": False, "pad": 0,
         "type": "f32"},
        # the scene-scale block, on the residual stream, trained
        {"name": "linear_100000x256x256_bf16", "op": "linear", "train": True, "rows": 100000,
         "cols": 256, "out": 256, "act": "silu", "bias": True, "residual": True, "pad": 0,
         "type": "bf16"},
        # the largest: the arithmetic of the matrix products
        {"name": "linear_16384x4096x4096_bf16", "op": "linear", "train": True, "rows": 16384,
         "cols": 4096, "out": 4096, "act": "gelu", "bias": True, "residual": True, "pad": 0,
         "type": "bf16"},
        # one token
        {"name": "close_1x1024_bf16", "op": "close", "train": False, "rows": 1, "cols": 1024,
         "after": "rms", "before": "rms", "gate": True, "pad": 0, "weights": "own", "type": "bf16"},
        # odd width, rows with gaps, layer norms, both passes
        {"name": "close_20000x59_f32", "op": "close", "train": True, "rows": 20000, "cols": 59,
         "after": "layer", "before": "layer", "gate": True, "pad": 5, "weights": "own",
         "type": "f32"},
        # a block's wide tokens, both passes: the bandwidth
        {"name": "close_100000x1024_bf16", "op": "close", "train": True, "rows": 100000,
         "cols": 1024, "after": "rms", "before": "layer", "gate": True, "pad": 0, "weights": "f32",
         "type": "bf16"},
        # a hidden matrix of the scene-scale block, kept and taken back
        {"name": "keep_100000x1024_bf16", "op": "keep", "rows": 100000, "cols": 1024, "pad": 0,
         "type": "bf16"},
        # a layer of that block: what it keeps, and its backward pass from that
        {"name": "ffkeep_100000x256x1024_bf16", "op": "ffkeep", "rows": 100000, "cols": 256,
         "ff": 1024, "act": "silu", "pad": 0, "type": "bf16"},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """A width between low and high, spread over the logarithm: half of them odd, half round."""
    n = _log_int(rng, low, high)
    if rng.random() < 0.5:
        return min(n | 1, high - 1 + high % 2)
    return min(high, rng.choice((4, 5, 7)) << (n.bit_length() - 3))


def draw(rng):
    op = rng.choice(("emb", "emb", "linear", "linear", "close", "close", "keep", "ffkeep"))
    c = {"op": op, "type": rng.choice(("f32", "f16", "bf16")), "pad": rng.choice((0, 0, 3, 8))}
    size = 2 if c["type"] == "f32" else 1
    if op == "emb":
        c["cols"] = _width(rng, 16, 2048)
        c["rows"] = _log_int(rng, 1, min(1000000, 2 * 64000000 // c["cols"] // size))
        c["table"] = _log_int(rng, 1, min(1000000, 2 * 64000000 // c["cols"] // size))
        c["index"] = rng.choice(("i32", "i64"))
        c["spread"] = rng.choice(("even", "skewed", "one"))
        c["train"] = rng.random() < 0.7
        c["add"] = rng.random() < 0.5
    elif op == "linear":
        c["cols"], c["out"] = _width(rng, 16, 8192), _width(rng, 16, 8192)
        most = 16384 * 4096 * 4096 // (c["cols"] * c["out"])
        if c["type"] == "f32":
            most //= 8              # the same cost at the rate of the 32-bit products
        most = min(most, 100000 * 2048 // max(c["cols"], c["out"]))
        c["rows"] = _log_int(rng, 1, max(1, min(200000, most)))
        # (relu's gradient jumps where 32 bits and 64 may see z on different sides of zero)
        c["act"] = rng.choice(("none", "silu", "gelu"))
        c["bias"] = rng.random() < 0.7
        c["residual"] = rng.random() < 0.5
        c["train"] = rng.random() < 0.6
    elif op == "close":
        c["cols"] = _width(rng, 16, 4096)
        c["rows"] = _log_int(rng, 1, max(1, min(100000, 100000 * 1024 // c["cols"] // size)))
        c["after"] = rng.choice((None, "layer", "rms"))
        c["before"] = rng.choice((None, "layer", "rms"))
        c["gate"] = rng.random() < 0.7
        c["weights"] = rng.choice(("own", "f32"))
        c["train"] = rng.random() < 0.6
    elif op == "keep":
        c["cols"] = _width(rng, 16, 8192)
        c["rows"] = _log_int(rng, 1, max(1, min(200000, 100000 * 1024 // c["cols"] // size)))
    else:
        c["cols"], c["ff"] = _width(rng, 32, 1024), _width(rng, 64, 4096)
        most = 100000 * 256 * 1024 // (c["cols"] * c["ff"]) // size ** 3
        c["rows"] = _log_int(rng, 16, max(32, min(100000, most, 100000 * 1024 // c["ff"])))
        c["act"] = rng.choice(("silu", "gelu", "relu"))
    return c


# ---------------------------------------------------------------------------------------
# what a program has in hand before the call

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, rows, cols, case, scale=1.0, pad=None):
    """[rows][cols] of N(0, scale^2) in the case's type, rows `pad` elements further apart."""
    pad = case["pad"] if pad is None else pad
    t = torch.randn(rows, cols + pad, generator=g, device=DEV).mul_(scale)
    return t.to(TYPES[case["type"]])[:, :cols]


def _vector(g, n, dtype, scale, about=0.0):
    return (about + scale * torch.randn(n, generator=g, device=DEV)).to(dtype)


def _like(t):
    """An empty matrix with the shape and the row stride of t."""
    return torch.empty(t.shape[0], t.stride(0), dtype=t.dtype, device=DEV)[:, :t.shape[1]]


def _act(z, name):
    """The activation of z in z's type."""
    if name == "none":
        return z
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return z * 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return torch.where(z > 0, z, 0.0)


def prepare(case, seed):
    g = _generator(seed)
    m, d, t = case["rows"], case["cols"], TYPES[case["type"]]
    s = {"case": dict(case)}
    if case["op"] == "emb":
        v = case["table"]
        u = torch.rand(m, generator=g, device=DEV, dtype=torch.float64)
        if case["spread"] == "skewed":
            u = u ** 4
        if case["spread"] == "one":
            u = torch.full_like(u, (seed % 97) / 97)
        at = (u * v).long().clamp_(max=v - 1)
        # one in twenty names no row
        at = torch.where(torch.rand(m, generator=g, device=DEV) < 0.05, -1, at)
        s["at"] = at.to(torch.int32 if case["index"] == "i32" else torch.int64)
        s["table"] = _normal(g, v, d, case, 1.0, 0)
        s["scale"] = math.sqrt(d)
        s["add"] = _normal(g, m, d, case) if case["add"] else None
        s["y"] = torch.empty(m, d + case["pad"], dtype=t, device=DEV)[:, :d]
        if case["train"]:
            s["dy"] = _normal(g, m, d, case, 0.1)
            s["dtable"] = torch.empty_like(s["table"])
    elif case["op"] == "linear":
        n = case["out"]
        s["x"] = _normal(g, m, d, case)
        s["w"] = _normal(g, n, d, case, 1.0 / math.sqrt(d), 0)
        s["b"] = _vector(g, n, t, 0.3) if case["bias"] else None
        s["res"] = _normal(g, m, n, case) if case["residual"] else None
        s["y"] = torch.empty(m, n + case["pad"], dtype=t, device=DEV)[:, :n]
        if case["train"]:
            s["dy"] = _normal(g, m, n, case, 0.1)
            s["z"] = torch.empty(m, n, dtype=t, device=DEV) if case["act"] != "none" else None
            s["dx"], s["dw"] = _like(s["x"]), torch.empty_like(s["w"])
            s["db"] = torch.empty_like(s["b"]) if case["bias"] else None
    elif case["op"] == "close":
        wt = torch.float32 if case["weights"] == "f32" else t
        # the residual stream, and a block's result off centre, each row with its own scale
        s["x"] = _normal(g, m, d, case)
        s["f"] = _normal(g, m, d, case)
        s["f"].mul_(torch.exp(0.5 * torch.randn(m, 1, generator=g, device=DEV)).to(t))
        s["f"].add_(0.5)
        s["scale"] = 0.7
        s["gate"] = _vector(g, d, wt, 0.3, 0.5) if case["gate"] else None
        for k in ("after", "before"):
            if case[k]:
                s[k + "_w"] = _vector(g, d, wt, 0.1, 1.0)
                s[k + "_b"] = _vector(g, d, wt, 0.1) if case[k] == "layer" else None
        s["y"], s["n"] = _like(s["x"]), _like(s["x"]) if case["before"] else None
        if case["train"]:
            s["dy"] = _normal(g, m, d, case, 0.1)
            s["dn"] = _normal(g, m, d, case, 0.1) if case["before"] else None
            s["dx"], s["df"] = _like(s["x"]), _like(s["x"])
            for k in ("gate", "after_w", "after_b", "before_w", "before_b"):
                s["d" + k] = torch.empty_like(s[k]) if s.get(k) is not None else None
            s["stat"] = torch.empty(4, m, dtype=torch.float32, device=DEV)
    elif case["op"] == "keep":
        # a gate's values: rows of their own scale
        s["x"] = _normal(g, m, d, case)
        s["x"].mul_(torch.exp(torch.randn(m, 1, generator=g, device=DEV)).to(t))
        s["y"] = _like(s["x"])
    else:
        f = case["ff"]
        s["x"] = _normal(g, m, d, case)
        s["dy"] = _normal(g, m, d, case, 0.1)
        s["wg"] = _normal(g, f, d, case, 1.0 / math.sqrt(d), 0)
        s["wu"] = _normal(g, f, d, case, 1.0 / math.sqrt(d), 0)
        s["wd"] = _normal(g, d, f, case, 1.0 / math.sqrt(f), 0)
        # what the forward pass left
        s["gate"], s["up"] = s["x"] @ s["wg"].T, s["x"] @ s["wu"].T
        s["dx"] = _like(s["x"])
        s["dwg"], s["dwu"] = torch.empty_like(s["wg"]), torch.empty_like(s["wu"])
        s["dwd"] = torch.empty_like(s["wd"])
    return s


# ---------------------------------------------------------------------------------------
# one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


_context = None


def _ready(s):
    """The context, its workspace and what the package's calls keep beside the caller's buffers."""
    global _context
    import paper_2608_27735_gb300 as ab
    c = s["case"]
    if _context is None:
        _context = ab.Context(torch.cuda.current_device())
    m, d, t = c["rows"], c["cols"], TYPES[c["type"]]
    if c["op"] == "emb":
        _context.reserve_embedding(m, c["table"], d)
    elif c["op"] == "linear":
        _context.reserve_linear(m, d, c["out"], t)
    elif c["op"] == "close":
        _context.reserve_residual_norm(m, d)
        for i, k in enumerate(("after", "before")):
            mean, rstd = (s["stat"][2 * i], s["stat"][2 * i + 1]) if c["train"] else (None, None)
            s["norm_" + k] = ab.Norm(c[k], s[k + "_w"], s[k + "_b"], EPS, mean, rstd) if c[k] else None
    elif c["op"] == "keep":
        s["packed"] = ab.Packed8(m, d)
    else:
        _context.reserve_packed8(m, d, c["ff"], t)
        s["packed"] = ab.Packed8(m, d), ab.Packed8(m, c["ff"]), ab.Packed8(m, c["ff"])
    return _context


def _run_own(s):
    import paper_2608_27735_gb300 as ab
    c = s["case"]
    if "ctx" not in s:
        s["ctx"] = _ready(s)
    ctx = s["ctx"]
    if c["op"] == "emb":
        ab.abcd_embedding(ctx, s["table"], s["at"], s["scale"], s["y"], s["add"])
        if not c["train"]:
            return {"y": s["y"]}
        ab.abcd_embedding_backward(ctx, s["dy"], s["at"], s["scale"], s["dtable"])
        return {k: s[k] for k in ("y", "dtable")}
    if c["op"] == "linear":
        if not c["train"]:
            ab.abcd_linear(ctx, s["x"], s["w"], s["b"], c["act"], s["y"], s["res"])
            return {"y": s["y"]}
        ab.abcd_linear(ctx, s["x"], s["w"], s["b"], c["act"], s["y"], s["res"], s["z"])
        ab.abcd_linear_backward(ctx, s["dy"], s["x"], s["w"], c["act"], s["z"], s["dx"], s["dw"],
                                s["db"])
        return {k: s[k] for k in ("y", "dx", "dw", "db") if s[k] is not None}
    if c["op"] == "close":
        norms = s["norm_after"], s["norm_before"]
        ab.abcd_residual_norm(ctx, s["x"], s["f"], *norms, s["gate"], s["scale"], s["y"], s["n"])
        out = ["y", "n"]
        if c["train"]:
            ab.abcd_residual_norm_backward(ctx, s["dy"], s["dn"], s["x"], s["f"], *norms, s["gate"],
                                           s["scale"], s["dx"], s["df"], s["dgate"], s["dafter_w"],
                                           s["dafter_b"], s["dbefore_w"], s["dbefore_b"])
            out += ["dx", "df", "dgate", "dafter_w", "dafter_b", "dbefore_w", "dbefore_b"]
        return {k: s[k] for k in out if s[k] is not None}
    if c["op"] == "keep":
        ab.abcd_pack8(ctx, s["x"], s["packed"])
        ab.abcd_unpack8(ctx, s["packed"], s["y"])
        return {"y": s["y"]}
    x, gate, up = s["packed"]
    ab.abcd_pack8(ctx, s["x"], x)
    ab.abcd_pack8(ctx, s["gate"], gate)
    ab.abcd_pack8(ctx, s["up"], up)
    ab.abcd_gated_ff_backward_packed8(ctx, s["dy"], x, s["wg"], s["wu"], s["wd"], c["act"], gate, up,
                                      s["dx"], s["dwg"], s["dwu"], s["dwd"])
    return {k: s[k] for k in ("dx", "dwg", "dwu", "dwd")}


def _slope(z, name):
    """The activation's slope at z, in z's type."""
    if name == "none":
        return torch.ones_like(z)
    if name == "silu":
        q = 1.0 / (1.0 + torch.exp(-z))
        return q * (1.0 + z * (1.0 - q))
    if name == "gelu":
        return (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2 * math.pi)))
    return (z > 0).to(z.dtype)


def _norm_plain(x, kind, w, b):
    """(result, normalised rows, 1 / spread)."""
    dev = x - x.mean(1, keepdim=True) if kind == "layer" else x
    r = 1.0 / torch.sqrt((dev * dev).mean(1, keepdim=True) + EPS)
    xh = dev * r
    y = xh * w.float()
    return (y if b is None else y + b.float()), xh, r


def _norm_back_plain(g, xh, r, kind):
    """The rows' gradient from that of xh."""
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if kind == "layer":
        dx = dx - g.mean(1, keepdim=True)
    return r * dx


def _packed_plain(x):
    """What is left of x (32 bits) in groups of 32 columns with 8 bits each: whole numbers up to 127
    times the power of two that is 64 times below the group's largest value's."""
    m, d = x.shape
    x = torch.nn.functional.pad(x, (0, -d % 32)).view(m, -1, 32)
    top = x.abs().amax(2, keepdim=True)
    # the power by its bits: the exponent of the largest magnitude, six less, 1 at the least
    power = (((top.view(torch.int32) >> 23) - 6).clamp_(min=1) << 23).view(torch.float32)
    return (torch.round(x / power).clamp_(-127, 127) * power).view(m, -1)[:, :d]


def _run_plain(s):
    c = s["case"]
    t = TYPES[c["type"]]
    if c["op"] == "emb":
        at = s["at"].long()
        named = at >= 0
        y = torch.where(named[:, None], s["table"][at.clamp(min=0)].float() * s["scale"], 0.0)
        if s["add"] is not None:
            y = s["add"].float() + y
        out = {"y": y.to(t)}
        if c["train"]:
            # sums of up to all tokens: in 64 bits
            dy = torch.where(named[:, None], s["dy"].double(), 0.0)
            d = torch.zeros(s["table"].shape, dtype=torch.float64, device=DEV)
            out["dtable"] = (d.index_add_(0, at.clamp(min=0), dy) * s["scale"]).to(t)
        return out
    if c["op"] == "linear":
        x, w = s["x"].float(), s["w"].float()
        z = x @ w.T
        if s["b"] is not None:
            z = z + s["b"].float()
        y = _act(z, c["act"])
        if s["res"] is not None:
            y = s["res"].float() + y
        out = {"y": y.to(t)}
        if c["train"]:
            dz = s["dy"].float() * _slope(z, c["act"])
            out.update(dx=(dz @ w).to(t), dw=(dz.T @ x).to(t))
            if s["b"] is not None:
                out["db"] = dz.sum(0).to(t)
        return out
    if c["op"] == "close":
        return _close_plain(s, c, t)
    if c["op"] == "keep":
        return {"y": _packed_plain(s["x"].float()).to(t)}
    x, gate, up = (_packed_plain(s[k].float()) for k in ("x", "gate", "up"))
    wg, wu, wd, dy = (s[k].float() for k in ("wg", "wu", "wd", "dy"))
    a = _act(gate, c["act"])
    dh = dy @ wd
    du, dg = dh * a, dh * up * _slope(gate, c["act"])
    return {"dx": (dg @ wg + du @ wu).to(t), "dwg": (dg.T @ x).to(t), "dwu": (du.T @ x).to(t),
            "dwd": (dy.T @ (a * up)).to(t)}


def _close_plain(s, c, t):
    x, f, scale = s["x"].float(), s["f"].float(), s["scale"]
    wt = torch.float32 if c["weights"] == "f32" else t
    h, fh, fr = _norm_plain(f, c["after"], s["after_w"], s["after_b"]) if c["after"] else (f, f, None)
    gate = s["gate"].float() if c["gate"] else 1.0
    y = x + scale * gate * h
    out = {"y": y.to(t)}
    if c["before"]:
        n, yh, yr = _norm_plain(y, c["before"], s["before_w"], s["before_b"])
        out["n"] = n.to(t)
    if not c["train"]:
        return out
    g = s["dy"].float()
    last = {}
    if c["before"]:
        dn = s["dn"].float()
        last["dbefore_w"] = (dn * yh).sum(0).to(wt)
        if s["before_b"] is not None:
            last["dbefore_b"] = dn.sum(0).to(wt)
        g = g + _norm_back_plain(dn * s["before_w"].float(), yh, yr, c["before"])
    dh = scale * gate * g
    out["dx"] = g.to(t)
    out["df"] = (_norm_back_plain(dh * s["after_w"].float(), fh, fr, c["after"]) if c["after"] else dh).to(t)
    if c["gate"]:
        out["dgate"] = (scale * g * h).sum(0).to(wt)
    if c["after"]:
        out["dafter_w"] = (dh * fh).sum(0).to(wt)
        if s["after_b"] is not None:
            out["dafter_b"] = dh.sum(0).to(wt)
    out.update(last)
    return out


# ---------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    m, d = case["rows"], case["cols"]
    e = 4 if case["type"] == "f32" else 2
    if case["op"] == "emb":
        i = 4 if case["index"] == "i32" else 8
        v = case["table"]
        n = (2 if case["add"] else 1) * m * d * e + min(m, v) * d * e + m * i
        if case["train"]:
            n += m * d * e + v * d * e
        return {"bytes": n, "flops": (3 if case["train"] else 1) * m * d}
    if case["op"] == "linear":
        o = case["out"]
        n = m * d + d * o + m * o * (2 if case["residual"] else 1)
        if case["train"]:
            n += m * o + m * d + d * o
        return {"bytes": n * e, "flops": (6 if case["train"] else 2) * m * d * o}
    if case["op"] == "close":
        n = 4 if case["before"] else 3
        if case["train"]:
            n += 4 if case["before"] else 3
        return {"bytes": n * m * d * e, "flops": (50 if case["train"] else 16) * m * d}
    if case["op"] == "keep":
        return {"bytes": 2 * m * d * e + m * (d + -(-d // 32)), "flops": 4 * m * d}
    f = case["ff"]
    return {"bytes": (3 * m * d + 2 * m * f + 6 * d * f) * e + m * (d + 2 * f) * 33 // 32,
            "flops": 12 * m * d * f}


# ---------------------------------------------------------------------------------------
# the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "emb":
        return _exact_emb(case, s)
    if case["op"] == "linear":
        x, w = s["x"].double(), s["w"].double()
        z = torch.einsum("md,nd->mn", x, w)
        if s["b"] is not None:
            z += s["b"].double()
        a, slope = _exact_act(z, case["act"])
        out = {"y": a if s["res"] is None else a + s["res"].double()}
        if case["train"]:
            dz = s["dy"].double() * slope
            out["dx"] = torch.einsum("mn,nd->md", dz, w)
            out["dw"] = torch.einsum("mn,md->nd", dz, x)
            if s["b"] is not None:
                out["db"] = torch.einsum("mn->n", dz)
        return out
    if case["op"] == "close":
        return _exact_close(case, s)
    if case["op"] == "keep":
        return {"y": _exact_packed(s["x"])}
    x, z, u = _exact_packed(s["x"]), _exact_packed(s["gate"]), _exact_packed(s["up"])
    wg, wu, wd, dy = (s[k].double() for k in ("wg", "wu", "wd", "dy"))
    a, slope = _exact_act(z, case["act"])
    dh = torch.einsum("md,df->mf", dy, wd)
    dz, du = dh * u * slope, dh * a
    return {"dx": torch.einsum("mf,fd->md", dz, wg) + torch.einsum("mf,fd->md", du, wu),
            "dwg": torch.einsum("mf,md->fd", dz, x), "dwu": torch.einsum("mf,md->fd", du, x),
            "dwd": torch.einsum("md,mf->df", dy, a * u)}


def _exact_act(z, name):
    """The activation and its slope."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * torch.sigmoid(-z)
    if name == "gelu":
        q = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * q, q + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z.clamp(min=0), torch.heaviside(z, torch.zeros_like(z))


def _exact_emb(case, s):
    at = s["at"].long()
    m, d = s["y"].shape
    y = torch.zeros(m, d, dtype=torch.float64, device=DEV)
    there = torch.nonzero(at >= 0)[:, 0]
    y[there] = s["table"].double()[at[there]] * s["scale"]
    out = {"y": y if s["add"] is None else y + s["add"].double()}
    if case["train"]:
        # the tokens in the order of the rows they name: sums between borders
        order = there[torch.argsort(at[there], stable=True)]
        total = torch.zeros(len(order) + 1, d, dtype=torch.float64, device=DEV)
        torch.cumsum(s["dy"][order].double(), 0, out=total[1:])
        border = torch.searchsorted(at[order].contiguous(), torch.arange(case["table"] + 1, device=DEV))
        out["dtable"] = (total[border[1:]] - total[border[:-1]]) * s["scale"]
    return out


def _exact_norm(v, kind, w, b):
    """(result, normalised rows, spread) by the definition."""
    n = v.shape[1]
    mean = v.sum(1, keepdim=True) / n if kind == "layer" else torch.zeros_like(v[:, :1])
    spread = (((v - mean) ** 2).sum(1, keepdim=True) / n + EPS) ** 0.5
    vh = (v - mean) / spread
    return vh * w.double() + (0.0 if b is None else b.double()), vh, spread


def _exact_norm_back(g, vh, spread, kind):
    """Through the spread, and of a layer norm the mean, as the chain rule gives them."""
    n = g.shape[1]
    dv = g / spread
    dspread = -(g * vh).sum(1, keepdim=True) / spread
    dv = dv + dspread * vh / n
    if kind == "layer":
        dv = dv - dv.sum(1, keepdim=True) / n
    return dv


def _exact_close(case, s):
    x, f = s["x"].double(), s["f"].double()
    factor = s["scale"] * (s["gate"].double() if case["gate"] else torch.ones_like(x[0]))
    h, fh, spread = (_exact_norm(f, case["after"], s["after_w"], s["after_b"]) if case["after"]
                     else (f, f, None))
    y = x + factor * h
    out = {"y": y}
    if case["before"]:
        out["n"], yh, yspread = _exact_norm(y, case["before"], s["before_w"], s["before_b"])
    if not case["train"]:
        return out
    g = s["dy"].double()
    sums = lambda a, b: torch.einsum("ij,ij->j", a, b)
    last = {}
    if case["before"]:
        dn = s["dn"].double()
        last["dbefore_w"] = sums(dn, yh)
        if s["before_b"] is not None:
            last["dbefore_b"] = dn.sum(0)
        g = g + _exact_norm_back(dn * s["before_w"].double(), yh, yspread, case["before"])
    out["dx"] = g
    dh = g * factor
    out["df"] = (_exact_norm_back(dh * s["after_w"].double(), fh, spread, case["after"])
                 if case["after"] else dh)
    if case["gate"]:
        out["dgate"] = s["scale"] * sums(g, h)
    if case["after"]:
        out["dafter_w"] = sums(dh, fh)
        if s["after_b"] is not None:
            out["dafter_b"] = dh.sum(0)
    out.update(last)
    return out


def _exact_packed(t):
    """The values that stay in 8 bits: of each 32 consecutive columns of a row, multiples of
    2^(e - 6), e the exponent of the largest magnitude, -120 at the least."""
    v = t.double()
    powers = torch.tensor([2.0 ** e for e in range(-120, 129)], dtype=torch.float64, device=DEV)
    kept = torch.empty_like(v)
    for at in range(0, v.shape[1], 32):
        part = v[:, at:at + 32]
        top = part.abs().max(1, keepdim=True).values
        e = (torch.searchsorted(powers, top, right=True) - 1).clamp(min=0)
        step = powers[e] / 64.0
        kept[:, at:at + 32] = torch.round(part / step).clamp(-127, 127) * step
    return kept
