"""The operators of a network over the Gaussians of a block, as cases that can be timed and compared.

A block trained on photographs wants a learned correction of its Gaussians' colours that depends
on the camera: one token per Gaussian goes through residual layers
x + dropout(gated_ff(layer_norm(x))).  The cases take the three operators, forward and with their
backward passes, from a single token to the tokens of a whole block.  `run` is either the plain
form (elementary torch operations in 32 bits, rounded once) or the package's calls; `exact` is the
definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


# ---------------------------------------------------------------------------------------
# the cases.  rows: tokens; cols: width of a token; ff: hidden width; pad: columns between the rows
# of the token matrices beyond their width (a token matrix that is a slice of a wider one).

def listed():
    return [
        # one token (a single Gaussian, or a camera's own token): the call's latency
        {"name": "norm_1x1024_bf16", "op": "norm", "train": False, "rows": 1, "cols": 1024,
         "pad": 0, "type": "bf16"},
        # the 59 parameters of 20,000 SH-3 Gaussians, as a slice of rows 64 wide: odd width, strides
        {"name": "norm_20000x59_f16", "op": "norm", "train": True, "rows": 20000, "cols": 59,
         "pad": 5, "type": "f16"},
        # a 64-wide token for each Gaussian of the scene-scale block
        {"name": "norm_100000x64_f32", "op": "norm", "train": True, "rows": 100000, "cols": 64,
         "pad": 0, "type": "f32"},
        # wide tokens of the same block: the bandwidth of both passes
        {"name": "norm_100000x1024_bf16", "op": "norm", "train": True, "rows": 100000,
         "cols": 1024, "pad": 0, "type": "bf16"},
        # one token through a wide layer: the weights are read once, latency counts
        {"name": "ff_1x1024x4096_bf16", "op": "ff", "train": False, "rows": 1, "cols": 1024,
         "ff": 4096, "act": "silu", "pad": 0, "type": "bf16"},
        # a token for each of the stage's 200 cameras: few rows, widths that no tile divides
        {"name": "ff_200x250x999_f16", "op": "ff", "train": False, "rows": 200, "cols": 250,
         "ff": 999, "act": "gelu", "pad": 0, "type": "f16"},
        # a narrow layer over a 20,000-Gaussian partition, trained in 32 bits
        {"name": "ff_20000x64x256_f32", "op": "ff", "train": True, "rows": 20000, "cols": 64,
         "ff": 256, "act": "silu", "pad": 0, "type": "f32"},
        # the scene-scale block through a layer of ordinary width, trained
        {"name": "ff_100000x256x1024_bf16", "op": "ff", "train": True, "rows": 100000,
         "cols": 256, "ff": 1024, "act": "silu", "pad": 0, "type": "bf16"},
        # the largest: the arithmetic of the matrix products
        {"name": "ff_16384x2048x8192_bf16", "op": "ff", "train": True, "rows": 16384,
         "cols": 2048, "ff": 8192, "act": "gelu", "pad": 0, "type": "bf16"},
        # one token
        {"name": "drop_1x1024_bf16", "op": "drop", "train": False, "rows": 1, "cols": 1024,
         "pad": 0, "residual": True, "p": 0.1, "type": "bf16"},
        # odd width, rows with gaps, both passes
        {"name": "drop_33333x59_f32", "op": "drop", "train": True, "rows": 33333, "cols": 59,
         "pad": 5, "residual": False, "p": 0.25, "type": "f32"},
        # a block's wide tokens, added to the residual stream, both passes
        {"name": "drop_100000x1024_bf16", "op": "drop", "train": True, "rows": 100000,
         "cols": 1024, "pad": 0, "residual": True, "p": 0.1, "type": "bf16"},
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
    op = rng.choice(("norm", "ff", "drop"))
    c = {"op": op, "train": rng.random() < 0.6, "type": rng.choice(("f32", "f16", "bf16")),
         "pad": rng.choice((0, 0, 3, 8))}
    if op == "ff":
        c["cols"] = _width(rng, 32, 2048)
        c["ff"] = _width(rng, 64, 8192)
        most = 16384 * 2048 * 8192 // (c["cols"] * c["ff"])
        if c["type"] == "f32":
            most //= 8              # the same cost at the rate of the 32-bit products
        c["rows"] = _log_int(rng, 1, max(1, min(100000, most)))
        c["act"] = rng.choice(("silu", "gelu"))
    else:
        c["cols"] = _width(rng, 16, 4096)
        most = 100000 * 1024 // c["cols"] // (2 if c["type"] == "f32" else 1)
        c["rows"] = _log_int(rng, 1, max(1, min(100000, most)))
    if op == "drop":
        c["residual"] = rng.random() < 0.5
        c["p"] = rng.choice((0.05, 0.1, 0.25, 0.5))
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


def _like(t):
    """An empty matrix with the shape and the row stride of t."""
    return torch.empty(t.shape[0], t.stride(0), dtype=t.dtype, device=DEV)[:, :t.shape[1]]


def prepare(case, seed):
    g = _generator(seed)
    m, d = case["rows"], case["cols"]
    s = {"case": dict(case)}
    if case["op"] == "norm":
        # tokens off centre, each row with its own scale; weights about one, in the tokens' type
        s["x"] = _normal(g, m, d, case)
        s["x"].mul_(torch.exp(0.5 * torch.randn(m, 1, generator=g, device=DEV)).to(s["x"].dtype))
        s["x"].add_(0.5)
        s["w"] = (1.0 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(s["x"].dtype)
        s["b"] = (0.1 * torch.randn(d, generator=g, device=DEV)).to(s["x"].dtype)
        if case["train"]:
            s["dy"] = _normal(g, m, d, case, 0.1)
    elif case["op"] == "ff":
        f = case["ff"]
        s["x"] = _normal(g, m, d, case)
        s["wg"] = _normal(g, f, d, case, 1.0 / math.sqrt(d), 0)
        s["wu"] = _normal(g, f, d, case, 1.0 / math.sqrt(d), 0)
        s["wd"] = _normal(g, d, f, case, 1.0 / math.sqrt(f), 0)
        if case["train"]:
            s["dy"] = _normal(g, m, d, case, 0.1)
    else:
        s["x"] = _normal(g, m, d, case)
        s["seed"] = (seed * 0x9E3779B97F4A7C15 + 0x632BE59BD9B4E019) % (1 << 63)
        s["offset"] = (1 << 32) - 1000 + 7 * (seed % 1000)     # blocks that pass 32 bits
        s["res"] = _normal(g, m, d, case) if case["residual"] else None
        if case["train"]:
            s["dy"] = _normal(g, m, d, case, 0.1)
    _buffers(s)
    return s


def _buffers(s):
    """The caller's output buffers."""
    c, x = s["case"], s["x"]
    m, d = x.shape
    s["y"] = _like(x)
    if not c["train"]:
        return
    s["dx"] = _like(x)
    if c["op"] == "norm":
        s["mean"] = torch.empty(m, dtype=torch.float32, device=DEV)
        s["rstd"] = torch.empty(m, dtype=torch.float32, device=DEV)
        s["dw"], s["db"] = torch.empty_like(s["w"]), torch.empty_like(s["b"])
    elif c["op"] == "ff":
        s["gate"] = torch.empty(m, c["ff"], dtype=x.dtype, device=DEV)
        s["up"] = torch.empty_like(s["gate"])
        s["dwg"], s["dwu"] = torch.empty_like(s["wg"]), torch.empty_like(s["wu"])
        s["dwd"] = torch.empty_like(s["wd"])


# ---------------------------------------------------------------------------------------
# one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


_context = None


def _run_own(s):
    global _context
    import paper_2608_27735_gb300 as ab
    c = s["case"]
    if "ctx" not in s:
        if _context is None:
            _context = ab.Context(torch.cuda.current_device())
        _context.reserve_network(c["rows"], c["cols"], c.get("ff", 0), TYPES[c["type"]])
        s["ctx"] = _context
    ctx = s["ctx"]
    if c["op"] == "norm":
        if not c["train"]:
            ab.abcd_layer_norm(ctx, s["x"], s["w"], s["b"], EPS, s["y"])
            return {"y": s["y"]}
        ab.abcd_layer_norm(ctx, s["x"], s["w"], s["b"], EPS, s["y"], s["mean"], s["rstd"])
        ab.abcd_layer_norm_backward(ctx, s["dy"], s["x"], s["w"], s["mean"], s["rstd"], s["dx"],
                                    s["dw"], s["db"])
        return {k: s[k] for k in ("y", "dx", "dw", "db")}
    if c["op"] == "ff":
        if not c["train"]:
            ab.abcd_gated_ff(ctx, s["x"], s["wg"], s["wu"], s["wd"], c["act"], s["y"])
            return {"y": s["y"]}
        ab.abcd_gated_ff(ctx, s["x"], s["wg"], s["wu"], s["wd"], c["act"], s["y"], s["gate"],
                         s["up"])
        ab.abcd_gated_ff_backward(ctx, s["dy"], s["x"], s["wg"], s["wu"], s["wd"], c["act"],
                                  s["gate"], s["up"], s["dx"], s["dwg"], s["dwu"], s["dwd"])
        return {k: s[k] for k in ("y", "dx", "dwg", "dwu", "dwd")}
    ab.abcd_dropout(ctx, s["x"], c["p"], s["seed"], s["offset"], s["y"], s["res"])
    if not c["train"]:
        return {"y": s["y"]}
    ab.abcd_dropout_backward(ctx, s["dy"], c["p"], s["seed"], s["offset"], s["dx"])
    return {"y": s["y"], "dx": s["dx"]}


def _run_plain(s):
    c = s["case"]
    x = s["x"].float()
    t = s["x"].dtype
    if c["op"] == "norm":
        w, b = s["w"].float(), s["b"].float()
        mean = x.mean(1, keepdim=True)
        dev = x - mean
        r = 1.0 / torch.sqrt((dev * dev).mean(1, keepdim=True) + EPS)
        xh = dev * r
        out = {"y": (xh * w + b).to(t)}
        if c["train"]:
            dy = s["dy"].float()
            g = dy * w
            dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
            out.update(dx=dx.to(t), dw=(dy * xh).sum(0).to(t), db=dy.sum(0).to(t))
        return out
    if c["op"] == "ff":
        wg, wu, wd = s["wg"].float(), s["wu"].float(), s["wd"].float()
        gate, up = x @ wg.T, x @ wu.T
        if c["act"] == "silu":
            sg = 1.0 / (1.0 + torch.exp(-gate))
            a = gate * sg
        else:
            cdf = 0.5 * (1.0 + torch.erf(gate * math.sqrt(0.5)))
            a = gate * cdf
        h = a * up
        out = {"y": (h @ wd.T).to(t)}
        if c["train"]:
            dy = s["dy"].float()
            dh = dy @ wd
            if c["act"] == "silu":
                da = sg * (1.0 + gate * (1.0 - sg))
            else:
                da = cdf + gate * torch.exp(-0.5 * gate * gate) * (1.0 / math.sqrt(2 * math.pi))
            du, dg = dh * a, dh * up * da
            out.update(dx=(dg @ wg + du @ wu).to(t), dwg=(dg.T @ x).to(t), dwu=(du.T @ x).to(t),
                       dwd=(dy.T @ h).to(t))
        return out
    keep, scale = _keep_torch(s)
    y = torch.where(keep, x * scale, 0.0)
    if s["res"] is not None:
        y = s["res"].float() + y
    out = {"y": y.to(t)}
    if c["train"]:
        out["dx"] = torch.where(keep, s["dy"].float() * scale, 0.0).to(t)
    return out


M32 = 0xFFFFFFFF
# multipliers and key increments of Philox4x32 (Salmon et al., Parallel random numbers: as easy as
# 1, 2, 3; 2011)
PHILOX_M = (0xD2511F53, 0xCD9E8D57)
PHILOX_W = (0x9E3779B9, 0xBB67AE85)


def _keep_torch(s):
    """Which elements stay ([rows][cols], truth values), and the scale of those that do."""
    c = s["case"]
    n = c["rows"] * c["cols"]
    block = torch.arange(-(-n // 8), dtype=torch.int64, device=DEV) + s["offset"]
    c0, c1 = block & M32, (block >> 32) & M32
    c2, c3 = torch.zeros_like(c0), torch.zeros_like(c0)
    k0, k1 = s["seed"] & M32, s["seed"] >> 32
    c0, c1, c2, c3 = _rounds(c0, c1, c2, c3, k0, k1, 10)
    words = torch.stack((c0, c1, c2, c3), 1)
    u = torch.stack((words & 0xFFFF, words >> 16), 2).reshape(-1)[:n]
    t = int(math.floor(c["p"] * 65536 + 0.5))
    return (u >= t).reshape(c["rows"], c["cols"]), (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _rounds(c0, c1, c2, c3, k0, k1, n):
    if n == 0:
        return c0, c1, c2, c3
    # the product of two 32-bit numbers wraps in 64 signed bits; its halves are read off by masks
    p0, p1 = c0 * PHILOX_M[0], c2 * PHILOX_M[1]
    return _rounds(((p1 >> 32) & M32) ^ c1 ^ k0, p1 & M32, ((p0 >> 32) & M32) ^ c3 ^ k1, p0 & M32,
                   (k0 + PHILOX_W[0]) & M32, (k1 + PHILOX_W[1]) & M32, n - 1)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    m, d = case["rows"], case["cols"]
    e = 4 if case["type"] == "f32" else 2
    if case["op"] == "norm":
        if not case["train"]:
            return {"bytes": 2 * m * d * e + 2 * d * e, "flops": 8 * m * d}
        return {"bytes": 4 * m * d * e + 4 * d * e, "flops": 22 * m * d}
    if case["op"] == "ff":
        f = case["ff"]
        if not case["train"]:
            return {"bytes": (2 * m * d + 3 * d * f) * e, "flops": 6 * m * d * f}
        return {"bytes": (4 * m * d + 6 * d * f) * e, "flops": 18 * m * d * f}
    n = 3 if case["residual"] else 2
    return {"bytes": (n + (2 if case["train"] else 0)) * m * d * e,
            "flops": (3 if case["train"] else 2) * m * d}


# ---------------------------------------------------------------------------------------
# the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["op"] == "norm":
        n = x.shape[1]
        mu = x.sum(1) / n
        var = ((x - mu[:, None]) ** 2).sum(1) / n
        xh = (x - mu[:, None]) / (var[:, None] + EPS) ** 0.5
        out = {"y": xh * s["w"].double() + s["b"].double()}
        if case["train"]:
            dy = s["dy"].double()
            g = dy * s["w"].double()
            # dL/dx through the mean and the variance, summed as the chain rule gives them
            dvar = (g * xh).sum(1) * -0.5 / (var + EPS)
            direct = g / (var[:, None] + EPS) ** 0.5
            out["dx"] = (direct - direct.sum(1)[:, None] / n
                         + dvar[:, None] * 2.0 * (x - mu[:, None]) / n)
            out["dw"] = torch.einsum("ij,ij->j", dy, xh)
            out["db"] = dy.sum(0)
        return out
    if case["op"] == "ff":
        wg, wu, wd = (s[k].double() for k in ("wg", "wu", "wd"))
        z = torch.einsum("md,fd->mf", x, wg)
        u = torch.einsum("md,fd->mf", x, wu)
        if case["act"] == "silu":
            q = torch.sigmoid(z)
            slope = q + z * q * torch.sigmoid(-z)
        else:
            q = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
            slope = q + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        a = z * q
        out = {"y": torch.einsum("mf,df->md", a * u, wd)}
        if case["train"]:
            dy = s["dy"].double()
            dh = torch.einsum("md,df->mf", dy, wd)
            dz, du = dh * u * slope, dh * a
            out["dx"] = torch.einsum("mf,fd->md", dz, wg) + torch.einsum("mf,fd->md", du, wu)
            out["dwg"] = torch.einsum("mf,md->fd", dz, x)
            out["dwu"] = torch.einsum("mf,md->fd", du, x)
            out["dwd"] = torch.einsum("md,mf->df", dy, a * u)
        return out
    keep = torch.from_numpy(_keep_numpy(case, s)).to(DEV)
    t = round(case["p"] * 65536)
    factor = keep.double() * (65536.0 / (65536 - t))
    out = {"y": x * factor if s["res"] is None else s["res"].double() + x * factor}
    if case["train"]:
        out["dx"] = s["dy"].double() * factor
    return out


def _keep_numpy(case, s):
    n = case["rows"] * case["cols"]
    kept = np.empty(-(-n // 8) * 8, bool)
    t = round(case["p"] * 65536)
    for a in range(0, kept.size // 8, 1 << 20):
        at = np.arange(a, min(a + (1 << 20), kept.size // 8), dtype=np.uint64) + np.uint64(s["offset"])
        c = [(at & np.uint64(M32)), at >> np.uint64(32), np.zeros_like(at), np.zeros_like(at)]
        k = [s["seed"] & M32, (s["seed"] >> 32) & M32]
        for _ in range(10):
            p0, p1 = c[0] * np.uint64(PHILOX_M[0]), c[2] * np.uint64(PHILOX_M[1])
            c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & np.uint64(M32),
                 (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & np.uint64(M32)]
            k = [(k[0] + PHILOX_W[0]) & M32, (k[1] + PHILOX_W[1]) & M32]
        half = np.empty((at.size, 8), np.uint64)
        half[:, 0::2] = np.stack(c, 1) & np.uint64(0xFFFF)
        half[:, 1::2] = np.stack(c, 1) >> np.uint64(16)
        kept[8 * a:8 * (a + at.size)] = (half >= t).reshape(-1)
    return kept[:n].reshape(case["rows"], case["cols"])
