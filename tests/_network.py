"""The network operators in 64 bits (numpy), from their definitions, with bounds on how far results
in fewer bits may be off.

The bounds are forward error bounds, element by element.  A sum of n products in 32 bits is off by at
most (n + 8) EPS times the sum of the products' magnitudes (EPS = 2^-23: the matrix instructions may
truncate where they align their addends; the 8 covers operands that are held as three 16-bit terms),
a function of it by its slope times that, and a result rounded to its type by half a unit of the
type.  The device's exp, erf and division are taken as off by 16 EPS of the value's scale."""
import math

import numpy as np

EPS = 2.0 ** -23
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}     # half a unit in the last place
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}  # the smallest steps near zero

erf = np.vectorize(math.erf, otypes=[np.float64])


def sigmoid(z):
    return 0.5 * (1.0 + np.tanh(0.5 * z))


def act(z, name):
    if name == "silu":
        return z * sigmoid(z)
    if name == "gelu":
        return z * 0.5 * (1.0 + erf(z / math.sqrt(2.0)))
    return np.maximum(z, 0.0)


def slope(z, name):
    if name == "silu":
        s = sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + erf(z / math.sqrt(2.0))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return (z > 0).astype(np.float64)


def norm(x, w, b, eps):
    mean = x.mean(1, keepdims=True)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(var + eps)
    return (x - mean) * rstd * w + b, mean, rstd


def norm_bound(x, w, b, eps, kind):
    """Bound of |y - exact|: the mean is off by (n + 8) EPS mean|x|, the variance by twice that sum
    against the deviations, so xh by (2 n + 24) EPS (|x| + mean|x|) rstd and its own share."""
    n = x.shape[1]
    y, mean, rstd = norm(x, w, b, eps)
    mag = np.abs(x).mean(1, keepdims=True)
    dev = (np.abs(x) + mag) * rstd
    k = (2 * n + 24) * EPS
    wide = np.abs(w) * k * (dev + np.abs(x - mean) * rstd * (1 + mag * rstd)) + 4 * EPS * np.abs(b)
    return wide + (np.abs(y) + wide) * UNIT[kind] + TINY[kind]


def norm_grad(dy, x, w, mean, rstd):
    xh = (x - mean) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def norm_grad_bounds(dy, x, w, mean, rstd, kind, wkind, extra=0.0):
    """Bounds of dx, dw, db: xh off by 8 EPS (|x| + |mean|) rstd, the row's sums over n and the
    column's over m by the sums of magnitudes."""
    m, n = x.shape
    dx, dw, db = norm_grad(dy, x, w, mean, rstd)
    xh = np.abs((x - mean) * rstd)
    exh = 8 * EPS * (np.abs(x) + np.abs(mean)) * rstd
    g = np.abs(dy * w)
    k = (n + 16) * EPS
    s2 = (g * xh).mean(1, keepdims=True)
    e2 = k * s2 + (g * exh).mean(1, keepdims=True)
    edx = rstd * (8 * EPS * g + k * g.mean(1, keepdims=True) + xh * e2 + exh * s2 + 8 * EPS * xh * s2)
    edx = edx + 4 * EPS * (np.abs(dx) + np.abs(extra))
    kc = (m + 16) * EPS
    edw = kc * (np.abs(dy) * xh).sum(0) + (np.abs(dy) * exh).sum(0)
    edb = kc * np.abs(dy).sum(0)
    return (edx + (np.abs(dx + extra) + edx) * UNIT[kind] + TINY[kind],
            edw + (np.abs(dw) + edw) * UNIT[wkind] + TINY[wkind],
            edb + (np.abs(db) + edb) * UNIT[wkind] + TINY[wkind])


def ff(x, wg, wu, wd, name):
    z, u = x @ wg.T, x @ wu.T
    h = act(z, name) * u
    return h @ wd.T, z, u


def ff_bounds(x, wg, wu, wd, name, kind):
    """Bounds of y, gate and up."""
    d, f = x.shape[1], wg.shape[0]
    y, z, u = ff(x, wg, wu, wd, name)
    ez = (d + 8) * EPS * (np.abs(x) @ np.abs(wg).T)
    eu = (d + 8) * EPS * (np.abs(x) @ np.abs(wu).T)
    a = np.abs(act(z, name))
    ea = 1.2 * ez + 16 * EPS * np.abs(z)
    eh = ea * (np.abs(u) + eu) + a * eu
    h = a * np.abs(u)
    eh = eh + (h + eh) * UNIT[kind] + TINY[kind]
    ey = eh @ np.abs(wd).T + (f + 8) * EPS * ((h + eh) @ np.abs(wd).T)
    return (ey + (np.abs(y) + ey) * UNIT[kind] + TINY[kind],
            ez + (np.abs(z) + ez) * UNIT[kind] + TINY[kind],
            eu + (np.abs(u) + eu) * UNIT[kind] + TINY[kind])


def ff_grad(dy, x, wg, wu, wd, name, z, u):
    """dx, dw_gate, dw_up, dw_down from the saved projections z and u."""
    dh = dy @ wd
    a = act(z, name)
    dg, du = dh * u * slope(z, name), dh * a
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x, dy.T @ (a * u)


def ff_grad_bounds(dy, x, wg, wu, wd, name, z, u, kind):
    m, d = x.shape
    f = wg.shape[0]
    A = np.abs
    dh = dy @ wd
    edh = (d + 8) * EPS * (A(dy) @ A(wd))
    a, s = act(z, name), slope(z, name)
    ea, es = 16 * EPS * A(z), 16 * EPS * (1 + A(z))
    edg = edh * A(u * s) + (A(dh) + edh) * A(u) * (es + 4 * EPS * A(s))
    edu = edh * A(a) + (A(dh) + edh) * (ea + 4 * EPS * A(a))
    r = lambda v, e: e + (A(v) + e) * UNIT[kind] + TINY[kind]
    dg, du, h = dh * u * s, dh * a, a * u
    edg, edu = r(dg, edg), r(du, edu)
    eh = r(h, ea * A(u) + 4 * EPS * A(h))
    out = ff_grad(dy, x, wg, wu, wd, name, z, u)
    edx = edg @ A(wg) + edu @ A(wu) + (2 * f + 8) * EPS * ((A(dg) + edg) @ A(wg) + (A(du) + edu) @ A(wu))
    ewg = edg.T @ A(x) + (m + 8) * EPS * ((A(dg) + edg).T @ A(x))
    ewu = edu.T @ A(x) + (m + 8) * EPS * ((A(du) + edu).T @ A(x))
    ewd = A(dy).T @ eh + (m + 8) * EPS * (A(dy).T @ (A(h) + eh))
    return tuple(r(v, e) for v, e in zip(out, (edx, ewg, ewu, ewd)))


def kept(rows, cols, p, seed, offset):
    """Dropout's mask [rows][cols] and scale: Philox4x32-10 over whole numbers of Python."""
    n = rows * cols
    t = int(math.floor(65536 * p + 0.5))
    bits = np.empty(n, bool)
    m32 = 0xFFFFFFFF
    for g in range(-(-n // 8)):
        block = (offset + g) & 0xFFFFFFFFFFFFFFFF
        c = [block & m32, block >> 32, 0, 0]
        k = [seed & m32, (seed >> 32) & m32]
        for _ in range(10):
            p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & m32, (p0 >> 32) ^ c[3] ^ k[1], p0 & m32]
            k = [(k[0] + 0x9E3779B9) & m32, (k[1] + 0xBB67AE85) & m32]
        for j in range(8):
            if 8 * g + j < n:
                u = c[j // 2] >> 16 if j & 1 else c[j // 2] & 0xFFFF
                bits[8 * g + j] = u >= t
    return bits.reshape(rows, cols), (65536.0 / (65536 - t) if t < 65536 else 0.0)
