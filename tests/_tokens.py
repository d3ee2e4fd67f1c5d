"""Embedding, linear layer, residual norm and 8-bit matrices in 64 bits (numpy), from their definitions,
with bounds on how far results in fewer bits may be off: those of tests/_network.py, carried on by first
order (an error e of a value that a function of slope s takes is s e of its result)."""
import numpy as np

from . import _network as N

EPS = N.EPS


def rounded(v, e, kind):
    """A bound e of a value v and the rounding to its type."""
    return e + (np.abs(v) + e) * N.UNIT[kind] + N.TINY[kind]


# ---- embedding

def embed(table, index, scale, add):
    y = np.zeros((len(index), table.shape[1]))
    named = (index >= 0) & (index < len(table))
    y[named] = scale * table[index[named]]
    return y if add is None else y + add


def embed_bound(table, index, scale, add, kind):
    """A product and a sum."""
    y = embed(table, index, scale, add)
    part = np.abs(embed(table, index, scale, None))
    return rounded(y, 2 * EPS * (part + (0 if add is None else np.abs(add))), kind)


def embed_grad(dy, index, scale, rows):
    d = np.zeros((rows, dy.shape[1]))
    named = (index >= 0) & (index < rows)
    np.add.at(d, index[named], dy[named])
    return scale * d


def embed_grad_bound(dy, index, scale, rows, kind):
    named = (index >= 0) & (index < rows)
    count = np.bincount(index[named], minlength=rows)[:, None]
    e = (count + 8) * EPS * embed_grad(np.abs(dy), index, abs(scale), rows)
    return rounded(embed_grad(dy, index, scale, rows), e, kind)


# ---- linear layer

def act(z, name):
    return z if name == "none" else N.act(z, name)


def slope(z, name):
    return np.ones_like(z) if name == "none" else N.slope(z, name)


def linear(x, w, b, name, residual):
    z = x @ w.T + b
    return residual + act(z, name), z


def linear_bounds(x, w, b, name, residual, kind):
    """Bounds of y and z."""
    k = x.shape[1]
    y, z = linear(x, w, b, name, residual)
    ez = (k + 9) * EPS * (np.abs(x) @ np.abs(w).T + np.abs(b))
    ey = 1.2 * ez + 16 * EPS * np.abs(z) + 2 * EPS * np.abs(residual)
    return rounded(y, ey, kind), rounded(z, ez, kind)


def linear_grad(dy, x, w, name, z):
    """dx, dweight, dbias from the saved z."""
    dz = dy * slope(z, name)
    return dz @ w, dz.T @ x, dz.sum(0)


def linear_grad_bounds(dy, x, w, name, z, kind, bkind):
    m, n = dy.shape
    A = np.abs
    dz = dy * slope(z, name)
    e = A(dy) * (16 * EPS * (1 + A(z)) + 4 * EPS * A(slope(z, name))) if name != "none" else np.zeros_like(dy)
    er = rounded(dz, e, kind) if name != "none" else e
    dx, dw, db = linear_grad(dy, x, w, name, z)
    return (rounded(dx, er @ A(w) + (n + 8) * EPS * ((A(dz) + er) @ A(w)), kind),
            rounded(dw, er.T @ A(x) + (m + 8) * EPS * ((A(dz) + er).T @ A(x)), kind),
            rounded(db, e.sum(0) + (m + 16) * EPS * A(dz).sum(0), bkind))


# ---- the norms around a residual sum

def stats(v, kind, eps):
    """(mean, rstd) of the rows."""
    mean = v.mean(1, keepdims=True) if kind == "layer" else np.zeros((len(v), 1))
    return mean, 1.0 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)


class Close:
    """y = x + A fh + C, n = yh w2 + b2.  after, before: None or (kind, weight, bias); vectors [cols]."""

    def __init__(self, cols, after, before, gate, scale, eps=1e-5):
        one, zero = np.ones(cols), np.zeros(cols)
        self.after, self.before, self.eps, self.scale = after, before, eps, scale
        self.kind = tuple(q[0] if q else None for q in (after, before))
        self.w = tuple(one if not q or q[1] is None else q[1] for q in (after, before))
        self.b = tuple(zero if not q or q[2] is None else q[2] for q in (after, before))
        self.gate = one if gate is None else gate
        self.A, self.C = scale * self.gate * self.w[0], scale * self.gate * self.b[0]

    def given(self, v, k, mean, rstd):
        """Normalised rows by statistics that are given."""
        return v if self.kind[k] is None else (v - mean) * rstd

    def forward(self, x, f):
        """y, n (or None) and [mean, rstd] of both norms."""
        s = [np.zeros((len(x), 1)), np.ones((len(x), 1))] * 2
        if self.after:
            s[:2] = stats(f, self.kind[0], self.eps)
        y = x + self.A * self.given(f, 0, *s[:2]) + self.C
        if not self.before:
            return y, None, s
        s[2:] = stats(y, self.kind[1], self.eps)
        return y, self.given(y, 1, *s[2:]) * self.w[1] + self.b[1], s

    def _own(self, v, k, mean, rstd):
        """How far normalised rows are off by their own arithmetic: the mean by (n + 8) EPS mean|v|, the
        variance by twice that sum against the deviations, an rms by the sum alone."""
        if self.kind[k] is None:
            return np.zeros_like(v)
        n = v.shape[1]
        if self.kind[k] == "rms":
            return (n + 16) * EPS * np.abs(v) * rstd
        mag = np.abs(v).mean(1, keepdims=True)
        return (2 * n + 24) * EPS * ((np.abs(v) + mag) * rstd + np.abs(v - mean) * rstd * (1 + mag * rstd))

    def forward_bounds(self, x, f, kind):
        y, n, s = self.forward(x, f)
        fh = self.given(f, 0, *s[:2])
        ey = np.abs(self.A) * self._own(f, 0, *s[:2]) + 8 * EPS * (np.abs(x) + np.abs(self.A * fh) + np.abs(self.C))
        if n is None:
            return rounded(y, ey, kind), None
        mean, rstd = s[2:]
        yh = self.given(y, 1, mean, rstd)
        e = self._own(y, 1, mean, rstd) + rstd * (ey + ey.mean(1, keepdims=True)) \
            + np.abs(yh) * rstd * (np.abs(yh) * ey).mean(1, keepdims=True)
        en = np.abs(self.w[1]) * e + 8 * EPS * (np.abs(yh * self.w[1]) + np.abs(self.b[1]))
        return rounded(y, ey, kind), rounded(n, en, kind)

    def _values(self, x, f, s):
        fh = self.given(f, 0, *s[:2])
        y = x + self.A * fh + self.C
        return fh, y, self.given(y, 1, *s[2:])

    def _through(self, k, g, vh, rstd):
        """The rows' gradient through norm k from that of its normalised rows."""
        if self.kind[k] is None:
            return g
        mean = g.mean(1, keepdims=True) if self.kind[k] == "layer" else 0.0
        return rstd * (g - mean - vh * (g * vh).mean(1, keepdims=True))

    def backward(self, dy, dn, x, f, s):
        """dx, df, dgate, dafter_weight, dafter_bias, dbefore_weight, dbefore_bias."""
        fh, y, yh = self._values(x, f, s)
        g = dy if dn is None else dy + self._through(1, dn * self.w[1], yh, s[3])
        u = self.A * g
        df = self._through(0, u, fh, s[1])
        dn0 = np.zeros_like(x) if dn is None else dn
        sg = self.scale * self.gate
        return (g, df, self.scale * (g * (fh * self.w[0] + self.b[0])).sum(0), sg * (g * fh).sum(0), sg * g.sum(0),
                (dn0 * yh).sum(0), dn0.sum(0))

    def backward_bounds(self, dy, dn, x, f, s, kind, wkind):
        A, k, kc = np.abs, (x.shape[1] + 16) * EPS, (len(x) + 16) * EPS
        mean = lambda v: v.mean(1, keepdims=True)
        fh, y, yh = self._values(x, f, s)
        m1, r1, m2, r2 = s
        efh = 8 * EPS * (A(f) + A(m1)) * r1 if self.after else np.zeros_like(f)
        ey = A(self.A) * efh + 8 * EPS * (A(x) + A(self.A * fh) + A(self.C))
        eyh = r2 * ey + 8 * EPS * (A(y) + A(m2)) * r2 if self.before else ey

        def through(g, eg, vh, evh, rstd):
            """_through of values that are off by eg and evh."""
            s2 = mean(A(g * vh))
            e2 = k * s2 + mean(A(g) * evh + eg * A(vh))
            return rstd * (eg + mean(eg) + 8 * EPS * A(g) + k * mean(A(g)) + A(vh) * e2 + evh * s2 + 8 * EPS * A(vh) * s2)

        g = dy if dn is None else dy + self._through(1, dn * self.w[1], yh, r2)
        eg = 4 * EPS * A(dy) if dn is None else \
            4 * EPS * (A(dy) + A(g)) + through(dn * self.w[1], 4 * EPS * A(dn * self.w[1]), yh, eyh, r2)
        u = self.A * g
        eu = A(self.A) * (eg + 8 * EPS * A(g))
        edf = through(u, eu, fh, efh, r1) if self.after else eu
        out = self.backward(dy, dn, x, f, s)
        sg = A(self.scale * self.gate)
        e1 = eg.sum(0) + kc * A(g).sum(0)
        e2 = (eg * A(fh) + (A(g) + eg) * efh).sum(0) + kc * A(g * fh).sum(0)
        dn0 = np.zeros_like(x) if dn is None else A(dn)
        errors = (eg, edf, abs(self.scale) * (A(self.w[0]) * e2 + A(self.b[0]) * e1
                                              + 8 * EPS * (A(self.w[0]) * A(g * fh).sum(0) + A(self.b[0]) * A(g).sum(0))),
                  sg * (e2 + 8 * EPS * A(g * fh).sum(0)), sg * (e1 + 8 * EPS * A(g).sum(0)),
                  (dn0 * eyh).sum(0) + kc * (dn0 * A(yh)).sum(0), kc * dn0.sum(0))
        return tuple(rounded(v, e, t) for v, e, t in zip(out, errors, (kind,) * 2 + (wkind,) * 5))


# ---- 8 bits

def packed(x):
    """(codes, powers) of float64 values: groups of 32 columns."""
    rows, cols = x.shape
    groups = -(-cols // 32)
    v = np.zeros((rows, 32 * groups))
    v[:, :cols] = x
    v = v.reshape(rows, groups, 32)
    finite = np.isfinite(v).all(2)
    top = np.abs(np.where(finite[..., None], v, 0.0)).max(2)
    e = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 1, -1000)
    p = np.maximum(e - 6 + 127, 1)
    q = np.clip(np.rint(np.where(finite[..., None], v, 0.0) * 2.0 ** (127.0 - p[..., None])), -127, 127)
    return q.reshape(rows, -1)[:, :cols].astype(np.int8), np.where(finite, p, 255).astype(np.uint8)


def unpacked(codes, powers):
    cols = codes.shape[1]
    p = np.repeat(powers, 32, 1)[:, :cols].astype(np.float64)
    return np.where(p == 255, np.nan, codes * 2.0 ** (p - 127))
