"""Operators of a network over a block's Gaussians (layer norm, gated feed-forward, dropout; embedding,
linear layer, the norms around a residual sum, matrices in 8 bits): the calls of ``include/abcd.h`` of the
same names, and the residual blocks that they make up.

Matrices are CUDA tensors [rows][cols] whose columns are consecutive (rows may be further apart);
types float32, float16 or bfloat16.  The calls run on the context's stream: tensors that another
stream fills or frees need that stream's events, as everywhere in this package."""
from __future__ import annotations

import struct

from dataclasses import dataclass

from . import (ABCD_GELU, ABCD_I32, ABCD_I64, ABCD_LAYER_NORM, ABCD_NO_ACTIVATION, ABCD_RELU,
               ABCD_RMS_NORM, ABCD_SILU, Context, _dtypes, _torch, lib)

ACTIVATIONS = {"silu": ABCD_SILU, "gelu": ABCD_GELU, "relu": ABCD_RELU}
LINEAR_ACTIVATIONS = {**ACTIVATIONS, "none": ABCD_NO_ACTIVATION}
NORMS = {"layer": ABCD_LAYER_NORM, "rms": ABCD_RMS_NORM}


_F32 = None
_KINDS = {}
_CALLS = {}


def _call(name):
    """The library's function; looked up once (these calls are short, and so is their host time)."""
    global _F32
    f = _CALLS.get(name)
    if f is None:
        _F32 = _torch().float32
        _KINDS.update(_dtypes())
        f = _CALLS[name] = getattr(lib(), name)
    return f


# The bytes of an abcd_matrix.  ctypes hands on the address of a bytes object as it is, which takes a
# quarter of the time that it takes to make a Structure and a reference to it (0.1 us instead of 0.4).
_pack = struct.Struct("@Pqqqi0q").pack


def _matrix(t, what):
    """(abcd_matrix as bytes, rows, columns) of a 2-D CUDA tensor."""
    try:
        rows, cols = t.shape
        stride, unit = t.stride()
    except ValueError:
        raise ValueError(f"{what} must be a 2-D CUDA tensor") from None
    if not t.is_cuda:
        raise ValueError(f"{what} must be a 2-D CUDA tensor")
    if unit != 1 and cols > 1:
        raise ValueError(f"{what} must have consecutive columns")
    kind = _KINDS.get(t.dtype)
    if kind is None:
        raise ValueError(f"{what} has type {t.dtype}; float32, float16 and bfloat16 are taken")
    if rows <= 1 and stride < cols:
        stride = cols
    return _pack(t.data_ptr(), rows, cols, stride, kind), rows, cols


def _optional(t, what):
    return None if t is None else _matrix(t, what)[0]


def _vector(t, n, what, dtype):
    """Address of a consecutive CUDA vector of n elements (None for None)."""
    if t is None:
        return None
    if not t.is_cuda or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} must be a consecutive CUDA vector of {n} elements")
    if t.dtype is not dtype:
        raise ValueError(f"{what} has type {t.dtype}, not {dtype}")
    return t.data_ptr()


def _weight_type(x, *vectors):
    """The torch type of the given weight vectors (x's or float32, one for all)."""
    for v in vectors:
        if v is not None:
            if v.dtype is not x.dtype and v.dtype is not _F32:
                raise ValueError("weights are of the matrices' type or float32")
            return v.dtype
    return x.dtype


def _activation(name):
    act = ACTIVATIONS.get(name)
    if act is None:
        raise ValueError(f"unknown activation {name!r}; one of {sorted(ACTIVATIONS)}")
    return act


def abcd_layer_norm(ctx: Context, x, weight, bias, eps, y, mean=None, rstd=None):
    """y = layer norm of x's rows; weight, bias: [cols] or None; mean, rstd: float32 [rows] that the
    backward pass needs, or None."""
    call = _call("abcd_layer_norm")
    mx, rows, cols = _matrix(x, "x")
    wt = _weight_type(x, weight, bias)
    st = call(ctx.h, mx, _vector(weight, cols, "weight", wt), _vector(bias, cols, "bias", wt),
              _KINDS[wt], eps, _matrix(y, "y")[0], _vector(mean, rows, "mean", _F32),
              _vector(rstd, rows, "rstd", _F32))
    if st:
        ctx.check(st)


def abcd_layer_norm_backward(ctx: Context, dy, x, weight, mean, rstd, dx=None, dweight=None,
                             dbias=None, d_residual=None):
    """dx, dweight and dbias (each may be None) of abcd_layer_norm; d_residual is added to dx (which
    may be dy or d_residual).  Takes the network workspace (Context.reserve_network)."""
    call = _call("abcd_layer_norm_backward")
    mx, rows, cols = _matrix(x, "x")
    wt = _weight_type(x, weight, dweight, dbias)
    st = call(ctx.h, _matrix(dy, "dy")[0], mx, _vector(weight, cols, "weight", wt), _KINDS[wt],
              _vector(mean, rows, "mean", _F32), _vector(rstd, rows, "rstd", _F32),
              _optional(d_residual, "d_residual"), _optional(dx, "dx"),
              _vector(dweight, cols, "dweight", wt), _vector(dbias, cols, "dbias", wt))
    if st:
        ctx.check(st)


def abcd_gated_ff(ctx: Context, x, w_gate, w_up, w_down, activation, y, gate=None, up=None):
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T; gate, up: [rows][ff] that the backward pass
    needs, or None; activation: "silu", "gelu" or "relu".  Takes the network workspace."""
    call = _call("abcd_gated_ff")
    st = call(ctx.h, _matrix(x, "x")[0], _matrix(w_gate, "w_gate")[0],
              _matrix(w_up, "w_up")[0], _matrix(w_down, "w_down")[0],
              _activation(activation), _matrix(y, "y")[0], _optional(gate, "gate"),
              _optional(up, "up"))
    if st:
        ctx.check(st)


def abcd_gated_ff_backward(ctx: Context, dy, x, w_gate, w_up, w_down, activation, gate, up,
                           dx=None, dw_gate=None, dw_up=None, dw_down=None):
    """dx and the weights' gradients (each may be None) of abcd_gated_ff, from what its forward call
    left in gate and up.  Takes the network workspace."""
    call = _call("abcd_gated_ff_backward")
    st = call(ctx.h, _matrix(dy, "dy")[0], _matrix(x, "x")[0],
              _matrix(w_gate, "w_gate")[0], _matrix(w_up, "w_up")[0],
              _matrix(w_down, "w_down")[0], _activation(activation),
              _matrix(gate, "gate")[0], _matrix(up, "up")[0], _optional(dx, "dx"),
              _optional(dw_gate, "dw_gate"), _optional(dw_up, "dw_up"),
              _optional(dw_down, "dw_down"))
    if st:
        ctx.check(st)


def abcd_dropout(ctx: Context, x, p, seed, offset, y, residual=None):
    """y = residual + dropout(x) with the mask of (seed, offset); y may be x or residual.  The next
    call's offset is past this one's: offset + ceil(rows * cols / 8)."""
    call = _call("abcd_dropout")
    st = call(ctx.h, _matrix(x, "x")[0], p, seed, offset, _optional(residual, "residual"),
              _matrix(y, "y")[0])
    if st:
        ctx.check(st)


def abcd_dropout_backward(ctx: Context, dy, p, seed, offset, dx):
    """dx = dropout's gradient of dy under the mask of (seed, offset); dx may be dy."""
    call = _call("abcd_dropout_backward")
    st = call(ctx.h, _matrix(dy, "dy")[0], p, seed, offset, _matrix(dx, "dx")[0])
    if st:
        ctx.check(st)


def _index(t, n):
    """(address, ABCD_* type) of a consecutive CUDA vector of n indices."""
    if not t.is_cuda or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"index must be a consecutive CUDA vector of {n} elements")
    torch = _torch()
    if t.dtype is torch.int64:
        return t.data_ptr(), ABCD_I64
    if t.dtype is torch.int32:
        return t.data_ptr(), ABCD_I32
    raise ValueError(f"index has type {t.dtype}; int32 and int64 are taken")


def abcd_embedding(ctx: Context, table, index, scale, y, add=None):
    """y[t] = add[t] + scale table[index[t]]; index: int32 or int64, negative ones name no row.  One that is
    past the table is reported by ctx.sync().  y may be add.  Takes the network workspace
    (Context.reserve_embedding)."""
    call = _call("abcd_embedding")
    my, rows, _ = _matrix(y, "y")
    at, kind = _index(index, rows)
    st = call(ctx.h, _matrix(table, "table")[0], at, kind, scale, _optional(add, "add"), my)
    if st:
        ctx.check(st)


def abcd_embedding_backward(ctx: Context, dy, index, scale, dtable):
    """dtable[v] = scale times the sum of dy[t] over the tokens that name row v; every row is written.
    Takes the network workspace (Context.reserve_embedding)."""
    call = _call("abcd_embedding_backward")
    my, rows, _ = _matrix(dy, "dy")
    at, kind = _index(index, rows)
    st = call(ctx.h, my, at, kind, scale, _matrix(dtable, "dtable")[0])
    if st:
        ctx.check(st)


def _linear_activation(name):
    act = LINEAR_ACTIVATIONS.get(name)
    if act is None:
        raise ValueError(f"unknown activation {name!r}; one of {sorted(LINEAR_ACTIVATIONS)}")
    return act


def abcd_linear(ctx: Context, x, weight, bias, activation, y, residual=None, z=None):
    """y = residual + act(z), z = x weight^T + bias; weight [out][cols]; bias [out] or None; activation
    "none", "silu", "gelu" or "relu"; z: kept for the backward pass, or None.  y may be residual.  Takes
    the network workspace (Context.reserve_linear)."""
    call = _call("abcd_linear")
    mx = _matrix(x, "x")[0]
    mw, out, _ = _matrix(weight, "weight")
    bt = _weight_type(x, bias)
    st = call(ctx.h, mx, mw, _vector(bias, out, "bias", bt), _KINDS[bt], _linear_activation(activation),
              _optional(residual, "residual"), _matrix(y, "y")[0], _optional(z, "z"))
    if st:
        ctx.check(st)


def abcd_linear_backward(ctx: Context, dy, x, weight, activation, z, dx=None, dweight=None, dbias=None):
    """dx, dweight and dbias (each may be None) of abcd_linear from the z that it left (None for "none").
    The residual's gradient is dy.  Takes the network workspace (Context.reserve_linear)."""
    call = _call("abcd_linear_backward")
    mw, out, _ = _matrix(weight, "weight")
    bt = _weight_type(x, dbias)
    st = call(ctx.h, _matrix(dy, "dy")[0], _matrix(x, "x")[0], mw, _linear_activation(activation),
              _optional(z, "z"), _optional(dx, "dx"), _optional(dweight, "dweight"),
              _vector(dbias, out, "dbias", bt), _KINDS[bt])
    if st:
        ctx.check(st)


@dataclass(slots=True)
class Norm:
    """A norm of abcd_residual_norm: kind "layer" or "rms"; weight, bias: [cols] or None; mean, rstd:
    float32 [rows] that the backward pass needs, or None (an rms norm has no mean; one that is given is
    left as it is)."""
    kind: str
    weight: object = None
    bias: object = None
    eps: float = 1e-5
    mean: object = None
    rstd: object = None


_pack_norm = struct.Struct("@iPPfPP").pack           # the bytes of an abcd_norm


_AFTER = "after.weight", "after.bias", "after.mean", "after.rstd"
_BEFORE = "before.weight", "before.bias", "before.mean", "before.rstd"


def _norm(q, rows, cols, dtype, names):
    if q is None:
        return None
    kind = NORMS.get(q.kind)
    if kind is None:
        raise ValueError(f"unknown norm {q.kind!r}; one of {sorted(NORMS)}")
    w, b, m, r = q.weight, q.bias, q.mean, q.rstd
    return _pack_norm(kind, 0 if w is None else _vector(w, cols, names[0], dtype),
                      0 if b is None else _vector(b, cols, names[1], dtype), q.eps,
                      0 if m is None or kind == ABCD_RMS_NORM else _vector(m, rows, names[2], _F32),
                      0 if r is None else _vector(r, rows, names[3], _F32))


def _norm_vectors(after, before):
    a = () if after is None else (after.weight, after.bias)
    return a if before is None else (*a, before.weight, before.bias)


def abcd_residual_norm(ctx: Context, x, f, after, before, gate, scale, y, n=None):
    """y = x + scale gate after(f), n = before(y): after and before Norms or None, gate [cols] or None;
    n as before is.  All vectors are of one type (the matrices' or float32).  y and n may be x or f."""
    call = _call("abcd_residual_norm")
    mx, rows, cols = _matrix(x, "x")
    wt = _weight_type(x, gate, *_norm_vectors(after, before))
    st = call(ctx.h, mx, _matrix(f, "f")[0], _norm(after, rows, cols, wt, _AFTER),
              _norm(before, rows, cols, wt, _BEFORE), _vector(gate, cols, "gate", wt), _KINDS[wt], scale,
              _matrix(y, "y")[0], _optional(n, "n"))
    if st:
        ctx.check(st)


def abcd_residual_norm_backward(ctx: Context, dy, dn, x, f, after, before, gate, scale, dx=None, df=None,
                                dgate=None, dafter_weight=None, dafter_bias=None, dbefore_weight=None,
                                dbefore_bias=None):
    """The gradients (each may be None) of abcd_residual_norm from x, f and the statistics that it left in
    after and before; dy: the gradient that reaches y past n, or None; dn: n's, as before is.  dx and df
    may be dy, dn, x or f.  Takes the network workspace (Context.reserve_residual_norm)."""
    call = _call("abcd_residual_norm_backward")
    mx, rows, cols = _matrix(x, "x")
    wt = _weight_type(x, gate, dgate, dafter_weight, dafter_bias, dbefore_weight, dbefore_bias,
                      *_norm_vectors(after, before))
    v = lambda t, what: _vector(t, cols, what, wt)
    st = call(ctx.h, _optional(dy, "dy"), _optional(dn, "dn"), mx, _matrix(f, "f")[0],
              _norm(after, rows, cols, wt, _AFTER), _norm(before, rows, cols, wt, _BEFORE),
              v(gate, "gate"), _KINDS[wt], scale, _optional(dx, "dx"), _optional(df, "df"),
              v(dgate, "dgate"), v(dafter_weight, "dafter_weight"), v(dafter_bias, "dafter_bias"),
              v(dbefore_weight, "dbefore_weight"), v(dbefore_bias, "dbefore_bias"))
    if st:
        ctx.check(st)


class Packed8:
    """A matrix of rows x cols in 8 bits: `codes`, int8, its rows `stride` bytes apart, and `powers`, uint8,
    one for each 32 columns of a row.  Allocated on the current stream (Context.hold for a context on
    another one)."""

    def __init__(self, rows, cols, device="cuda"):
        torch = _torch()
        rows, cols = int(rows), int(cols)
        groups = -(-cols // 32)
        self.rows, self.cols, self.stride = rows, cols, 32 * groups
        self.codes = torch.empty(rows, self.stride, dtype=torch.int8, device=device)
        self.powers = torch.empty(rows, groups, dtype=torch.uint8, device=device)
        self._at(self.codes.data_ptr(), self.powers.data_ptr(), rows)

    def _at(self, codes, powers, rows):
        self.c = _pack_packed(codes, powers, rows, self.cols, self.stride, self.stride // 32)

    def head(self, rows):
        """Its first rows, as a packed matrix over the same memory."""
        if not 0 <= rows <= self.rows:
            raise ValueError(f"{rows} of {self.rows} rows")
        part = Packed8.__new__(Packed8)
        part.rows, part.cols, part.stride = int(rows), self.cols, self.stride
        part.codes, part.powers = self.codes[:rows], self.powers[:rows]
        part._at(part.codes.data_ptr(), part.powers.data_ptr(), part.rows)
        return part


_pack_packed = struct.Struct("@PPqqqq").pack         # the bytes of an abcd_packed8


def _packed(q, what):
    """The abcd_packed8 as bytes of a Packed8 in device memory."""
    if not isinstance(q, Packed8) or not q.codes.is_cuda:
        raise ValueError(f"{what} must be a Packed8 of CUDA memory")
    return q.c


def abcd_pack8(ctx: Context, x, packed: Packed8):
    """packed = x in 8 bits: an element is off by at most a 128th of the largest magnitude of the 32 columns
    that share its power of two."""
    st = _call("abcd_pack8")(ctx.h, _matrix(x, "x")[0], _packed(packed, "packed"))
    if st:
        ctx.check(st)


def abcd_unpack8(ctx: Context, packed: Packed8, y):
    """y = what packed stands for."""
    st = _call("abcd_unpack8")(ctx.h, _packed(packed, "packed"), _matrix(y, "y")[0])
    if st:
        ctx.check(st)


def abcd_gated_ff_backward_packed8(ctx: Context, dy, x, w_gate, w_up, w_down, activation, gate, up,
                                   dx=None, dw_gate=None, dw_up=None, dw_down=None):
    """abcd_gated_ff_backward with x, gate and up as Packed8.  Takes the network workspace
    (Context.reserve_packed8)."""
    call = _call("abcd_gated_ff_backward_packed8")
    st = call(ctx.h, _matrix(dy, "dy")[0], _packed(x, "x"), _matrix(w_gate, "w_gate")[0], _matrix(w_up, "w_up")[0],
              _matrix(w_down, "w_down")[0], _activation(activation), _packed(gate, "gate"), _packed(up, "up"), _optional(dx, "dx"),
              _optional(dw_gate, "dw_gate"), _optional(dw_up, "dw_up"), _optional(dw_down, "dw_down"))
    if st:
        ctx.check(st)


class FeedForwardBlock:
    """The residual block x + dropout(gated_ff(layer_norm(x))) over up to `rows` tokens of width
    `cols`, with the buffers that its backward pass reads.

    weights: {"norm_w", "norm_b": [cols], "w_gate", "w_up": [ff][cols], "w_down": [cols][ff]} CUDA
    tensors of type dtype; `grads` holds their gradients under the same names after backward()."""

    def __init__(self, ctx: Context, weights, rows, activation="silu", eps=1e-5, p=0.0, seed=0):
        torch = _torch()
        self.ctx, self.w = ctx, dict(weights)
        self.ff, self.cols = self.w["w_gate"].shape
        self.act, self.eps, self.p, self.seed = activation, float(eps), float(p), int(seed)
        self.rows = int(rows)
        dt, dev = self.w["w_gate"].dtype, self.w["w_gate"].device
        new = lambda n, c: torch.empty(n, c, dtype=dt, device=dev)
        self.normed, self.out = new(self.rows, self.cols), new(self.rows, self.cols)
        self.gate, self.up = new(self.rows, self.ff), new(self.rows, self.ff)
        self.d_out, self.d_normed = new(self.rows, self.cols), new(self.rows, self.cols)
        self.mean = torch.empty(self.rows, dtype=torch.float32, device=dev)
        self.rstd = torch.empty_like(self.mean)
        self.grads = {k: torch.empty_like(t) for k, t in self.w.items()}
        self.offset = 0
        self.kept = None                                # rows of the last training pass
        ctx.hold(self.normed, self.out, self.gate, self.up, self.d_out, self.d_normed, self.mean, self.rstd,
                 *self.grads.values())
        ctx.reserve_network(self.rows, self.cols, self.ff, dt)

    def _counters(self, rows):
        return (rows * self.cols + 7) // 8

    def forward(self, x, y, train=True):
        """y = the block of x (both [rows'][cols], rows' <= rows).  train: keep what the backward pass
        needs (x among it: y is another matrix), and drop with the next counters of the block's
        generator; otherwise y may be x, and what an earlier pass kept stays."""
        n, w = x.shape[0], self.w
        if not train:
            # in the backward pass's buffers: what the last training pass kept stays
            nx, out = self.d_normed[:n], self.d_out[:n]
            abcd_layer_norm(self.ctx, x, w["norm_w"], w["norm_b"], self.eps, nx)
            abcd_gated_ff(self.ctx, nx, w["w_gate"], w["w_up"], w["w_down"], self.act, out)
            abcd_dropout(self.ctx, out, 0.0, self.seed, 0, y, x)
            return
        nx, out = self.normed[:n], self.out[:n]
        self.kept, self.drawn = None, self.offset
        self.offset += self._counters(n)
        abcd_layer_norm(self.ctx, x, w["norm_w"], w["norm_b"], self.eps, nx, self.mean[:n],
                        self.rstd[:n])
        abcd_gated_ff(self.ctx, nx, w["w_gate"], w["w_up"], w["w_down"], self.act, out,
                      self.gate[:n], self.up[:n])
        abcd_dropout(self.ctx, out, self.p, self.seed, self.drawn, y, x)
        self.kept = n

    def backward(self, dy, x, dx):
        """dx (may be dy) and `grads` of the last forward(x, ..., train=True); x as it was given."""
        n, w, g = x.shape[0], self.w, self.grads
        if n != self.kept:
            raise ValueError(f"x has {n} rows, the last training pass {self.kept}")
        d_out, d_nx = self.d_out[:n], self.d_normed[:n]
        abcd_dropout_backward(self.ctx, dy, self.p, self.seed, self.drawn, d_out)
        abcd_gated_ff_backward(self.ctx, d_out, self.normed[:n], w["w_gate"], w["w_up"],
                               w["w_down"], self.act, self.gate[:n], self.up[:n], d_nx,
                               g["w_gate"], g["w_up"], g["w_down"])
        abcd_layer_norm_backward(self.ctx, d_nx, x, w["norm_w"], self.mean[:n], self.rstd[:n], dx,
                                 g["norm_w"], g["norm_b"], dy)


class NormedStack:
    """Residual blocks with a norm before and one after: block k takes n = before_k(x) to
    x + scale gate_k after_k(gated_ff(n)), whose sum, gate and both norms around it (the next block's
    `before` among them) are one call.  Up to `rows` tokens; `before` is a layer norm, `after` an rms norm.

    weights: for each block {"before_w", "before_b", "after_w", "gate": [cols], "w_gate", "w_up": [ff][cols],
    "w_down": [cols][ff]}, CUDA tensors of one type; `grads` holds their gradients under the same names
    after backward().  packed: what a block keeps for its backward pass of its normed tokens and its
    projections is in 8 bits (33/32 bytes an element instead of two or four); the gradients are then those
    of what the packed matrices stand for."""

    def __init__(self, ctx: Context, weights, rows, activation="silu", scale=1.0, eps=1e-5, packed=False):
        torch = _torch()
        self.ctx, self.w, self.rows = ctx, [dict(w) for w in weights], int(rows)
        self.act, self.scale, self.eps, self.packed = activation, float(scale), float(eps), bool(packed)
        self.ff, self.cols = self.w[0]["w_gate"].shape
        dt, dev = self.w[0]["w_gate"].dtype, self.w[0]["w_gate"].device
        new = lambda c: torch.empty(self.rows, c, dtype=dt, device=dev)
        blocks = len(self.w)
        self.x = [new(self.cols) for _ in range(blocks)]             # the blocks' inputs
        self.f = [new(self.cols) for _ in range(blocks)]             # their feed-forward results
        self.stats = torch.empty(blocks, 4, self.rows, dtype=torch.float32, device=dev)
        # mean and rstd of a block's `before`, rstd of its `after`
        full = 1 if packed else blocks
        self.normed, self.gate, self.up = ([new(c) for _ in range(full)] for c in (self.cols, self.ff, self.ff))
        self.d, self.df = [new(self.cols) for _ in range(2)], new(self.cols)
        self.kept8 = [[Packed8(self.rows, c, dev) for c in (self.cols, self.ff, self.ff)] for _ in range(blocks)] if packed else []
        self.grads = [{k: torch.empty_like(t) for k, t in w.items()} for w in self.w]
        self.kept = None                                             # rows of the last training pass
        ctx.hold(*self.x, *self.f, self.stats, *self.normed, *self.gate, *self.up, *self.d, self.df,
                 *(t for g in self.grads for t in g.values()), *(t for q in self.kept8 for m in q for t in (m.codes, m.powers)))
        (ctx.reserve_packed8 if packed else ctx.reserve_network)(self.rows, self.cols, self.ff, dt)
        ctx.reserve_residual_norm(self.rows, self.cols)
        ctx.reserve_network(self.rows, self.cols)                    # the first norm's backward pass

    def _norms(self, k, n, train=True):
        """`after` of block k and `before` of the next one (None after the last), over n rows."""
        stat = lambda b, i: self.stats[b, i, :n] if train else None
        after = Norm("rms", self.w[k]["after_w"], None, self.eps, None, stat(k, 2))
        if k + 1 == len(self.w):
            return after, None
        nxt = self.w[k + 1]
        return after, Norm("layer", nxt["before_w"], nxt["before_b"], self.eps, stat(k + 1, 0), stat(k + 1, 1))

    def forward(self, x, y, train=True):
        """y = the blocks of x (both [rows'][cols], rows' <= rows).  train: keep what the backward pass
        needs; otherwise what an earlier pass kept stays, and y may be x."""
        n, ctx, first = x.shape[0], self.ctx, self.w[0]
        if not train:
            # in the backward pass's buffers
            at, normed, f = self.d[0][:n], self.d[1][:n], self.df[:n]
            abcd_layer_norm(ctx, x, first["before_w"], first["before_b"], self.eps, normed)
            for k, w in enumerate(self.w):
                abcd_gated_ff(ctx, normed, w["w_gate"], w["w_up"], w["w_down"], self.act, f)
                after, before = self._norms(k, n, False)
                last = before is None
                abcd_residual_norm(ctx, x, f, after, before, w["gate"], self.scale, y if last else at, None if last else normed)
                x = at
            return
        self.kept = None
        with ctx.on_stream():
            self.x[0][:n].copy_(x)
        s = self.stats[0]
        abcd_layer_norm(ctx, self.x[0][:n], first["before_w"], first["before_b"], self.eps, self.normed[0][:n], s[0, :n], s[1, :n])
        for k, w in enumerate(self.w):
            b = 0 if self.packed else k
            normed, gate, up, f = self.normed[b][:n], self.gate[b][:n], self.up[b][:n], self.f[k][:n]
            abcd_gated_ff(ctx, normed, w["w_gate"], w["w_up"], w["w_down"], self.act, f, gate, up)
            if self.packed:
                for t, q in zip((normed, gate, up), self.kept8[k]):
                    abcd_pack8(ctx, t, q.head(n))
            after, before = self._norms(k, n)
            last = before is None
            to = y if last else self.x[k + 1][:n]
            abcd_residual_norm(ctx, self.x[k][:n], f, after, before, w["gate"], self.scale, to,
                               None if last else self.normed[0 if self.packed else k + 1][:n])
        self.kept = n

    def backward(self, dy, dx):
        """dx (may be dy) and `grads` of the last forward(..., train=True) from its result's gradient."""
        n, ctx, blocks = dy.shape[0], self.ctx, len(self.w)
        if n != self.kept:
            raise ValueError(f"dy has {n} rows, the last training pass {self.kept}")
        d, dn, df = dy, None, self.df[:n]
        for k in reversed(range(blocks)):
            w, g = self.w[k], self.grads[k]
            after, before = self._norms(k, n)
            nxt = {} if before is None else self.grads[k + 1]
            to = self.d[0][:n]
            abcd_residual_norm_backward(ctx, d, dn, self.x[k][:n], self.f[k][:n], after, before, w["gate"], self.scale,
                                        to, df, g["gate"], g["after_w"], None, nxt.get("before_w"), nxt.get("before_b"))
            d, dn = to, self.d[1][:n]
            out = dn, g["w_gate"], g["w_up"], g["w_down"]
            if self.packed:
                q = [m.head(n) for m in self.kept8[k]]
                abcd_gated_ff_backward_packed8(ctx, df, q[0], w["w_gate"], w["w_up"], w["w_down"], self.act, q[1], q[2], *out)
            else:
                abcd_gated_ff_backward(ctx, df, self.normed[k][:n], w["w_gate"], w["w_up"], w["w_down"], self.act,
                                       self.gate[k][:n], self.up[k][:n], *out)
        s, g = self.stats[0], self.grads[0]
        abcd_layer_norm_backward(ctx, dn, self.x[0][:n], self.w[0]["before_w"], s[0, :n], s[1, :n], dx, g["before_w"],
                                 g["before_b"], d)
