"""Operators of a network over a block's Gaussians (layer norm, gated feed-forward, dropout): the
calls of ``include/abcd.h`` of the same names, and the residual block that they make up.

Matrices are CUDA tensors [rows][cols] whose columns are consecutive (rows may be further apart);
types float32, float16 or bfloat16.  The calls run on the context's stream: tensors that another
stream fills or frees need that stream's events, as everywhere in this package."""
from __future__ import annotations

import struct

from . import ABCD_GELU, ABCD_RELU, ABCD_SILU, Context, _dtypes, _torch, lib

ACTIVATIONS = {"silu": ABCD_SILU, "gelu": ABCD_GELU, "relu": ABCD_RELU}


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
