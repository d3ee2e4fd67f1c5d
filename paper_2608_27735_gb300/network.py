"""Operators of a network over a block's Gaussians (layer norm, gated feed-forward, dropout): the
calls of ``include/abcd.h`` of the same names, and the residual block that they make up.

Matrices are CUDA tensors [rows][cols] whose columns are consecutive (rows may be further apart);
types float32, float16 or bfloat16.  The calls run on the context's stream: tensors that another
stream fills or frees need that stream's events, as everywhere in this package."""
from __future__ import annotations

import ctypes as C

from . import (ABCD_GELU, ABCD_RELU, ABCD_SILU, Context, _dtypes, _torch, abcd_matrix, lib)

ACTIVATIONS = {"silu": ABCD_SILU, "gelu": ABCD_GELU, "relu": ABCD_RELU}


def _matrix(t, what):
    """abcd_matrix of a 2-D CUDA tensor (None for None)."""
    if t is None:
        return None
    if not t.is_cuda or t.dim() != 2:
        raise ValueError(f"{what} must be a 2-D CUDA tensor")
    rows, cols = t.shape
    stride, unit = t.stride()
    if cols > 1 and unit != 1:
        raise ValueError(f"{what} must have consecutive columns")
    dtype = _dtypes().get(t.dtype)
    if dtype is None:
        raise ValueError(f"{what} has type {t.dtype}; float32, float16 and bfloat16 are taken")
    return abcd_matrix(t.data_ptr(), rows, cols, stride if rows > 1 else max(stride, cols), dtype)


def _ref(m):
    return None if m is None else C.byref(m)


def _vector(t, n, what, dtypes):
    """Address of a consecutive CUDA vector of n elements (None for None)."""
    if t is None:
        return None
    if not t.is_cuda or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what} must be a consecutive CUDA vector of {n} elements")
    if t.dtype not in dtypes:
        raise ValueError(f"{what} has type {t.dtype}")
    return t.data_ptr()


def _weight_type(x, *vectors):
    """The torch type of the given weight vectors (x's or float32, one for all)."""
    torch = _torch()
    kinds = {v.dtype for v in vectors if v is not None} or {x.dtype}
    if len(kinds) > 1 or not kinds <= {x.dtype, torch.float32}:
        raise ValueError("weights are all of the matrices' type or all float32")
    return kinds.pop()


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"unknown activation {name!r}; one of {sorted(ACTIVATIONS)}")
    return ACTIVATIONS[name]


def abcd_layer_norm(ctx: Context, x, weight, bias, eps, y, mean=None, rstd=None):
    """y = layer norm of x's rows; weight, bias: [cols] or None; mean, rstd: float32 [rows] that the
    backward pass needs, or None."""
    mx, my = _matrix(x, "x"), _matrix(y, "y")
    wt = _weight_type(x, weight, bias)
    f32 = (_torch().float32,)
    ctx.check(lib().abcd_layer_norm(
        ctx.h, C.byref(mx), _vector(weight, mx.cols, "weight", (wt,)),
        _vector(bias, mx.cols, "bias", (wt,)), _dtypes()[wt], float(eps), C.byref(my),
        _vector(mean, mx.rows, "mean", f32), _vector(rstd, mx.rows, "rstd", f32)))


def abcd_layer_norm_backward(ctx: Context, dy, x, weight, mean, rstd, dx=None, dweight=None,
                             dbias=None, d_residual=None):
    """dx, dweight and dbias (each may be None) of abcd_layer_norm; d_residual is added to dx (which
    may be dy or d_residual).  Takes the network workspace (Context.reserve_network)."""
    md, mx, mg = _matrix(dy, "dy"), _matrix(x, "x"), _matrix(dx, "dx")
    mr = _matrix(d_residual, "d_residual")
    wt = _weight_type(x, weight, dweight, dbias)
    f32 = (_torch().float32,)
    ctx.check(lib().abcd_layer_norm_backward(
        ctx.h, C.byref(md), C.byref(mx), _vector(weight, mx.cols, "weight", (wt,)), _dtypes()[wt],
        _vector(mean, mx.rows, "mean", f32), _vector(rstd, mx.rows, "rstd", f32), _ref(mr), _ref(mg),
        _vector(dweight, mx.cols, "dweight", (wt,)), _vector(dbias, mx.cols, "dbias", (wt,))))


def abcd_gated_ff(ctx: Context, x, w_gate, w_up, w_down, activation, y, gate=None, up=None):
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T; gate, up: [rows][ff] that the backward pass
    needs, or None; activation: "silu", "gelu" or "relu".  Takes the network workspace."""
    ms = [_matrix(t, n) for t, n in ((x, "x"), (w_gate, "w_gate"), (w_up, "w_up"),
                                     (w_down, "w_down"), (y, "y"), (gate, "gate"), (up, "up"))]
    r = [_ref(m) for m in ms]
    ctx.check(lib().abcd_gated_ff(ctx.h, *r[:4], _activation(activation), *r[4:]))


def abcd_gated_ff_backward(ctx: Context, dy, x, w_gate, w_up, w_down, activation, gate, up,
                           dx=None, dw_gate=None, dw_up=None, dw_down=None):
    """dx and the weights' gradients (each may be None) of abcd_gated_ff, from what its forward call
    left in gate and up.  Takes the network workspace."""
    ms = [_matrix(t, n) for t, n in ((dy, "dy"), (x, "x"), (w_gate, "w_gate"), (w_up, "w_up"),
                                     (w_down, "w_down"), (gate, "gate"), (up, "up"), (dx, "dx"),
                                     (dw_gate, "dw_gate"), (dw_up, "dw_up"),
                                     (dw_down, "dw_down"))]
    r = [_ref(m) for m in ms]
    ctx.check(lib().abcd_gated_ff_backward(ctx.h, *r[:5], _activation(activation), *r[5:]))


def abcd_dropout(ctx: Context, x, p, seed, offset, y, residual=None):
    """y = residual + dropout(x) with the mask of (seed, offset); y may be x or residual.  The next
    call's offset is past this one's: offset + ceil(rows * cols / 8)."""
    mx, my, mr = _matrix(x, "x"), _matrix(y, "y"), _matrix(residual, "residual")
    ctx.check(lib().abcd_dropout(ctx.h, C.byref(mx), float(p), int(seed), int(offset), _ref(mr),
                                 C.byref(my)))


def abcd_dropout_backward(ctx: Context, dy, p, seed, offset, dx):
    """dx = dropout's gradient of dy under the mask of (seed, offset); dx may be dy."""
    md, mx = _matrix(dy, "dy"), _matrix(dx, "dx")
    ctx.check(lib().abcd_dropout_backward(ctx.h, C.byref(md), float(p), int(seed), int(offset),
                                          C.byref(mx)))


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
        ctx.reserve_network(self.rows, self.cols, self.ff, dt)

    def _counters(self, rows):
        return (rows * self.cols + 7) // 8

    def forward(self, x, y, train=True):
        """y = the block of x (both [rows'][cols], rows' <= rows; y may be x).  train: keep what the
        backward pass needs, and drop with the next counters of the block's generator."""
        n, w = x.shape[0], self.w
        nx, out = self.normed[:n], self.out[:n]
        if not train:
            abcd_layer_norm(self.ctx, x, w["norm_w"], w["norm_b"], self.eps, nx)
            abcd_gated_ff(self.ctx, nx, w["w_gate"], w["w_up"], w["w_down"], self.act, out)
            abcd_dropout(self.ctx, out, 0.0, self.seed, 0, y, x)
            return
        self.drawn = self.offset
        self.offset += self._counters(n)
        abcd_layer_norm(self.ctx, x, w["norm_w"], w["norm_b"], self.eps, nx, self.mean[:n],
                        self.rstd[:n])
        abcd_gated_ff(self.ctx, nx, w["w_gate"], w["w_up"], w["w_down"], self.act, out,
                      self.gate[:n], self.up[:n])
        abcd_dropout(self.ctx, out, self.p, self.seed, self.drawn, y, x)

    def backward(self, dy, x, dx):
        """dx (may be dy) and `grads` of the last forward(x, ..., train=True); x as it was given."""
        n, w, g = x.shape[0], self.w, self.grads
        d_out, d_nx = self.d_out[:n], self.d_normed[:n]
        abcd_dropout_backward(self.ctx, dy, self.p, self.seed, self.drawn, d_out)
        abcd_gated_ff_backward(self.ctx, d_out, self.normed[:n], w["w_gate"], w["w_up"],
                               w["w_down"], self.act, self.gate[:n], self.up[:n], d_nx,
                               g["w_gate"], g["w_up"], g["w_down"])
        abcd_layer_norm_backward(self.ctx, d_nx, x, w["norm_w"], self.mean[:n], self.rstd[:n], dx,
                                 g["norm_w"], g["norm_b"], dy)
