"""A learned appearance of a block: SH coefficients that depend on the camera.

Photographs of one scene differ in exposure and white balance, which no single colour per Gaussian
can fit.  Here one token per Gaussian (its SH coefficients next to a learned embedding of the
camera) goes through residual layers x + dropout(gated_ff(layer_norm(x))), whose first columns are
the coefficients that the camera sees.  They are rendered by the calls of a training step, and the
gradient that abcd_backward leaves for the coefficients goes back through the layers.  Everything is
in 32 bits; all weights lie in one buffer, which abcd_adam_active updates.

``TokenAppearance`` is the same with tokens of any width: a linear layer makes them from the
coefficients, a row for the camera and one for the cell of the block that the Gaussian lies in are looked
up and added, blocks with norms before and after follow, and a linear layer adds to the coefficients what
comes out.  What the blocks keep for the backward pass may be held in 8 bits.

``appearance_experiment()`` runs them on a small seeded scene: the same block is fitted to photographs
with and without the layers, and with tokens."""
from __future__ import annotations

import numpy as np

from . import (ABCD_F32, Context, FeedForwardBlock, FwdState, Gaussians, NormedStack, Projected, Tiles,
               _torch, abcd_adam_active, abcd_assign_cells, abcd_backward, abcd_bin_sort, abcd_embedding,
               abcd_embedding_backward, abcd_linear, abcd_linear_backward, abcd_loss, abcd_project,
               abcd_render_composite_fwd, camera)


class Adam:
    """abcd_adam_active over one float32 buffer of any length with one learning rate: the call's five
    parameter arrays (3, 3, 4, 1 and 3 values per Gaussian) are consecutive parts of the buffer,
    whose length is rounded up to whole Gaussians of 14 values."""

    def __init__(self, ctx: Context, length, lr, device="cuda"):
        torch = _torch()
        self.ctx, self.lr, self.step_no = ctx, float(lr), 0
        n = (int(length) + 13) // 14
        self.values, self.grads = (torch.zeros(14 * n, device=device) for _ in range(2))
        m, v = (torch.zeros(14 * n, device=device) for _ in range(2))
        ctx.hold(self.values, self.grads, m, v)
        self.parts = [self._parts(t, n) for t in (self.values, self.grads, m, v)]

    @staticmethod
    def _parts(t, n):
        a, b, c, d, e = t.split([3 * n, 3 * n, 4 * n, n, 3 * n])
        return Gaussians(a.view(n, 3), b.view(n, 3), c.view(n, 4), d, e.view(n, 1, 3), 0)

    def step(self):
        self.step_no += 1
        p, g, m, v = self.parts
        abcd_adam_active(self.ctx, p, g, m, v, [self.lr] * 6, 0.9, 0.999, 1e-8, self.step_no)


class Appearance:
    """The layers and the cameras' embeddings for a block of n Gaussians.

    layers: residual blocks; embed: width of a camera's embedding; widen: hidden width over token
    width; p: dropout.  The last product of every block starts at zero, so the layers start as the
    identity: at first every camera sees the block's own coefficients."""

    def __init__(self, ctx: Context, n, sh_degree, n_cameras, layers=2, embed=16, widen=4, p=0.0,
                 lr=2e-3, seed=0):
        torch = _torch()
        self.ctx, self.n = ctx, int(n)
        self.sh_cols = 3 * (sh_degree + 1) ** 2
        self.cols = self.sh_cols + int(embed)
        ff = int(widen) * self.cols
        shapes = {"norm_w": (self.cols,), "norm_b": (self.cols,), "w_gate": (ff, self.cols),
                  "w_up": (ff, self.cols), "w_down": (self.cols, ff)}
        per_layer = sum(int(np.prod(s)) for s in shapes.values())
        self.adam = Adam(ctx, layers * per_layer + n_cameras * embed, lr)
        rng = np.random.default_rng(seed)
        self.blocks, at = [], 0
        for k in range(layers):
            w, g = {}, {}
            for name, shape in shapes.items():
                size = int(np.prod(shape))
                w[name] = self.adam.values[at:at + size].view(shape)
                g[name] = self.adam.grads[at:at + size].view(shape)
                at += size
            w["norm_w"].fill_(1.0)
            for name in ("w_gate", "w_up"):
                w[name].copy_(torch.from_numpy(rng.normal(0, self.cols ** -0.5, shapes[name]).astype(np.float32)))
            block = FeedForwardBlock(ctx, w, n, "silu", p=p, seed=seed * 1000 + k)
            block.grads = g                      # the block's gradients land in Adam's buffer
            self.blocks.append(block)
        size = n_cameras * embed
        self.embed = self.adam.values[at:at + size].view(n_cameras, embed)
        self.d_embed = self.adam.grads[at:at + size].view(n_cameras, embed)
        self.embed.copy_(torch.from_numpy(rng.normal(0, 1, (n_cameras, embed)).astype(np.float32)))
        self.x = [torch.empty(n, self.cols, device="cuda") for _ in range(layers + 1)]
        self.dx = torch.empty(n, self.cols, device="cuda")
        ctx.hold(*self.x, self.dx)

    def forward(self, sh, ci, train=True):
        """The coefficients that camera ci sees of sh [n][D][3]: a new tensor of that shape."""
        # without training in place, in the backward pass's buffer: what the last training pass kept stays
        x = self.x if train else [self.dx] * len(self.x)
        out = _torch().empty(self.n, self.sh_cols, device=self.dx.device)
        self.ctx.hold(out)
        with self.ctx.on_stream():
            x[0][:, :self.sh_cols] = sh.reshape(self.n, self.sh_cols)
            x[0][:, self.sh_cols:] = self.embed[ci]
            for k, block in enumerate(self.blocks):
                block.forward(x[k], x[k + 1], train)
            out.copy_(x[-1][:, :self.sh_cols])
        return out.view(sh.shape)

    def backward(self, d_sh, ci):
        """The gradient of sh from that of the last training forward(sh, ci)'s result; leaves the
        weights' and the embeddings' gradients in Adam's buffer."""
        out = _torch().empty(self.n, self.sh_cols, device=self.dx.device)
        self.ctx.hold(out)
        with self.ctx.on_stream():
            self.dx[:, :self.sh_cols] = d_sh.reshape(self.n, self.sh_cols)
            self.dx[:, self.sh_cols:] = 0.0
            for k in reversed(range(len(self.blocks))):
                self.blocks[k].backward(self.dx, self.x[k], self.dx)
            self.d_embed.zero_()
            self.d_embed[ci] = self.dx[:, self.sh_cols:].sum(0)
            out.copy_(self.dx[:, :self.sh_cols])
        return out.view(d_sh.shape)

    def step(self):
        self.adam.step()


class TokenAppearance:
    """As Appearance, with tokens of width `width` for a block of Gaussians with the given means (numpy
    [n][3]): a grid of `cells` cells per axis over the means' box gives each Gaussian the row of a learned
    table.  packed: NormedStack's.  The layer behind the blocks starts at zero, so every camera first sees
    the block's own coefficients."""

    def __init__(self, ctx: Context, means, sh_degree, n_cameras, layers=2, width=64, widen=4, cells=4,
                 packed=False, lr=2e-3, seed=0):
        torch = _torch()
        self.ctx, self.n, self.width = ctx, len(means), int(width)
        self.sh_cols = 3 * (sh_degree + 1) ** 2
        ff = int(widen) * self.width
        low, high = means.min(0), means.max(0)
        side = float(max(high - low)) / cells * (1 + 1e-6) or 1.0
        cell = abcd_assign_cells(means, low.astype(np.float64), side, (cells,) * 3)
        shapes = {"w_in": (self.width, self.sh_cols), "b_in": (self.width,), "cameras": (n_cameras, self.width),
                  "cells": (cells ** 3, self.width), "w_out": (self.sh_cols, self.width), "b_out": (self.sh_cols,)}
        block = {"before_w": (self.width,), "before_b": (self.width,), "after_w": (self.width,), "gate": (self.width,),
                 "w_gate": (ff, self.width), "w_up": (ff, self.width), "w_down": (self.width, ff)}
        size = lambda shape: (int(np.prod(shape)) + 3) // 4 * 4       # each on a 16-byte boundary
        self.adam = Adam(ctx, sum(map(size, shapes.values())) + layers * sum(map(size, block.values())), lr)
        rng = np.random.default_rng(seed)
        at = 0

        def take(shapes, start):
            nonlocal at
            w, g = {}, {}
            for name, shape in shapes.items():
                n = int(np.prod(shape))
                w[name], g[name] = (t[at:at + n].view(shape) for t in (self.adam.values, self.adam.grads))
                at += size(shape)
                w[name].copy_(torch.from_numpy(np.broadcast_to(start(name, shape), shape).astype(np.float32)))
            return w, g

        def start(name, shape):
            if name in ("w_out", "b_in", "b_out", "before_b"):
                return 0.0
            if name in ("before_w", "after_w"):
                return 1.0
            if name == "gate":
                return 0.5
            return rng.normal(0, 0.1 if name in ("cameras", "cells") else shape[1] ** -0.5, shape)

        self.w, self.g = take(shapes, start)
        blocks = [take(block, start) for _ in range(layers)]
        self.stack = NormedStack(ctx, [w for w, _ in blocks], self.n, "silu", packed=packed)
        self.stack.grads = [g for _, g in blocks]
        self.cell = torch.from_numpy(cell.astype(np.int32)).cuda()
        self.seen = torch.empty(self.n, dtype=torch.int32, device="cuda")          # the camera, for each token
        new = lambda c: torch.empty(self.n, c, device="cuda")
        self.tokens, self.result, self.d = new(self.width), new(self.width), new(self.width)
        self.x, self.d_sh = new(self.sh_cols), new(self.sh_cols)
        ctx.hold(self.cell, self.seen, self.tokens, self.result, self.d, self.x, self.d_sh)
        for a, b in ((self.sh_cols, self.width), (self.width, self.sh_cols)):
            ctx.reserve_linear(self.n, a, b)
        ctx.reserve_embedding(self.n, max(n_cameras, cells ** 3), self.width)

    def forward(self, sh, ci, train=True):
        """The coefficients that camera ci sees of sh [n][D][3]: a new tensor of that shape."""
        w, ctx = self.w, self.ctx
        tokens = self.tokens if train else self.d
        result = self.result if train else self.d
        out = _torch().empty_like(self.x)
        ctx.hold(out)
        with ctx.on_stream():                           # (what reshape copies, too)
            x = sh.reshape(self.n, self.sh_cols)
            if train:
                self.x.copy_(x)
            self.seen.fill_(ci)
            abcd_linear(ctx, x, w["w_in"], w["b_in"], "none", tokens)
            abcd_embedding(ctx, w["cameras"], self.seen, 1.0, tokens, tokens)
            abcd_embedding(ctx, w["cells"], self.cell, 1.0, tokens, tokens)
            self.stack.forward(tokens, result, train)
            abcd_linear(ctx, result, w["w_out"], w["b_out"], "none", out, x)
        return out.view(sh.shape)

    def backward(self, d_sh, ci):
        """The gradient of sh from that of the last training forward(sh, ci)'s result; leaves the weights'
        gradients in Adam's buffer."""
        w, g, ctx = self.w, self.g, self.ctx
        out = _torch().empty_like(self.x)
        ctx.hold(out)
        with ctx.on_stream():
            d = d_sh.reshape(self.n, self.sh_cols)
            abcd_linear_backward(ctx, d, self.result, w["w_out"], "none", None, self.d, g["w_out"], g["b_out"])
            self.stack.backward(self.d, self.d)
            self.seen.fill_(ci)
            abcd_embedding_backward(ctx, self.d, self.seen, 1.0, g["cameras"])
            abcd_embedding_backward(ctx, self.d, self.cell, 1.0, g["cells"])
            abcd_linear_backward(ctx, self.d, self.x, w["w_in"], "none", None, self.d_sh, g["w_in"], g["b_in"])
            _torch().add(self.d_sh, d, out=out)
        return out.view(d_sh.shape)

    def step(self):
        self.adam.step()


class AppearanceStage:
    """Fits a block's SH coefficients, and with `appearance` the layers (True: Appearance, "tokens":
    TokenAppearance), to photographs.

    gaussians: scenegen.Gaussians; cameras: objects as camera() takes; photos: float32
    [C][H][W][3]."""

    def __init__(self, gaussians, cameras, photos, appearance=True, lr_sh=2.5e-3, seed=0, device=0,
                 max_pairs=1_000_000, **layers):
        torch = _torch()
        self.ctx = Context(device)
        self.theta = Gaussians.from_numpy(gaussians)
        n, W, H = self.theta.n, int(cameras[0].width), int(cameras[0].height)
        self.W, self.H = W, H
        self.cams = [camera(c) for c in cameras]
        self.photos = torch.from_numpy(np.ascontiguousarray(photos, np.float32)).cuda()
        self.ctx.reserve(n, max_pairs, W * H)
        self.proj, self.tiles = Projected.alloc(n), Tiles.alloc(max_pairs, W, H)
        self.out = torch.empty(H, W, 4, device="cuda")
        self.state = FwdState.alloc(W, H)
        self.grads, self.m, self.v = (Gaussians.zeros_like(self.theta) for _ in range(3))
        self.loss = torch.zeros(1, device="cuda")
        self.lr = [0.0, 0.0, 0.0, 0.0, lr_sh, lr_sh / 20]         # the shapes stay
        if appearance == "tokens":
            self.appearance = TokenAppearance(self.ctx, np.ascontiguousarray(gaussians.means, np.float32),
                                              gaussians.sh_degree, len(self.cams), seed=seed, **layers)
        else:
            self.appearance = Appearance(self.ctx, n, gaussians.sh_degree, len(self.cams), seed=seed,
                                         **layers) if appearance else None
        self.rng = np.random.default_rng(seed)
        self.t = 0

    def render(self, ci, train=False):
        """Camera ci's render (into self.out) and the Gaussians it shows."""
        seen = self.theta
        if self.appearance is not None:
            sh = self.appearance.forward(self.theta.sh, ci, train)
            seen = Gaussians(*self.theta.tensors()[:4], sh, self.theta.sh_degree)
        cam = self.cams[ci]
        abcd_project(self.ctx, seen, cam, None, self.proj)
        abcd_bin_sort(self.ctx, self.proj, seen.n, cam, self.tiles)
        abcd_render_composite_fwd(self.ctx, cam, None, self.proj, self.tiles, None, None, ABCD_F32,
                                  None, self.out, self.state)
        return seen

    def step(self):
        """One step on the next camera of a shuffled round."""
        if self.t % len(self.cams) == 0:
            self.order = self.rng.permutation(len(self.cams))
        ci = int(self.order[self.t % len(self.cams)])
        self.t += 1
        seen = self.render(ci, train=True)
        abcd_backward(self.ctx, seen, self.cams[ci], None, self.proj, self.tiles, None, None,
                      ABCD_F32, None, self.out, self.state, self.photos[ci], 0.2, self.loss, None,
                      self.grads)
        if self.appearance is not None:
            d_sh = self.appearance.backward(self.grads.sh, ci)
            with self.ctx.on_stream():
                self.grads.sh.copy_(d_sh)
            self.appearance.step()
        abcd_adam_active(self.ctx, self.theta, self.grads, self.m, self.v, self.lr, 0.9, 0.999,
                         1e-15, self.t)

    def eval_loss(self):
        """Mean loss over the photographs, without dropout."""
        with self.ctx.on_stream():
            acc = _torch().zeros(len(self.cams), device=self.out.device)
            for ci in range(len(self.cams)):
                self.render(ci)
                abcd_loss(self.ctx, self.out, self.photos[ci], self.W, self.H, 0.2, acc[ci:ci + 1], None)
            self.ctx.sync()
            return float(acc.mean().item())


def appearance_experiment(T=400, n=1500, n_cams=6, size=96, p=0.05, seed=7):
    """A block seen by cameras of different exposure and white balance (each scales the true colours
    by a gain per channel), fitted for T steps without layers, with them and with tokens, from the same
    SH coefficients.  Returns {name: (loss before, loss after)}."""
    from . import scenegen as sg
    s = sg.grid_scene((1, 1, 1), 5.0, n, 1, seed=seed)
    cams = sg.ring_cameras(n_cams, 1.5 * sg.half_diagonal(s.grid), np.zeros(3), size, size, seed=seed,
                           height_jitter=1.0)
    blank = np.zeros((n_cams, size, size, 3), np.float32)
    truth = AppearanceStage(s.gaussians, cams, blank, appearance=False)
    gains = np.random.default_rng(seed + 1).uniform(0.4, 1.0, (n_cams, 3)).astype(np.float32)
    photos = []
    for ci in range(n_cams):
        truth.render(ci)
        photos.append(truth.out[..., :3].cpu().numpy() * gains[ci])
    out = {}
    for name, layers, more in (("one_colour", False, {}), ("appearance", True, {"p": p}),
                               ("tokens", "tokens", {"packed": True})):
        run = AppearanceStage(s.gaussians, cams, np.stack(photos), appearance=layers, seed=seed, **more)
        before = run.eval_loss()
        for _ in range(T):
            run.step()
        out[name] = (before, run.eval_loss())
    return out


if __name__ == "__main__":
    for name, (before, after) in appearance_experiment().items():
        print(f"{name}: loss {before:.5f} -> {after:.5f}")
