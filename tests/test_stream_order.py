"""Classes that mix the library's calls with torch's operations, on a context whose stream is not the current
one: every operation that reads or writes a tensor is queued on the context's stream.  Without a GPU: the
calls do nothing, the tensors lie in host memory, and the operations say where they would have run."""
import contextlib

import numpy as np
import pytest

from paper_2608_27735_gb300 import Gaussians, appearance, network

torch = pytest.importorskip("torch")
from torch.utils._python_dispatch import TorchDispatchMode  # noqa: E402

# operations that neither read nor write elements
STILL = {"slice", "select", "view", "_unsafe_view", "alias", "detach", "as_strided", "unsqueeze", "expand", "t", "transpose",
         "empty", "empty_like", "new_empty", "empty_strided", "split", "split_with_sizes", "_reshape_alias"}


class FakeContext:
    """A context with a stream of its own."""

    def __init__(self):
        self.depth, self.held = 0, []

    def hold(self, *tensors):
        self.held += tensors

    @contextlib.contextmanager
    def on_stream(self):
        self.depth += 1
        yield
        self.depth -= 1

    def sync(self):
        pass

    def __getattr__(self, name):
        if name.startswith("reserve"):
            return lambda *sizes: None
        raise AttributeError(name)


class Watch(TorchDispatchMode):
    """Collects the operations that ran elsewhere than on the context's stream, and counts those on it."""

    def __init__(self, ctx):
        super().__init__()
        self.ctx, self.astray, self.there = ctx, [], 0

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        name = func._schema.name.split("::")[-1]
        if name not in STILL:
            if self.ctx.depth:
                self.there += 1
            else:
                self.astray.append(name)
        return func(*args, **(kwargs or {}))


@pytest.fixture
def ctx(monkeypatch):
    for module in (network, appearance):
        for name in dir(module):
            if name.startswith("abcd_"):
                monkeypatch.setattr(module, name, lambda *a, **k: None)
    return FakeContext()


def block_weights(cols, ff):
    return {**{k: torch.zeros(cols) for k in ("before_w", "before_b", "after_w", "gate")},
            "w_gate": torch.zeros(ff, cols), "w_up": torch.zeros(ff, cols), "w_down": torch.zeros(cols, ff)}


@pytest.mark.parametrize("packed", [False, True])
def test_stack(ctx, packed):
    stack = network.NormedStack(ctx, [block_weights(8, 16) for _ in range(2)], 5, packed=packed)
    x, y = torch.zeros(4, 8), torch.zeros(4, 8)
    with Watch(ctx) as watch:
        for _ in range(2):
            stack.forward(x, y)
            stack.forward(x, y, train=False)
            stack.backward(x, y)
    assert not watch.astray and watch.there == 2


def bare(cls, **fields):
    """An instance without its constructor, which takes a GPU."""
    self = cls.__new__(cls)
    vars(self).update(fields)
    return self


def test_token_appearance(ctx):
    """And what it returns is held: the library's calls write it on the context's stream."""
    n, width, cols = 4, 8, 12
    new = lambda c: torch.zeros(n, c)
    weights = dict.fromkeys(("w_in", "b_in", "cameras", "cells", "w_out", "b_out"))
    app = bare(appearance.TokenAppearance, ctx=ctx, n=n, width=width, sh_cols=cols, w=weights, g=weights, seen=torch.zeros(n, dtype=torch.int32),
               cell=torch.zeros(n, dtype=torch.int32), tokens=new(width), result=new(width), d=new(width), x=new(cols), d_sh=new(cols),
               stack=network.NormedStack(ctx, [block_weights(width, 16)], n))
    for sh in (torch.zeros(n, 4, 3), torch.zeros(n, 4, 4)[:, :, :3]):      # the second is copied to be a matrix
        with Watch(ctx) as watch:
            out = app.forward(sh, 1), app.forward(sh, 0, train=False), app.backward(sh, 1)
        assert not watch.astray and watch.there >= 6
        assert all(t.shape == sh.shape and any(t.data_ptr() == h.data_ptr() for h in ctx.held) for t in out)


def test_appearance(ctx):
    n, cols = 4, 16
    new = lambda c: torch.zeros(n, c)
    weights = {"norm_w": torch.zeros(cols), "norm_b": torch.zeros(cols), "w_gate": torch.zeros(8, cols), "w_up": torch.zeros(8, cols),
               "w_down": torch.zeros(cols, 8)}
    app = bare(appearance.Appearance, ctx=ctx, n=n, sh_cols=12, cols=cols, embed=new(4), d_embed=new(4), x=[new(cols) for _ in range(2)],
               dx=new(cols), blocks=[network.FeedForwardBlock(ctx, weights, n)])
    sh = torch.zeros(n, 4, 4)[:, :, :3]
    with Watch(ctx) as watch:
        out = app.forward(sh, 1), app.forward(sh, 0, train=False), app.backward(sh, 1)
    assert not watch.astray and watch.there >= 9
    assert all(t.shape == sh.shape and any(t.data_ptr() == h.data_ptr() for h in ctx.held) for t in out)


def test_appearance_stage(ctx):
    class Layers:
        forward = lambda self, sh, ci, train=True: sh
        backward = lambda self, d_sh, ci: d_sh
        step = lambda self: None

    n = 3
    new = lambda: Gaussians(torch.zeros(n, 3), torch.zeros(n, 3), torch.zeros(n, 4), torch.zeros(n), torch.zeros(n, 1, 3), 0)
    stage = bare(appearance.AppearanceStage, ctx=ctx, theta=new(), grads=new(), m=None, v=None, cams=[None], photos=[None], W=8, H=8, proj=None,
                 tiles=None, out=torch.zeros(8, 8, 4), state=None, loss=None, lr=None, appearance=Layers(), rng=np.random.default_rng(1), t=0)
    with Watch(ctx) as watch:
        stage.step()
        stage.eval_loss()
    assert not watch.astray and watch.there >= 3


def test_adam_holds_its_buffers(ctx):
    adam = appearance.Adam(ctx, 20, 1e-3, "cpu")
    assert {t.data_ptr() for t in ctx.held} == {p.means.data_ptr() for p in adam.parts}
