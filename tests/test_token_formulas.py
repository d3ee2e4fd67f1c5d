"""The 64-bit formulas of tests/_tokens.py against differences and against their own definitions."""
import numpy as np
import pytest

from . import _tokens as K


def differences(value, at, step=1e-6):
    """The gradient of value() by central differences over the array `at`, in place."""
    g = np.zeros_like(at)
    for i in np.ndindex(at.shape):
        keep = at[i]
        at[i] = keep + step
        up = value()
        at[i] = keep - step
        g[i] = (up - value()) / (2 * step)
        at[i] = keep
    return g


def test_embedding_gradient():
    r = np.random.default_rng(1)
    table, dy = r.normal(size=(5, 3)), r.normal(size=(9, 3))
    index = np.array([0, 4, -1, 2, 2, 7, 0, 2, -5])
    value = lambda: (K.embed(table, index, 0.7, dy) * dy).sum()
    assert np.allclose(K.embed_grad(dy, index, 0.7, 5), differences(value, table), atol=1e-8)
    assert (K.embed(table, index, 0.7, None)[[2, 5, 8]] == 0).all()


@pytest.mark.parametrize("name", ["none", "silu", "gelu", "relu"])
def test_linear_gradients(name):
    r = np.random.default_rng(2)
    x, w, b = r.normal(size=(4, 5)), r.normal(size=(3, 5)), r.normal(size=3)
    dy, res = r.normal(size=(4, 3)), r.normal(size=(4, 3))
    z = K.linear(x, w, b, name, res)[1]
    value = lambda: (K.linear(x, w, b, name, res)[0] * dy).sum()
    for got, at in zip(K.linear_grad(dy, x, w, name, z), (x, w, b)):
        assert np.allclose(got, differences(value, at), atol=1e-7)


@pytest.mark.parametrize("after", [None, "layer", "rms"])
@pytest.mark.parametrize("before", [None, "layer", "rms"])
def test_residual_norm_gradients(after, before):
    r = np.random.default_rng(3)
    x, f, dy, dn = (r.normal(size=(3, 6)) for _ in range(4))
    v = {k: r.normal(1, 0.3, 6) for k in ("gate", "w1", "b1", "w2", "b2")}

    def layer():
        return K.Close(6, after and (after, v["w1"], v["b1"]), before and (before, v["w2"], v["b2"]), v["gate"], 0.7)

    def value():
        y, n, _ = layer().forward(x, f)
        return (y * dy).sum() + (0 if n is None else (n * dn).sum())

    s = layer().forward(x, f)[2]
    got = layer().backward(dy, dn if before else None, x, f, s)
    for g, at in zip(got, (x, f, v["gate"], v["w1"], v["b1"], v["w2"], v["b2"])):
        if (at is v["w1"] or at is v["b1"]) and not after or (at is v["w2"] or at is v["b2"]) and not before:
            continue
        assert np.allclose(g, differences(value, at), atol=1e-7)


def test_packed_values():
    """Within a 128th of a group's largest magnitude, exact where that is a power of two's multiple; groups
    that are not finite, zero, tiny."""
    r = np.random.default_rng(4)
    x = r.normal(size=(50, 70)) * np.exp(4 * r.normal(size=(50, 1)))
    x[3], x[4, 40], x[5, 2] = 0.0, np.inf, np.nan
    x[6] = 2.0 ** -140
    x[7, :32] = np.arange(32) * 4.0
    codes, powers = K.packed(x)
    y = K.unpacked(codes, powers)
    bad = np.zeros((50, 3), bool)
    bad[4, 1] = bad[5, 0] = True
    assert (np.isnan(y) == np.repeat(bad, 32, 1)[:, :70]).all() and (codes[4, 32:64] == 0).all()
    for g in range(3):
        at = slice(32 * g, min(70, 32 * g + 32))
        keep = ~bad[:, g]
        top = np.abs(x[keep, at]).max(1, keepdims=True)
        assert (np.abs(y[keep, at] - x[keep, at]) <= top / 128 + 2.0 ** -127).all()
    assert (y[7, :32] == x[7, :32]).all() and (y[3] == 0).all() and (powers[3] == 1).all()
    assert np.abs(codes).max() <= 127
    # again: what was packed stays
    keep = ~np.isnan(y).any(1)
    assert (K.unpacked(*K.packed(y[keep])) == y[keep]).all()


