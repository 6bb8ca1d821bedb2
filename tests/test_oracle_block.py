"""Pins of the block oracle (embedding, layer norm, gated feed-forward): torch autograd in fp64 and central differences."""
import numpy as np
import pytest
import torch

from oracle import psattn_block_oracle as blk

RNG = np.random.default_rng(5)


def _t(x):
    return torch.from_numpy(x).requires_grad_(True)


def _diff(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = f()
        x[i] = keep - h
        g[i] = (up - f()) / (2 * h)
        x[i] = keep
    return g


def test_embed_and_gradient():
    ids = np.array([3, -1, 0, 3, 7, 9, 3])
    W, dX = RNG.standard_normal((8, 5)), RNG.standard_normal((7, 5))
    w = _t(W)
    real = (ids >= 0) & (ids < 8)
    x = torch.where(torch.from_numpy(real)[:, None], w[np.where(real, ids, 0)] * 1.5, 0.0)
    x.backward(torch.from_numpy(dX))
    assert np.allclose(blk.embed(ids, W, 1.5), x.detach().numpy(), atol=1e-14)
    assert np.allclose(blk.embed_grad(ids, dX, 8, 1.5), w.grad.numpy(), atol=1e-13)


@pytest.mark.parametrize("bias", [True, False])
def test_layernorm_and_gradient(bias):
    S, dY, dS = RNG.standard_normal((6, 9)), RNG.standard_normal((6, 9)), RNG.standard_normal((6, 9))
    w, b = RNG.standard_normal(9), RNG.standard_normal(9) if bias else None
    s, tw, tb = _t(S), _t(w), _t(b) if bias else None
    y = torch.nn.functional.layer_norm(s, (9,), tw, tb, 1e-3)
    ((y * torch.from_numpy(dY)).sum() + (s * torch.from_numpy(dS)).sum()).backward()
    dX, dw, db = blk.layernorm_grad(S, w, 1e-3, dY, dS)
    assert np.allclose(blk.layernorm(S, w, b, 1e-3)[0], y.detach().numpy(), atol=1e-13)
    assert np.allclose(dX, s.grad.numpy(), atol=1e-12) and np.allclose(dw, tw.grad.numpy(), atol=1e-12)
    if bias:
        assert np.allclose(db, tb.grad.numpy(), atol=1e-12)
    f = lambda: (blk.layernorm(S, w, b, 1e-3)[0] * dY).sum() + (S * dS).sum()
    assert np.allclose(_diff(f, S), dX, atol=1e-7)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_ffn_and_gradient(kind):
    T, h, n = 4, 5, 6
    X, dY = RNG.standard_normal((T, h)), RNG.standard_normal((T, h))
    Wg, Wu, Wd = RNG.standard_normal((n, h)), RNG.standard_normal((n, h)), RNG.standard_normal((h, n))
    Y, G, U, H = blk.ffn(X, Wg, Wu, Wd, kind)
    got = blk.ffn_grad(X, Wg, Wu, Wd, G, U, H, dY, kind)[:4]
    x, wg, wu, wd = (_t(a) for a in (X, Wg, Wu, Wd))
    fn = torch.nn.functional.silu if kind == "silu" else torch.nn.functional.gelu
    y = (fn(x @ wg.T) * (x @ wu.T)) @ wd.T
    y.backward(torch.from_numpy(dY))
    assert np.allclose(Y, y.detach().numpy(), atol=1e-13)
    for a, t in zip(got, (x, wg, wu, wd)):
        assert np.allclose(a, t.grad.numpy(), atol=1e-12)
    f = lambda: (blk.ffn(X, Wg, Wu, Wd, kind)[0] * dY).sum()
    for a, v in zip(got, (X, Wg, Wu, Wd)):
        assert np.allclose(_diff(f, v), a, atol=1e-7)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_activation_far_out(kind):
    """Closed and open gates: the derivative against differences, and the limits."""
    g = np.array([-800.0, -40.0, -9.0, -1.0, 0.0, 1e-9, 2.0, 40.0, 800.0])
    a, da = blk.act(g, kind)
    assert np.all(np.isfinite(a)) and np.all(np.isfinite(da))
    assert a[0] == 0 and a[-1] == 800 and da[-1] == 1 and da[4] == 0.5
    h = 1e-5
    num = (blk.act(g + h, kind)[0] - blk.act(g - h, kind)[0]) / (2 * h)
    assert np.allclose(num, da, atol=1e-6)
