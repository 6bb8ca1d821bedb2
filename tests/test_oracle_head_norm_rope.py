"""Pins of the oracle of the vocabulary head, the gated norms and rotary positions of any layout (CPU): torch's own functions with
autograd, differences, and properties of the definitions."""
import numpy as np
import pytest
import torch

from oracle import psattn_block_oracle as blk
from oracle import psattn_oracle as orc


def _t(x):
    return None if x is None else torch.tensor(x, dtype=torch.float64, requires_grad=True)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", [None, "row", "all"])
def test_gatednorm_against_autograd(post, gate):
    rng = np.random.default_rng(5)
    n, h, eps, res = 7, 12, 0.01, 0.75
    X, B, dY, dS = (rng.standard_normal((n, h)) for _ in range(4))
    w_pre, w_post = rng.standard_normal(h), rng.standard_normal(h) if post else None
    g = None if gate is None else rng.standard_normal(h if gate == "row" else (n, h))
    tX, tB, tp, tw, tg = (_t(x) for x in (X, B, w_pre, w_post, g))
    N = torch.nn.functional.rms_norm(tB, (h,), tw, eps) if post else tB
    S = res * tX + (N if g is None else tg * N)
    Y = torch.nn.functional.rms_norm(S, (h,), tp, eps)
    got = blk.gatednorm(X, B, w_pre, w_post, g, res, eps)
    assert np.allclose(got[0], Y.detach().numpy()) and np.allclose(got[1], S.detach().numpy())
    ((Y * torch.tensor(dY)).sum() + (S * torch.tensor(dS)).sum()).backward()
    grads = blk.gatednorm_grad(B, got[1], w_pre, w_post, g, res, eps, dY, dS)
    for a, t in zip(grads, (tX, tB, tp, tw, tg)):
        assert (a is None) == (t is None)
        if a is not None:
            assert np.allclose(a, t.grad.numpy())


def test_gatednorm_without_a_block_is_a_norm():
    rng = np.random.default_rng(6)
    X, dY, w = rng.standard_normal((5, 9)), rng.standard_normal((5, 9)), rng.standard_normal(9)
    tX, tw = _t(X), _t(w)
    Y = torch.nn.functional.rms_norm(tX, (9,), tw, 1e-3)
    got = blk.gatednorm(X, None, w, None, None, 3.0, 1e-3)
    assert np.allclose(got[0], Y.detach().numpy()) and got[1] is X
    (Y * torch.tensor(dY)).sum().backward()
    dX, dB, dw, _, _ = blk.gatednorm_grad(None, X, w, None, None, 3.0, 1e-3, dY)
    assert np.allclose(dX, tX.grad.numpy()) and np.allclose(dw, tw.grad.numpy()) and dB is None


def test_gatednorm_differences():
    rng = np.random.default_rng(7)
    n, h, eps = 3, 5, 0.05
    a = {k: rng.standard_normal(s) for k, s in dict(X=(n, h), B=(n, h), w_pre=h, w_post=h, gate=h).items()}
    dY, dS = rng.standard_normal((n, h)), rng.standard_normal((n, h))

    def loss(**x):
        Y, S, _, _ = blk.gatednorm(x["X"], x["B"], x["w_pre"], x["w_post"], x["gate"], 0.5, eps)
        return (Y * dY).sum() + (S * dS).sum()

    S = blk.gatednorm(a["X"], a["B"], a["w_pre"], a["w_post"], a["gate"], 0.5, eps)[1]
    grads = dict(zip(("X", "B", "w_pre", "w_post", "gate"), blk.gatednorm_grad(a["B"], S, a["w_pre"], a["w_post"], a["gate"], 0.5, eps, dY, dS)))
    for k, g in grads.items():
        step = rng.standard_normal(a[k].shape)
        up, down = dict(a), dict(a)
        up[k], down[k] = a[k] + 1e-5 * step, a[k] - 1e-5 * step
        assert abs((loss(**up) - loss(**down)) / 2e-5 - (g * step).sum()) <= 1e-7 * max(1.0, abs((g * step).sum())), k


def test_rotary_is_the_library_s_rotation_where_both_apply():
    rng = np.random.default_rng(8)
    x, pos = rng.standard_normal((6, 3, 16)), np.array([0, 1, 2, 7, 100, 3])
    f = blk.rotary_frequencies(16, 10000.0)
    assert np.allclose(blk.rotary(x, pos, f), orc.rope_rotate(x, pos, 10000.0))
    assert np.allclose(blk.rotary(x, pos, f, transposed=True), orc.rope_rotate(x, pos, 10000.0, inverse=True))


def test_rotary_interleaved_is_complex_multiplication():
    rng = np.random.default_rng(9)
    x, pos = rng.standard_normal((5, 2, 12)), np.array([4, 0, 9, 2, 1])
    f = blk.rotary_frequencies(8, 500.0)
    z = (x[..., 0:8:2] + 1j * x[..., 1:8:2]) * (1.5 * np.exp(1j * pos[:, None, None] * f))
    y = blk.rotary(x, pos, f, interleaved=True, amplitude=1.5)
    assert np.allclose(y[..., 0:8:2], z.real) and np.allclose(y[..., 1:8:2], z.imag) and np.array_equal(y[..., 8:], x[..., 8:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_properties(interleaved):
    rng = np.random.default_rng(10)
    q, k = rng.standard_normal((1, 1, 10)), rng.standard_normal((1, 1, 10))
    f = blk.rotary_frequencies(6, 100.0)
    score = lambda a, b: (blk.rotary(q, [a], f, interleaved) * blk.rotary(k, [b], f, interleaved)).sum()
    assert abs(score(3, 1) - score(40, 38)) < 1e-12  # relative positions alone
    x, g, pos = rng.standard_normal((4, 2, 10)), rng.standard_normal((4, 2, 10)), [5, 6, 7, 30]
    # <rotary(x), g> = <x, transposed(g)>; rows of unknown positions give and get nothing
    a = (blk.rotary(x, pos, f, interleaved, 0.7, n_positions=20) * g).sum()
    assert abs(a - (x * blk.rotary(g, pos, f, interleaved, 0.7, transposed=True, n_positions=20)).sum()) < 1e-12
    assert np.all(blk.rotary(x, pos, f, interleaved, n_positions=20)[3] == 0)


def test_frequencies():
    n, theta, s, L = 32, 10000.0, 4.0, 2048
    f = blk.rotary_frequencies(n, theta)
    assert f[0] == 1 and np.allclose(f[1:] / f[:-1], theta ** (-2 / n))
    assert np.allclose(blk.rotary_frequencies(n, theta, "linear", s), f / s)
    b = blk.rotary_frequencies(n, theta, "base", s)
    assert np.isclose(b[0], f[0]) and np.isclose(b[-1], f[-1] / s) and np.all(np.diff(b / f) < 0)
    p = blk.rotary_frequencies(n, theta, "parts", s, L, 1.0, 32.0)
    turns = f * L / (2 * np.pi)
    assert np.array_equal(p[turns >= 32], f[turns >= 32]) and np.allclose(p[turns <= 1], f[turns <= 1] / s)
    mid = (turns > 1) & (turns < 32)
    assert mid.sum() > 3 and np.all(p[mid] < f[mid]) and np.all(p[mid] > f[mid] / s)


def _samples():
    return [2, 30], [3, 4], [0, 2, 5], [4, 6, 1, 0, 5], 45


def test_head_against_the_head_on_logits_and_autograd():
    rng = np.random.default_rng(11)
    off, P, ptr, rl, T = _samples()
    V, h = 11, 6
    X, W, ids, d = rng.standard_normal((T, h)), rng.standard_normal((V, h)), rng.integers(0, V, T), rng.standard_normal(len(rl))
    items = orc.prediction_items(off, P, ptr, rl)
    lse, logp = blk.head(X, W, ids, items)
    per = np.zeros(len(rl))
    np.add.at(per, [j for j, _, _ in items], logp)
    assert np.allclose(per, orc.response_logprobs(X @ W.T, ids, off, P, ptr, rl))
    dX, dW, G = blk.head_grad(X, W, ids, items, d)
    assert np.allclose(G, orc.response_logprobs_grad(X @ W.T, ids, off, P, ptr, rl, d))
    tX, tW = _t(X), _t(W)
    lp = torch.log_softmax(tX @ tW.T, 1)
    sum(d[j] * lp[r, ids[t]] for j, r, t in items).backward()
    assert np.allclose(dX, tX.grad.numpy()) and np.allclose(dW, tW.grad.numpy())
    assert np.allclose(lse, torch.logsumexp(tX @ tW.T, 1).detach().numpy())


def test_head_ignores_ids_outside_the_vocabulary():
    rng = np.random.default_rng(12)
    off, P, ptr, rl, T = _samples()
    X, W = rng.standard_normal((T, 4)), rng.standard_normal((7, 4))
    ids = rng.integers(0, 7, T)
    items = orc.prediction_items(off, P, ptr, rl)
    gone = {items[2][2], items[7][2]}
    kept = [x for x in items if x[2] not in gone]
    d = rng.standard_normal(len(rl))
    bad = ids.copy()
    bad[list(gone)] = [-1, 7]
    assert np.allclose(blk.head_grad(X, W, bad, items, d)[0], blk.head_grad(X, W, ids, kept, d)[0])
    assert np.count_nonzero(blk.head(X, W, bad, items)[1] == 0) == 2


def test_head_differences():
    rng = np.random.default_rng(13)
    off, P, ptr, rl, T = _samples()
    X, W, ids, d = rng.standard_normal((T, 5)), rng.standard_normal((9, 5)), rng.integers(0, 9, T), rng.standard_normal(len(rl))
    items = orc.prediction_items(off, P, ptr, rl)
    loss = lambda x, w: sum(d[j] * l for (j, _, _), l in zip(items, blk.head(x, w, ids, items)[1]))
    dX, dW, _ = blk.head_grad(X, W, ids, items, d)
    u, v = rng.standard_normal(X.shape), rng.standard_normal(W.shape)
    e = 1e-5
    assert abs((loss(X + e * u, W) - loss(X - e * u, W)) / (2 * e) - (dX * u).sum()) < 1e-7
    assert abs((loss(X, W + e * v) - loss(X, W - e * v)) / (2 * e) - (dW * v).sum()) < 1e-7
