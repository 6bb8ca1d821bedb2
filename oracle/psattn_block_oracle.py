"""CPU oracle of what stands beside attention: embedding, layer norm, gated feed-forward block.  numpy, fp64, written
from the definitions; shares no code with the GPU path.  Test infrastructure only."""
import math

import numpy as np

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def embed(ids, W, scale):
    X = np.zeros((len(ids), W.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < W.shape[0]:
            X[t] = scale * W[v]
    return X


def embed_grad(ids, dX, vocab, scale):
    dW = np.zeros((vocab, dX.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < vocab:
            dW[v] += scale * dX[t]
    return dW


def layernorm(S, w, b, eps):
    """Y, mean, rstd."""
    mean = S.mean(1)
    c = S - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).mean(1) + eps)
    Y = c * rstd[:, None] * w
    return (Y if b is None else Y + b), mean, rstd


def layernorm_grad(S, w, eps, dY, dS=None):
    """dX, dw, db."""
    _, mean, rstd = layernorm(S, w, None, eps)
    xh = (S - mean[:, None]) * rstd[:, None]
    q = dY * w
    dX = rstd[:, None] * (q - q.mean(1)[:, None] - xh * (q * xh).mean(1)[:, None])
    return (dX if dS is None else dX + dS), (dY * xh).sum(0), dY.sum(0)


def act(g, kind):
    """act(g) and its derivative."""
    if kind == "silu":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s + g * s * (1.0 - s)
    cdf = 0.5 * _erfc(-g / math.sqrt(2.0))
    return g * cdf, cdf + g * np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def ffn(X, Wg, Wu, Wd, kind, hold=lambda x: x):
    """Y, G, U, H; `hold` is the rounding of H to the element type."""
    G, U = X @ Wg.T, X @ Wu.T
    H = hold(act(G, kind)[0] * U)
    return H @ Wd.T, G, U, H


def ffn_grad(X, Wg, Wu, Wd, G, U, H, dY, kind, hold=lambda x: x):
    """dX, dWg, dWu, dWd and the held dG, dU, from the kept G, U, H."""
    a, da = act(G, kind)
    dH = dY @ Wd
    dG, dU = hold(dH * U * da), hold(dH * a)
    return dG @ Wg + dU @ Wu, dG.T @ X, dU.T @ X, dY.T @ H, dG, dU


def gatednorm(X, B, w_pre, w_post, gate, res, eps, hold=lambda x: x):
    """Y, S, rstd_b, rstd_s: S = res X + gate o rmsnorm(B) w_post (X itself without B), Y = rmsnorm(S) w_pre; `hold` is the
    rounding of S to the element type."""
    S, rb = X, None
    if B is not None:
        N = B
        if w_post is not None:
            rb = 1.0 / np.sqrt((B * B).mean(1) + eps)
            N = B * rb[:, None] * w_post
        S = hold(res * X + (N if gate is None else gate * N))
    rs = 1.0 / np.sqrt((S * S).mean(1) + eps)
    return S * rs[:, None] * w_pre, S, rb, rs


def rmsnorm_grad(x, eps, g):
    """Gradient of x from that of x / sqrt(mean(x^2) + eps)."""
    r = 1.0 / np.sqrt((x * x).mean(1) + eps)[:, None]
    return r * g - x * r ** 3 * (g * x).mean(1)[:, None]


def gatednorm_grad(B, S, w_pre, w_post, gate, res, eps, dY, dS=None):
    """dX, dB, dw_pre, dw_post, dgate (None where there is none)."""
    r = 1.0 / np.sqrt((S * S).mean(1) + eps)[:, None]
    ds = rmsnorm_grad(S, eps, dY * w_pre)
    if dS is not None:
        ds = ds + dS
    dw_pre = (dY * S * r).sum(0)
    if B is None:
        return ds, None, dw_pre, None, None
    n = B if w_post is None else B / np.sqrt((B * B).mean(1) + eps)[:, None]
    out = n if w_post is None else n * w_post  # what the gate multiplies
    dgate = None
    if gate is not None:
        dgate = ds * out if gate.ndim == 2 and gate.shape[0] == B.shape[0] and B.shape[0] > 1 else (ds * out).sum(0).reshape(gate.shape)
    dN = ds if gate is None else ds * gate
    if w_post is None:
        return res * ds, dN, dw_pre, None, dgate
    return res * ds, rmsnorm_grad(B, eps, dN * w_post), dw_pre, (dN * n).sum(0), dgate


def rotary(x, pos, freqs, interleaved=False, amplitude=1.0, transposed=False, n_positions=None):
    """x [T, H, d]: pairs of the first 2 len(freqs) dimensions turned by pos * freqs, the others as they are; rows of positions outside
    [0, n_positions) are zeros."""
    n = len(freqs)
    y = np.array(x, dtype=np.float64)
    for t, p in enumerate(pos):
        if n_positions is not None and not 0 <= p < n_positions:
            y[t] = 0
            continue
        for i, f in enumerate(freqs):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
            turn = amplitude * np.array([[math.cos(p * f), -math.sin(p * f)], [math.sin(p * f), math.cos(p * f)]])
            if transposed:
                turn = turn.T
            y[t][:, [a, b]] = x[t][:, [a, b]] @ turn.T
    return y


def rotary_frequencies(n, theta, scaling="none", factor=1.0, original=0.0, low=1.0, high=32.0):
    if scaling == "base" and n > 2:
        theta = theta * factor ** (n / (n - 2.0))
    f = np.array([theta ** (-2.0 * i / n) for i in range(n // 2)])
    if scaling == "linear":
        return f / factor
    if scaling != "parts":
        return f
    out = []
    for x in f:
        turns = original * x / (2 * math.pi)
        k = 0.0 if turns <= low else 1.0 if turns >= high else (turns - low) / (high - low)
        out.append(k * x + (1 - k) * x / factor)
    return np.array(out)


def head(X, W, token_ids, items):
    """Log-sum-exp of every row's logits X W^T, and log-probabilities of the items (response, row, token's place); one whose id is no
    token of the vocabulary gets 0."""
    Z = X @ W.T
    top = Z.max(1)
    lse = top + np.log(np.exp(Z - top[:, None]).sum(1))
    ok = lambda t: 0 <= token_ids[t] < W.shape[0]
    return lse, np.array([Z[r, token_ids[t]] - lse[r] if ok(t) else 0.0 for _, r, t in items])


def head_grad(X, W, token_ids, items, d):
    """dX, dW and dlogits of sum over the items of d[response] * log-probability."""
    Z = X @ W.T
    P = np.exp(Z - Z.max(1)[:, None])
    P /= P.sum(1)[:, None]
    G = np.zeros_like(Z)
    for j, r, t in items:
        if 0 <= token_ids[t] < W.shape[0]:
            G[r] -= d[j] * P[r]
            G[r, token_ids[t]] += d[j]
    return G @ W, G.T @ X, G
