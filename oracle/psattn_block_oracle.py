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
