"""What stands beside attention in a model trained on prefix-shared sequences: the embedding, the layer norm (with the
residual sum in front of it) and the gated feed-forward block, forward and backward.

`run` makes one pass, in elementary torch operations or (`own`) through the library's entry points.  All three
operators act on single tokens: a packed buffer of T tokens is T rows.

Kinds
  embed  rows of a table by token id, scaled; the table's gradient.  Ids are log-uniform (a natural text's few frequent
         and many rare tokens), one in twenty is padding (-1), whose rows are zero and give no gradient
  norm   layer norm over the last axis, of X or of X + residual; gradients of X, weight and bias
  ffn    Y = (act(X Wg^T) * (X Wu^T)) Wd^T; gradients of X and of the three weights
`train` adds the backward pass.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # generation: the embedding of one token per step
        dict(name="embed_one_token", kind="embed", dtype="bf16", tokens=1, vocab=32000, hidden=4096, train=False),
        # a training step's packed rows, four of 16 384 tokens, on the width of 64 heads of 128
        dict(name="embed_packed_rows", kind="embed", dtype="bf16", tokens=65536, vocab=32000, hidden=8192, train=True),
        # a batch of moderate samples in fp32: odd vocabulary, rows that are not 16-byte aligned
        dict(name="embed_odd_fp32", kind="embed", dtype="f32", tokens=8334, vocab=50257, hidden=1001, train=True),
        # generation: the norm of one token behind a residual sum
        dict(name="norm_one_token", kind="norm", dtype="bf16", rows=1, hidden=4096, residual=True, bias=True, train=False),
        # a batch of moderate samples, between two sub-layers of a block
        dict(name="norm_moderate_batch", kind="norm", dtype="bf16", rows=8334, hidden=4096, residual=True, bias=True, train=True),
        # a training step's packed rows
        dict(name="norm_packed_rows", kind="norm", dtype="bf16", rows=65536, hidden=8192, residual=False, bias=True, train=True),
        # numerics check in fp32, odd width, no bias
        dict(name="norm_odd_fp32", kind="norm", dtype="f32", rows=2331, hidden=1001, residual=False, bias=False, train=True),
        # generation: one token through the feed-forward block, whose weights have to be read
        dict(name="ffn_one_token", kind="ffn", dtype="bf16", tokens=1, hidden=4096, inner=14336, act="silu", train=False),
        # one short dialogue per device: few rows, gradients of all weights
        dict(name="ffn_short_sample", kind="ffn", dtype="bf16", tokens=221, hidden=4096, inner=14336, act="silu", train=True),
        # packed rows of moderate samples: the largest step
        dict(name="ffn_packed_rows", kind="ffn", dtype="bf16", tokens=16384, hidden=4096, inner=14336, act="silu", train=True),
        # sizes that are no multiples of anything
        dict(name="ffn_odd_sizes", kind="ffn", dtype="bf16", tokens=1037, hidden=1001, inner=2731, act="gelu", train=True),
        # numerics check in fp32 on one short sample
        dict(name="ffn_fp32", kind="ffn", dtype="f32", tokens=168, hidden=512, inner=1376, act="gelu", train=True),
    ]


# a drawn case costs no more than the largest listed one
_MOST_EMBED = 65536 * 8192 * 2 * 2
_MOST_NORM = 65536 * 8192 * 2
_MOST_FFN = 18 * 16384 * 4096 * 14336


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: two in three are multiples of 64, as models have them, one in three is any number."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 1 / 3 else max(lo, n // 64 * 64)


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    while True:
        kind = rng.choice(("embed", "norm", "ffn", "ffn"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        train = rng.random() < 0.7
        if kind == "embed":
            case = dict(kind=kind, dtype=dtype, tokens=_log(rng, 1, 65536), vocab=_log(rng, 1000, 130000), hidden=_width(rng, 64, 8192),
                        train=train)
            if (2 * case["tokens"] + case["vocab"]) * case["hidden"] * _BYTES[dtype] <= _MOST_EMBED:
                return case
        elif kind == "norm":
            case = dict(kind=kind, dtype=dtype, rows=_log(rng, 1, 65536), hidden=_width(rng, 64, 16384), residual=rng.random() < 0.5,
                        bias=rng.random() < 0.5, train=train)
            if case["rows"] * case["hidden"] * _BYTES[dtype] * (2 if case["residual"] else 1) <= _MOST_NORM:
                return case
        else:
            case = dict(kind=kind, dtype=dtype, tokens=_log(rng, 1, 16384), hidden=_width(rng, 256, 8192), inner=_width(rng, 512, 28672),
                        act=rng.choice(("silu", "gelu")), train=train)
            # an fp32 product costs some sixteen bf16 ones
            if work(case)["flops"] * (16 if dtype == "f32" else 1) <= _MOST_FFN:
                return case


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 17)
    dt, kind = _DTYPES[case["dtype"]], case["kind"]

    def randn(*shape, scale=1.0, shift=0.0):
        t = torch.empty(shape, dtype=dt, device="cuda")
        rows = max(1, (1 << 26) // max(1, shape[-1])) if len(shape) > 1 else shape[0]
        for at in range(0, shape[0], rows):
            part = t[at:at + rows]
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(scale).add_(shift))
        return t

    s = {"case": dict(case)}
    if kind == "embed":
        T, V, h = case["tokens"], case["vocab"], case["hidden"]
        u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * math.log(V + 1.0)).to(torch.int64) - 1).clamp_(0, V - 1).to(torch.int32)
        if T > 1:
            ids[torch.rand(T, generator=gen, device="cuda") < 0.05] = -1
        s["ids"], s["W"], s["scale"] = ids, randn(V, h, scale=0.02), math.sqrt(h)
        if case["train"]:
            s["dX"] = randn(T, h)
    elif kind == "norm":
        n, h = case["rows"], case["hidden"]
        s["X"] = randn(n, h, shift=0.1)
        s["R"] = randn(n, h, scale=2.0) if case["residual"] else None
        s["w"], s["b"], s["eps"] = randn(h, scale=0.1, shift=1.0), randn(h, scale=0.1) if case["bias"] else None, 1e-5
        if case["train"]:
            s["dY"] = randn(n, h)
            s["dS"] = randn(n, h) if case["residual"] else None  # what reaches the sum from the other branch
    else:
        T, h, n = case["tokens"], case["hidden"], case["inner"]
        s["X"], s["act"] = randn(T, h), case["act"]
        s["Wg"], s["Wu"] = randn(n, h, scale=h ** -0.5), randn(n, h, scale=h ** -0.5)
        s["Wd"] = randn(h, n, scale=n ** -0.5)
        if case["train"]:
            s["dY"] = randn(T, h)
    return s


# ------------------------------------------------------------------ plain forms
def _embed(s):
    ids, W, scale = s["ids"].long(), s["W"], s["scale"]
    real = (ids >= 0) & (ids < W.shape[0])
    at = torch.where(real, ids, torch.zeros_like(ids))
    X = torch.where(real[:, None], W[at].float() * scale, 0.0).to(W.dtype)
    if not s["case"]["train"]:
        return {"X": X}
    dW = torch.zeros(W.shape, dtype=torch.float32, device=W.device)
    dW.index_add_(0, at, torch.where(real[:, None], s["dX"].float() * scale, 0.0))
    return {"X": X, "dW": dW.to(W.dtype)}


def _norm(s):
    dt = s["X"].dtype
    # the residual stream is held in the element type, and the norm is that of the held sum
    S = s["X"] if s["R"] is None else (s["X"].float() + s["R"].float()).to(dt)
    x, w = S.float(), s["w"].float()
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + s["eps"])
    xh = (x - mean) * rstd
    Y = xh * w if s["b"] is None else xh * w + s["b"].float()
    out = {"Y": Y.to(dt)}
    if s["R"] is not None:
        out["S"] = S
    if s["case"]["train"]:
        dy = s["dY"].float()
        g = dy * w
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        if s["dS"] is not None:
            dx = dx + s["dS"].float()
        out["dX"], out["dw"] = dx.to(dt), (dy * xh).sum(0).to(dt)
        if s["b"] is not None:
            out["db"] = dy.sum(0).to(dt)
    return out


def _act(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        sg = 1.0 / (1.0 + torch.exp(-g))
        return g * sg, sg * (1.0 + g * (1.0 - sg))
    cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _ffn(s):
    dt = s["X"].dtype
    x, wg, wu, wd = (s[k].float() for k in ("X", "Wg", "Wu", "Wd"))
    g, u = x @ wg.T, x @ wu.T
    a, da = _act(g, s["act"])
    h = a * u
    out = {"Y": (h @ wd.T).to(dt)}
    if s["case"]["train"]:
        dy = s["dY"].float()
        dh = dy @ wd
        out["dWd"] = (dy.T @ h).to(dt)
        du, dg = dh * a, dh * u * da
        out["dX"] = (dg @ wg + du @ wu).to(dt)
        out["dWg"], out["dWu"] = (dg.T @ x).to(dt), (du.T @ x).to(dt)
    return out


# ------------------------------------------------------------------ the library's entry points
def _own(s):
    import paper_2410_20305_amd as ps
    case = s["case"]
    if case["kind"] == "embed":
        out = {"X": ps.psattn_embed_fwd(s["ids"], s["W"], scale=s["scale"])}
        if case["train"]:
            out["dW"] = ps.psattn_embed_bwd(s["ids"], s["dX"], case["vocab"], scale=s["scale"])
        return out
    if case["kind"] == "norm":
        Y, S, mean, rstd = ps.psattn_layernorm_fwd(s["X"], s["w"], s["b"], s["eps"], residual=s["R"])
        out = {"Y": Y}
        if s["R"] is not None:
            out["S"] = S
        if case["train"]:
            out["dX"], out["dw"], db = ps.psattn_layernorm_bwd(S, s["w"], mean, rstd, s["dY"], dS=s["dS"], bias=s["b"] is not None)
            if s["b"] is not None:
                out["db"] = db
        return out
    W = (s["X"], s["Wg"], s["Wu"], s["Wd"])
    if not case["train"]:
        return {"Y": ps.psattn_ffn_fwd(*W, act=s["act"], keep=False)[0]}
    Y, kept = ps.psattn_ffn_fwd(*W, act=s["act"])
    dX, dWg, dWu, dWd = ps.psattn_ffn_bwd(*W, kept, s["dY"], act=s["act"])
    return {"Y": Y, "dWd": dWd, "dX": dX, "dWg": dWg, "dWu": dWu}


def run(state):
    if own:
        return _own(state)
    return {"embed": _embed, "norm": _norm, "ffn": _ffn}[state["case"]["kind"]](state)


def work(case):
    e = _BYTES[case["dtype"]]
    if case["kind"] == "embed":
        T, V, h = case["tokens"], case["vocab"], case["hidden"]
        n = min(T, V) * h * e + 4 * T + T * h * e
        return {"bytes": n + (T * h * e + V * h * e if case["train"] else 0), "flops": T * h * (2 if case["train"] else 1)}
    if case["kind"] == "norm":
        n, h = case["rows"], case["hidden"]
        fwd, bwd = (4, 2) if case["residual"] else (2, 2)  # rows in and out; S is in hand when the backward starts
        return {"bytes": n * h * e * (fwd + (bwd + (1 if case["residual"] else 0) if case["train"] else 0)), "flops": n * h * (20 if case["train"] else 8)}
    T, h, n = case["tokens"], case["hidden"], case["inner"]
    weights, rows = 3 * h * n * e, T * h * e
    return {"bytes": weights + 2 * rows + (weights + 2 * rows if case["train"] else 0), "flops": (18 if case["train"] else 6) * T * h * n}


def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits."""
    s = prepare(case, seed)
    d = lambda t: t.to(torch.float64)
    if case["kind"] == "embed":
        ids, V = s["ids"].long(), case["vocab"]
        keep = torch.nonzero((ids >= 0) & (ids < V))[:, 0]
        X = torch.zeros(ids.shape[0], case["hidden"], dtype=torch.float64, device="cuda")
        X[keep] = d(s["W"])[ids[keep]] * s["scale"]
        if not case["train"]:
            return {"X": X}
        dW = torch.zeros(V, case["hidden"], dtype=torch.float64, device="cuda")
        dW.index_put_((ids[keep],), d(s["dX"][keep]), accumulate=True)
        return {"X": X, "dW": dW * s["scale"]}
    if case["kind"] == "norm":
        held = s["X"] if s["R"] is None else (d(s["X"]) + d(s["R"])).to(s["X"].dtype)
        x, h = d(held), case["hidden"]
        mu = x.sum(1) / h
        c = x - mu[:, None]
        r = ((c * c).sum(1) / h + s["eps"]).rsqrt()
        n = c * r[:, None]
        Y = n * d(s["w"])
        out = {"Y": Y if s["b"] is None else Y + d(s["b"])}
        if s["R"] is not None:
            out["S"] = d(s["X"]) + d(s["R"])
        if case["train"]:
            dy = d(s["dY"])
            q = dy * d(s["w"])
            dx = (q - (q.sum(1) / h)[:, None] - n * ((q * n).sum(1) / h)[:, None]) * r[:, None]
            out["dX"] = dx if s["dS"] is None else dx + d(s["dS"])
            out["dw"] = torch.sum(dy * n, 0)
            if s["b"] is not None:
                out["db"] = torch.sum(dy, 0)
        return out
    x, wg, wu, wd = d(s["X"]), d(s["Wg"]), d(s["Wu"]), d(s["Wd"])
    G, U = torch.mm(x, wg.t()), torch.mm(x, wu.t())
    if case["act"] == "silu":
        sig = torch.sigmoid(G)
        A, dA = G * sig, sig + G * sig * (1 - sig)
    else:
        phi = 0.5 * torch.erfc(-G / math.sqrt(2.0))
        A, dA = G * phi, phi + G * torch.exp(-G * G / 2) / math.sqrt(2 * math.pi)
    H = A * U
    out = {"Y": torch.mm(H, wd.t())}
    if case["train"]:
        dy = d(s["dY"])
        dH = torch.mm(dy, wd)
        dG, dU = dH * U * dA, dH * A
        out["dWd"] = torch.mm(dy.t(), H)
        out["dX"] = torch.mm(dG, wg) + torch.mm(dU, wu)
        out["dWg"], out["dWu"] = torch.mm(dG.t(), x), torch.mm(dU.t(), x)
    return out
