"""Further parts of a model trained on prefix-shared sequences: the vocabulary head that never keeps its logits, rotary positions
of any layout, and RMS norms before and after a block with its gate and residual scale; forward and backward.

`run` makes one pass, in elementary torch operations or (`own`) through the library's entry points.

Kinds
  head   log-probabilities of the responses of packed samples [prompt | response 1 | ... | response k] from hidden rows X and the
         vocabulary matrix W: log pi = sum over a response's tokens of X[row].W[token] - log sum exp(X[row].W^T); gradients of X and W.
         The row of a token predicts the next token of its branch, the last prompt row the first token of every response
  rope   Q and K turned by position: pairs (i, i + n / 2) or (2 i, 2 i + 1) of the first n dimensions of a head, frequencies as they
         are or scaled for long contexts; the gradient (the transposed turn)
  join   S = res * X + gate * rmsnorm(B) w_post, Y = rmsnorm(S) w_pre: a block's output joins the residual stream and the next
         block's input leaves it; gradients of X, B, the weights and the gate
`train` adds the backward pass.
"""
import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # generation: what one sampled token's log-probability costs
        dict(name="head_one_token", kind="head", dtype="bf16", tokens=2, samples=1, responses=1, prompt=0.5, vocab=32000, hidden=4096, train=False),
        # one short dialogue per device, two responses
        dict(name="head_short_sample", kind="head", dtype="bf16", tokens=221, samples=1, responses=2, prompt=0.45, vocab=32000, hidden=4096, train=True),
        # a frozen policy's log-probabilities of a batch of moderate samples
        dict(name="head_frozen_policy", kind="head", dtype="bf16", tokens=8334, samples=8, responses=2, prompt=0.6, vocab=128000, hidden=4096, train=False),
        # a training step on packed rows, four responses to a prompt, large vocabulary: the largest
        dict(name="head_packed_rows", kind="head", dtype="bf16", tokens=16384, samples=24, responses=4, prompt=0.4, vocab=128000, hidden=4096, train=True),
        # numerics check in fp32: odd vocabulary, rows that are not 16-byte aligned
        dict(name="head_odd_fp32", kind="head", dtype="f32", tokens=1037, samples=5, responses=2, prompt=0.3, vocab=50257, hidden=1001, train=True),
        # generation: Q and K of one token far into a conversation
        dict(name="rope_one_token", kind="rope", dtype="bf16", tokens=1, q_heads=32, kv_heads=8, head_dim=128, rotary=128, layout="half", scaling="none",
             positions=8192, fused=True, train=False),
        # a training step's packed rows, four of 16 384 tokens
        dict(name="rope_packed_rows", kind="rope", dtype="bf16", tokens=65536, q_heads=64, kv_heads=8, head_dim=128, rotary=128, layout="half", scaling="none",
             positions=16384, fused=True, train=True),
        # half of each small head, neighbours paired, frequencies stretched by parts for a long context, fp32
        dict(name="rope_part_of_head", kind="rope", dtype="f32", tokens=8334, q_heads=16, kv_heads=16, head_dim=64, rotary=32, layout="interleaved",
             scaling="parts", positions=131072, fused=False, train=True),
        # generation: one token between two parts of a block
        dict(name="join_one_token", kind="join", dtype="bf16", rows=1, hidden=4096, post=True, gate="row", train=False),
        # a batch of moderate samples, one learned gate for all rows
        dict(name="join_moderate_batch", kind="join", dtype="bf16", rows=8334, hidden=4096, post=True, gate="row", train=True),
        # a training step's packed rows, a gate of its own for each row
        dict(name="join_packed_rows", kind="join", dtype="bf16", rows=65536, hidden=8192, post=True, gate="all", train=True),
        # numerics check in fp32, odd width, without a gate
        dict(name="join_odd_fp32", kind="join", dtype="f32", rows=2331, hidden=1001, post=True, gate="none", train=True),
    ]


# a drawn case costs no more than the largest listed one
_MOST_HEAD = 6 * 9700 * 128000 * 4096
_MOST_ROPE = 65536 * 72 * 128 * 2 * 4
_MOST_JOIN = 65536 * 8192 * 2 * 10


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: two in three are multiples of 64, as models have them, one in three is any number."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 1 / 3 else max(lo, n // 64 * 64)


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    while True:
        kind = rng.choice(("head", "head", "rope", "join"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        train = rng.random() < 0.7
        if kind == "head":
            tokens = _log(rng, 2, 16384)
            samples = min(_log(rng, 1, 64), max(1, tokens // 8))
            case = dict(kind=kind, dtype=dtype, tokens=tokens, samples=samples, responses=rng.choice((1, 2, 2, 2, 4, 8)), prompt=round(rng.uniform(0.1, 0.8), 3),
                        vocab=_log(rng, 1000, 130000), hidden=_width(rng, 256, 8192), train=train)
            # an fp32 product costs some sixteen bf16 ones
            if work(case)["flops"] * (16 if dtype == "f32" else 1) <= _MOST_HEAD:
                return case
        elif kind == "rope":
            head_dim = rng.choice((64, 128, 128, 256, 80))
            group = rng.choice((1, 4, 8))
            kv = _log(rng, 1, 16)
            case = dict(kind=kind, dtype=dtype, tokens=_log(rng, 1, 65536), q_heads=kv * group, kv_heads=kv, head_dim=head_dim,
                        rotary=rng.choice((head_dim, head_dim, head_dim // 2, head_dim // 4 // 2 * 2)), layout=rng.choice(("half", "interleaved")),
                        scaling=rng.choice(("none", "linear", "base", "parts")), positions=_log(rng, 2048, 131072), fused=rng.random() < 0.5, train=train)
            if work(case)["bytes"] <= _MOST_ROPE:
                return case
        else:
            case = dict(kind=kind, dtype=dtype, rows=_log(rng, 1, 65536), hidden=_width(rng, 64, 16384), post=rng.random() < 0.8,
                        gate=rng.choice(("none", "row", "all")), train=train)
            if work(case)["bytes"] <= _MOST_JOIN:
                return case


def _table(case):
    """A packed buffer of `tokens`: offset, prompt length and response lengths of every sample."""
    rng = random.Random(case["tokens"] * 1009 + case["samples"])
    n, k, T = case["samples"], case["responses"], case["tokens"]
    if n * (k + 1) > T:
        n, k = 1, min(k, T - 1)
    share = [rng.uniform(0.5, 1.5) for _ in range(n)]
    free, whole = T - n * (k + 1), sum(share)
    off, prefix, resp, at = [], [], [], 0
    for s in share:
        more = int(free * s / whole)
        p = int(more * case["prompt"])
        part = [rng.uniform(0.5, 1.5) for _ in range(k)]
        lens = [1 + int((more - p) * x / sum(part)) for x in part]
        off.append(at)
        prefix.append(1 + p)
        resp.append(lens)
        at += 1 + p + sum(lens)
    return off, prefix, resp


def _items(table):
    """(row that predicts, token that is predicted, response) of every token of every response; responses count on over the samples."""
    rows, toks, which, j = [], [], [], 0
    for off, p, lens in zip(*table):
        at = off + p
        for n in lens:
            for u in range(n):
                rows.append(off + p - 1 if u == 0 else at + u - 1)
                toks.append(at + u)
                which.append(j)
            at += n
            j += 1
    return rows, toks, which


_THETA, _FACTOR, _ORIGINAL, _LOW, _HIGH = 10000.0, 8.0, 4096, 1.0, 32.0


def _amplitude(case):
    """Rotary tables stretched by parts also turn the scores' temperature."""
    return 0.1 * math.log(_FACTOR) + 1.0 if case["scaling"] == "parts" else 1.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 29)
    dt, kind = _DTYPES[case["dtype"]], case["kind"]

    def randn(*shape, scale=1.0, shift=0.0):
        t = torch.empty(shape, dtype=dt, device="cuda")
        flat = t.view(shape[0], -1) if len(shape) > 1 else t
        rows = max(1, (1 << 26) // max(1, flat.shape[-1])) if len(shape) > 1 else shape[0]
        for at in range(0, shape[0], rows):
            part = flat[at:at + rows]
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(scale).add_(shift))
        return t

    s = {"case": dict(case)}
    if kind == "head":
        T, V, h = case["tokens"], case["vocab"], case["hidden"]
        table = _table(case)
        u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * math.log(V + 1.0)).to(torch.int64) - 1).clamp_(0, V - 1)
        W = randn(V, h, scale=1.3 * h ** -0.5)
        rows, toks, which = (torch.tensor(x, device="cuda") for x in _items(table))
        # a trained model: the rows lean towards the tokens that follow, by anything from nothing to certainty
        X = torch.randn((T, h), generator=gen, device="cuda")
        to = dict(zip(rows.tolist(), toks.tolist()))  # of a row with several such tokens, the last
        lean, to = torch.tensor(list(to.keys()), device="cuda"), torch.tensor(list(to.values()), device="cuda")
        X[lean] += W[ids[to]].float() * (torch.rand((len(lean), 1), generator=gen, device="cuda") * 8.0)
        s["X"], s["W"], s["ids"] = X.to(dt), W, ids.to(torch.int32)
        s["rows"], s["toks"], s["which"], s["n"] = rows, toks, which, sum(len(x) for x in table[2])
        if case["train"]:
            # beta times a sigmoid, chosen responses up and the others down
            d = torch.rand(s["n"], generator=gen, device="cuda") * 0.1
            s["d"] = torch.where(torch.arange(s["n"], device="cuda") % max(1, case["responses"]) == 0, -d, d)
        if own:
            import paper_2410_20305_amd as ps
            ptr = [0]
            for x in table[2]:
                ptr.append(ptr[-1] + len(x))
            s["plan"] = ps.LogprobPlan(table[0], table[1], ptr, [n for x in table[2] for n in x], T)
    elif kind == "rope":
        T, hq, hk, d = case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
        s["pos"] = torch.randint(0, case["positions"], (T,), generator=gen, device="cuda", dtype=torch.int32)
        if T > 1:  # runs that count on, as prompts and responses have them
            run = torch.arange(T, device="cuda", dtype=torch.int32)
            step = max(1, min(case["positions"], T // 7 + 1))
            s["pos"] = (run % step + s["pos"][run.long() // step] % max(1, case["positions"] - step + 1)).to(torch.int32)
        if case["fused"]:  # slices of what one projection has written
            whole = randn(T, hq + 2 * hk, d)
            s["Q"], s["K"] = whole[:, :hq], whole[:, hq:hq + hk]
        else:
            s["Q"], s["K"] = randn(T, hq, d), randn(T, hk, d)
        if case["train"]:
            s["dQ"], s["dK"] = randn(T, hq, d), randn(T, hk, d)
        if own:
            import paper_2410_20305_amd as ps
            freqs = ps.psattn_rope_frequencies(case["rotary"], _THETA, scaling=case["scaling"], factor=_FACTOR, original_positions=_ORIGINAL, low=_LOW, high=_HIGH)
            s["rope"] = ps.Rope(d, _THETA, case["positions"], rotary_dim=case["rotary"], layout=case["layout"], frequencies=freqs, amplitude=_amplitude(case))
    else:
        n, h = case["rows"], case["hidden"]
        s["X"], s["B"], s["res"], s["eps"] = randn(n, h, scale=2.0), randn(n, h, scale=0.5, shift=0.05), 0.875, 1e-6
        s["w_pre"], s["w_post"] = randn(h, scale=0.1, shift=1.0), randn(h, scale=0.1, shift=0.7) if case["post"] else None
        s["gate"] = None if case["gate"] == "none" else randn(h, scale=0.2, shift=0.5) if case["gate"] == "row" else randn(n, h, scale=0.3, shift=0.5)
        if case["train"]:
            s["dY"], s["dS"] = randn(n, h), randn(n, h)
    return s


# ------------------------------------------------------------------ plain forms
_PIECE = 16384  # rows of the vocabulary at a time


def _head(s):
    case, dt = s["case"], s["X"].dtype
    T, V = case["tokens"], case["vocab"]
    rows, W = s["rows"], s["W"]
    target = s["ids"][s["toks"]].long()
    x = s["X"][rows].float()
    top = torch.full((len(rows),), -math.inf, device=x.device)
    total, hit = torch.zeros_like(top), torch.zeros_like(top)
    for at in range(0, V, _PIECE):
        z = x @ W[at:at + _PIECE].float().T
        new = torch.maximum(top, z.max(1).values)
        total = total * torch.exp(top - new) + torch.exp(z - new[:, None]).sum(1)
        top = new
        inside = (target >= at) & (target < at + z.shape[1])
        col = torch.where(inside, target - at, 0)
        hit = torch.where(inside, z[torch.arange(len(rows), device=x.device), col], hit)
    lse = top + torch.log(total)
    row_lse = torch.zeros(T, device=x.device)
    row_lse[rows] = lse
    logp = torch.zeros(s["n"], device=x.device).index_add_(0, s["which"], hit - lse)
    out = {"row_lse": row_lse, "logp": logp}
    if case["train"]:
        w = s["d"][s["which"]][:, None]
        dx, dW = torch.zeros_like(x), torch.empty(W.shape, dtype=dt, device=x.device)
        for at in range(0, V, _PIECE):
            part = W[at:at + _PIECE].float()
            g = -w * torch.exp(x @ part.T - lse[:, None])
            inside = torch.nonzero((target >= at) & (target < at + g.shape[1]))[:, 0]
            g[inside, target[inside] - at] += w[inside, 0]
            dx += g @ part
            dW[at:at + _PIECE] = (g.T @ x).to(dt)
        out["dX"] = torch.zeros(s["X"].shape, device=x.device).index_add_(0, rows, dx).to(dt)
        out["dW"] = dW
    return out


def _frequencies(case, device):
    n = case["rotary"]
    theta = _THETA * _FACTOR ** (n / (n - 2)) if case["scaling"] == "base" and n > 2 else _THETA
    f = theta ** (-2.0 * torch.arange(n // 2, dtype=torch.float64, device=device) / n)
    if case["scaling"] == "linear":
        f = f / _FACTOR
    elif case["scaling"] == "parts":
        turns = f * _ORIGINAL / (2.0 * math.pi)  # that a dimension makes over the original context
        keep = ((turns - _LOW) / (_HIGH - _LOW)).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / _FACTOR
    return f


def _turn(x, cos, sin, case):
    n = case["rotary"]
    y = x.float()
    if case["layout"] == "half":
        a, b = y[..., :n // 2], y[..., n // 2:n]
    else:
        a, b = y[..., 0:n:2], y[..., 1:n:2]
    u, v = a * cos - b * sin, b * cos + a * sin
    out = y.clone()
    if case["layout"] == "half":
        out[..., :n // 2], out[..., n // 2:n] = u, v
    else:
        out[..., 0:n:2], out[..., 1:n:2] = u, v
    return out.to(x.dtype)


def _rope(s):
    case = s["case"]
    angle = s["pos"].double()[:, None, None] * _frequencies(case, s["pos"].device)
    a = _amplitude(case)
    cos, sin = (a * torch.cos(angle)).float(), (a * torch.sin(angle)).float()
    out = {"Qr": _turn(s["Q"], cos, sin, case), "Kr": _turn(s["K"], cos, sin, case)}
    if case["train"]:
        out["dQ"], out["dK"] = _turn(s["dQ"], cos, -sin, case), _turn(s["dK"], cos, -sin, case)
    return out


def _join(s):
    dt, h = s["X"].dtype, s["case"]["hidden"]
    b, w_pre = s["B"].float(), s["w_pre"].float()
    gate = 1.0 if s["gate"] is None else s["gate"].float()
    if s["w_post"] is not None:
        rb = 1.0 / torch.sqrt((b * b).mean(1, keepdim=True) + s["eps"])
        bh, w_post = b * rb, s["w_post"].float()
    else:
        bh, w_post = b, 1.0
    # the residual stream is held in the element type, and the second norm is that of the held sum
    S = (s["res"] * s["X"].float() + gate * (bh * w_post)).to(dt)
    x = S.float()
    rs = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + s["eps"])
    xh = x * rs
    out = {"S": S, "Y": (xh * w_pre).to(dt)}
    if s["case"]["train"]:
        dy = s["dY"].float()
        q = dy * w_pre
        ds = s["dS"].float() + rs * (q - xh * (q * xh).mean(1, keepdim=True))
        out["dX"], out["dw_pre"] = (s["res"] * ds).to(dt), (dy * xh).sum(0).to(dt)
        c = ds * bh
        if s["gate"] is not None:
            dg = c * w_post
            out["dgate"] = (dg.sum(0) if s["gate"].dim() == 1 else dg).to(dt)
        db = ds * gate
        if s["w_post"] is not None:
            out["dw_post"] = (c * gate).sum(0).to(dt)
            db = db * w_post
            db = rb * (db - bh * (db * bh).mean(1, keepdim=True))
        out["dB"] = db.to(dt)
    return out


# ------------------------------------------------------------------ the library's entry points
def _own(s):
    import paper_2410_20305_amd as ps
    case = s["case"]
    if case["kind"] == "head":
        row_lse, logp = ps.psattn_head_logprob_fwd(s["plan"], s["X"], s["W"], s["ids"])
        out = {"row_lse": row_lse, "logp": logp}
        if case["train"]:
            out["dX"], out["dW"] = ps.psattn_head_logprob_bwd(s["plan"], s["X"], s["W"], s["ids"], row_lse, s["d"])
        return out
    if case["kind"] == "rope":
        Qr, Kr = ps.psattn_rope_apply(s["rope"], s["Q"], s["K"], positions=s["pos"])
        out = {"Qr": Qr, "Kr": Kr}
        if case["train"]:
            out["dQ"], out["dK"] = ps.psattn_rope_apply_bwd(s["rope"], s["dQ"], s["dK"], positions=s["pos"])
        return out
    form = dict(w_post=s["w_post"], gate=s["gate"], res_scale=s["res"])
    Y, S, rstd_b, rstd_s = ps.psattn_gatednorm_fwd(s["X"], s["B"], s["w_pre"], eps=s["eps"], **form)
    out = {"S": S, "Y": Y}
    if case["train"]:
        dX, dB, dw_pre, dw_post, dgate = ps.psattn_gatednorm_bwd(s["B"], S, s["w_pre"], rstd_b, rstd_s, s["dY"], dS=s["dS"], **form)
        out.update(dX=dX, dw_pre=dw_pre, dB=dB)
        if dw_post is not None:
            out["dw_post"] = dw_post
        if dgate is not None:
            out["dgate"] = dgate
    return out


def run(state):
    if own:
        return _own(state)
    return {"head": _head, "rope": _rope, "join": _join}[state["case"]["kind"]](state)


def work(case):
    e = _BYTES[case["dtype"]]
    if case["kind"] == "head":
        T, V, h = case["tokens"], case["vocab"], case["hidden"]
        rows = len(set(_items(_table(case))[0]))
        # three products of this size in a training step; a fourth makes the logits again, which are not kept
        return {"bytes": V * h * e + rows * h * e + 8 * T + (V * h * e + T * h * e if case["train"] else 0),
                "flops": (6 if case["train"] else 2) * rows * V * h}
    if case["kind"] == "rope":
        T, n = case["tokens"], case["q_heads"] + case["kv_heads"]
        ways = 4 if case["train"] else 2
        return {"bytes": ways * T * n * case["head_dim"] * e + 4 * T, "flops": ways // 2 * 3 * T * n * case["rotary"]}
    n, h = case["rows"], case["hidden"]
    gates = {"none": 0, "row": 0, "all": 1}[case["gate"]]
    # rows in and out; a training step reads X, B, dY, dS (and gates) and writes S, Y, dX, dB (and gates' gradients)
    rows = 8 + 2 * gates if case["train"] else 4 + gates
    return {"bytes": n * h * e * rows, "flops": n * h * (34 if case["train"] else 10)}


def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits."""
    s = prepare(case, seed)
    d = lambda t: t.to(torch.float64)
    if case["kind"] == "head":
        T = case["tokens"]
        x, w = d(s["X"]), d(s["W"])
        rows, target = s["rows"], s["ids"].long()[s["toks"]]
        some = torch.unique(rows)
        z = torch.mm(x[some], w.t())
        at = torch.searchsorted(some, rows)
        lse = torch.logsumexp(z, 1)
        row_lse = torch.zeros(T, dtype=torch.float64, device="cuda")
        row_lse[some] = lse
        gain = z[at, target] - lse[at]
        logp = torch.zeros(s["n"], dtype=torch.float64, device="cuda")
        logp.scatter_add_(0, s["which"], gain)
        out = {"row_lse": row_lse, "logp": logp}
        if case["train"]:
            z.sub_(lse[:, None]).exp_()
            weight = d(s["d"])[s["which"]]
            sums = torch.zeros(len(some), dtype=torch.float64, device="cuda").scatter_add_(0, at, weight)
            z.mul_(-sums[:, None])
            z.index_put_((at, target), weight, accumulate=True)
            out["dX"] = torch.zeros(T, case["hidden"], dtype=torch.float64, device="cuda")
            out["dX"][some] = torch.mm(z, w)
            out["dW"] = torch.mm(z.t(), x[some])
        return out
    if case["kind"] == "rope":
        n, c = case["rotary"], _amplitude(case)
        i = torch.arange(0, n, 2, dtype=torch.float64, device="cuda") / n
        base = math.log(_THETA)
        if case["scaling"] == "base" and n > 2:
            base += math.log(_FACTOR) * n / (n - 2)
        f = torch.exp(-i * base)
        if case["scaling"] == "linear":
            f = f * (1 / _FACTOR)
        if case["scaling"] == "parts":
            wave = 2 * math.pi / f
            r = torch.clip((_ORIGINAL / wave - _LOW) / (_HIGH - _LOW), 0, 1)
            f = f * (r + (1 - r) / _FACTOR)
        unit = torch.polar(torch.full((), c, dtype=torch.float64, device="cuda").expand(len(s["pos"]), n // 2), s["pos"].double()[:, None] * f)[:, None, :]

        def turned(t, by):
            x = d(t)
            pairs = x[..., :n].unflatten(-1, (2, n // 2)).transpose(-1, -2) if case["layout"] == "half" else x[..., :n].unflatten(-1, (n // 2, 2))
            y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by)
            y = y.transpose(-1, -2) if case["layout"] == "half" else y
            return torch.cat([y.flatten(-2), x[..., n:]], -1)

        out = {"Qr": turned(s["Q"], unit), "Kr": turned(s["K"], unit)}
        if case["train"]:
            out["dQ"], out["dK"] = turned(s["dQ"], unit.conj()), turned(s["dK"], unit.conj())
        return out
    h, x, b = case["hidden"], d(s["X"]), d(s["B"])
    one = torch.ones((), dtype=torch.float64, device="cuda")
    g = one if s["gate"] is None else d(s["gate"])
    wp = one if s["w_post"] is None else d(s["w_post"])
    k = one if s["w_post"] is None else ((b * b).sum(1, keepdim=True) / h + s["eps"]).rsqrt()
    total = s["res"] * x + g * wp * b * k
    held = d(total.to(s["X"].dtype))
    r = ((held * held).sum(1, keepdim=True) / h + s["eps"]).rsqrt()
    out = {"S": total, "Y": held * r * d(s["w_pre"])}
    if case["train"]:
        dy = d(s["dY"])
        a = dy * d(s["w_pre"])
        ds = d(s["dS"]) + r * a - held * r ** 3 * ((a * held).sum(1, keepdim=True) / h)
        out["dX"], out["dw_pre"] = s["res"] * ds, torch.sum(dy * held * r, 0)
        if s["gate"] is not None:
            out["dgate"] = ds * wp * b * k
            if s["gate"].dim() == 1:
                out["dgate"] = torch.sum(out["dgate"], 0)
        u = ds * g * wp
        if s["w_post"] is None:
            out["dB"] = u
        else:
            out["dw_post"] = torch.sum(ds * g * b * k, 0)
            out["dB"] = k * u - b * k ** 3 * ((u * b).sum(1, keepdim=True) / h)
    return out
