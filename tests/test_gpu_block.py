"""Embedding, layer norm, attention, feed-forward block and loss head together: one block of a model through a DPO step on
packed prefix-shared samples, against the same model in torch, fp64, with autograd; the step captured into a graph; the
step on a stream of its own."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import rnd
from oracle import psattn_oracle as orc

pytestmark = pytest.mark.gpu

OFF, PRE, PTR, RESP, T = [2, 190], [60, 90], [0, 2, 4], [40, 55, 33, 70], 400
HEADS, HIDDEN, INNER, VOCAB, SCALE, EPS, BETA = 2, 256, 520, 200, 1.0 / np.sqrt(128.0), 1e-5, 0.1


def _data():
    rng = np.random.default_rng(77)
    real = np.zeros(T, dtype=bool)
    for o, p, i in zip(OFF, PRE, range(2)):
        real[o:o + p + sum(RESP[PTR[i]:PTR[i + 1]])] = True
    ids = np.where(real, rng.integers(0, VOCAB, T), -1).astype(np.int32)
    w = dict(E=rnd(rng, VOCAB, HIDDEN, scale=0.06), Wg=rnd(rng, INNER, HIDDEN, scale=HIDDEN ** -0.5), Wu=rnd(rng, INNER, HIDDEN, scale=HIDDEN ** -0.5),
             Wd=rnd(rng, HIDDEN, INNER, scale=INNER ** -0.5), head=rnd(rng, VOCAB, HIDDEN, scale=HIDDEN ** -0.5))
    for k in "123":
        w["w" + k], w["b" + k] = rnd(rng, HIDDEN, scale=0.2, shift=1.0), rnd(rng, HIDDEN, scale=0.2)
    return ids, real, w, rng.standard_normal(4) * 3 - 200.0


class Step:
    """The step on given buffers; nothing is allocated but by the calls themselves."""

    def __init__(self):
        ids, _, w, lref = _data()
        self.ids = torch.from_numpy(ids).cuda()
        self.w = {k: torch.from_numpy(v).to(torch.bfloat16).cuda() for k, v in w.items()}
        self.lref = torch.from_numpy(lref).float().cuda()
        self.meta = ps.psattn_build_meta_multi(OFF, PRE, PTR, RESP, T)
        self.plan = ps.LogprobPlan(OFF, PRE, PTR, RESP, T)
        # padding's logits rows predict nothing, but row_lse keeps their places: zeros
        self.row_lse = torch.zeros(T, device="cuda")

    def __call__(self):
        w, heads = self.w, lambda t: t.view(T, HEADS, 128)
        X0 = ps.psattn_embed_fwd(self.ids, w["E"], scale=16.0)
        A, _, m1, r1 = ps.psattn_layernorm_fwd(X0, w["w1"], w["b1"], EPS)
        O, LSE = ps.psattn_fwd(self.meta, heads(A), heads(A), heads(A), SCALE)
        N2, S1, m2, r2 = ps.psattn_layernorm_fwd(O.view(T, HIDDEN), w["w2"], w["b2"], EPS, residual=X0)
        F, kept = ps.psattn_ffn_fwd(N2, w["Wg"], w["Wu"], w["Wd"])
        N3, S2, m3, r3 = ps.psattn_layernorm_fwd(F, w["w3"], w["b3"], EPS, residual=S1)
        logits = N3 @ w["head"].T
        _, logp = ps.psattn_logprob_fwd(self.plan, logits, self.ids, row_lse=self.row_lse)
        loss, dlogp = ps.psattn_dpo_loss(logp, self.lref, BETA)
        dlogits = ps.psattn_logprob_bwd(self.plan, logits, self.ids, self.row_lse, dlogp)
        g = dict(head=dlogits.T @ N3)
        dS2, g["w3"], g["b3"] = ps.psattn_layernorm_bwd(S2, w["w3"], m3, r3, dlogits @ w["head"])
        dN2, g["Wg"], g["Wu"], g["Wd"] = ps.psattn_ffn_bwd(N2, w["Wg"], w["Wu"], w["Wd"], kept, dS2)
        dS1, g["w2"], g["b2"] = ps.psattn_layernorm_bwd(S1, w["w2"], m2, r2, dN2, dS=dS2)
        dQ, dK, dV = ps.psattn_bwd(self.meta, heads(A), heads(A), heads(A), O, heads(dS1), LSE, SCALE)
        dA = (dQ.float() + dK.float() + dV.float()).to(torch.bfloat16).view(T, HIDDEN)
        dX0, g["w1"], g["b1"] = ps.psattn_layernorm_bwd(X0, w["w1"], m1, r1, dA, dS=dS1)
        g["E"] = ps.psattn_embed_bwd(self.ids, dX0, VOCAB, scale=16.0)
        return loss, logp, g


def _reference():
    ids, real, w, lref = _data()
    w = {k: torch.from_numpy(v).requires_grad_(True) for k, v in w.items()}
    D, B = orc.branch_arrays(OFF, PRE, PTR, RESP, T)
    mask = torch.from_numpy(np.asarray(orc.dense_branch_mask(D, B))).bool()
    norm = lambda x, k: torch.nn.functional.layer_norm(x, (HIDDEN,), w["w" + k], w["b" + k], EPS)
    tid = torch.from_numpy(np.where(real, ids, 0)).long()
    X0 = torch.where(torch.from_numpy(real)[:, None], w["E"][tid] * 16.0, 0.0)
    A = norm(X0, "1")
    q = A.view(T, HEADS, 128).transpose(0, 1)
    s = (q @ q.transpose(1, 2)) * SCALE
    some = mask.any(1)
    p = torch.softmax(torch.where(mask | ~some[:, None], s, -torch.inf), -1) * some[:, None]
    S1 = (p @ q).transpose(0, 1).reshape(T, HIDDEN) + X0
    N2 = norm(S1, "2")
    S2 = (torch.nn.functional.silu(N2 @ w["Wg"].T) * (N2 @ w["Wu"].T)) @ w["Wd"].T + S1
    lp = torch.log_softmax(norm(S2, "3") @ w["head"].T, -1)
    logp = []
    for i, (o, n) in enumerate(zip(OFF, PRE)):
        at = o + n
        for j in range(PTR[i], PTR[i + 1]):
            rows = [o + n - 1] + list(range(at, at + RESP[j] - 1))
            logp.append(lp[rows, tid[at:at + RESP[j]]].sum())
            at += RESP[j]
    logp = torch.stack(logp)
    d = logp - torch.from_numpy(lref)
    loss = torch.nn.functional.softplus(-BETA * (d[0::2] - d[1::2]))
    loss.sum().backward()
    return loss.detach(), logp.detach(), {k: v.grad for k, v in w.items()}


def test_step_against_torch():
    """Some 22 tensors on the longest way to a gradient are rounded to bf16, each off by at most 2^-8 / sqrt(3) of its norm:
    0.011 where they add up like independent ones; the attention's own gradients are within 0.02 (relative L2)."""
    loss, logp, grads = Step()()
    rloss, rlogp, rgrads = _reference()
    bar = 0.02 + 2.0 ** -8 / np.sqrt(3.0) * np.sqrt(22.0)
    rel = lambda a, b: ((a.double().cpu() - b).norm() / b.norm()).item()
    assert rel(logp, rlogp) <= bar and rel(loss, rloss) <= bar
    assert set(grads) == set(rgrads)
    for k in grads:
        assert torch.isfinite(grads[k].float()).all(), k
        assert rel(grads[k], rgrads[k]) <= bar, (k, rel(grads[k], rgrads[k]))


def _flat(out):
    return [out[0], out[1], *(out[2][k] for k in sorted(out[2]))]


def test_step_on_another_stream():
    step = Step()
    want = [t.clone() for t in _flat(step())]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _flat(step())
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def _block_only(d):
    """The three operators, forward and backward, on d's tensors."""
    X = ps.psattn_embed_fwd(d["ids"], d["E"], scale=16.0)
    Y, S, mean, rstd = ps.psattn_layernorm_fwd(X, d["w"], d["b"], residual=d["R"])
    F, kept = ps.psattn_ffn_fwd(Y, d["Wg"], d["Wu"], d["Wd"], act="gelu")
    dY, *dW = ps.psattn_ffn_bwd(Y, d["Wg"], d["Wu"], d["Wd"], kept, d["dF"], act="gelu")
    dX, dw, db = ps.psattn_layernorm_bwd(S, d["w"], mean, rstd, dY, dS=d["dF"])
    return [F, S, *dW, dX, dw, db, ps.psattn_embed_bwd(d["ids"], dX, VOCAB, scale=16.0)]


@pytest.mark.parametrize("tokens,dtype", [(1, torch.bfloat16), (70, torch.float32), (333, torch.bfloat16), (1100, torch.bfloat16)])
def test_captured_and_replayed(tokens, dtype):
    """Two graphs of one pass each, replayed in turn with new inputs and with eager passes between: every replay as the eager pass."""
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    rn = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)
    d = dict(ids=torch.zeros(tokens, dtype=torch.int32, device="cuda"), E=rn(VOCAB, HIDDEN), w=rn(HIDDEN), b=rn(HIDDEN), R=rn(tokens, HIDDEN),
             Wg=rn(INNER, HIDDEN), Wu=rn(INNER, HIDDEN), Wd=rn(HIDDEN, INNER), dF=rn(tokens, HIDDEN))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _block_only(d)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = _block_only(d)
        graphs.append((g, out))
    for turn in range(4):
        d["ids"].copy_(torch.randint(-1, VOCAB, (tokens,), generator=gen, device="cuda", dtype=torch.int32))
        d["R"].copy_(rn(tokens, HIDDEN))
        want = [t.clone() for t in _block_only(d)]
        torch.cuda.synchronize()
        g, out = graphs[turn % 2]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), turn


def test_two_calls_at_once():
    """Two streams, each with its own workspaces, at the same time: as one after the other."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    rn = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    sets = [dict(ids=torch.randint(-1, VOCAB, (n,), generator=gen, device="cuda", dtype=torch.int32), E=rn(VOCAB, HIDDEN), w=rn(HIDDEN), b=rn(HIDDEN),
                 R=rn(n, HIDDEN), Wg=rn(INNER, HIDDEN), Wu=rn(INNER, HIDDEN), Wd=rn(HIDDEN, INNER), dF=rn(n, HIDDEN)) for n in (600, 37)]
    want = [[t.clone() for t in _block_only(d)] for d in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for d, s in zip(sets, streams):
            with torch.cuda.stream(s):
                got.append(_block_only(d))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(want[i % 2], out)), i


def test_stream_argument():
    """A stream that is not the current one, as an object and as a handle; workspaces that the calls take for themselves live on."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    rn = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    X, W, Wd, w = rn(300, HIDDEN), rn(INNER, HIDDEN), rn(HIDDEN, INNER), rn(HIDDEN)
    ids = torch.randint(0, VOCAB, (300,), generator=gen, device="cuda", dtype=torch.int32)

    def run(stream):
        Y, kept = ps.psattn_ffn_fwd(X, W, W, Wd, stream=stream)
        Y0, _ = ps.psattn_ffn_fwd(X, W, W, Wd, keep=False, stream=stream)
        grads = ps.psattn_ffn_bwd(X, W, W, Wd, kept, Y, stream=stream)
        N, S, mean, rstd = ps.psattn_layernorm_fwd(X, w, w, residual=X, stream=stream)
        ln = ps.psattn_layernorm_bwd(S, w, mean, rstd, X, stream=stream)
        return [Y, Y0, *grads, N, *ln, ps.psattn_embed_fwd(ids, W[:VOCAB], stream=stream), ps.psattn_embed_bwd(ids, X, VOCAB, stream=stream)]

    want = run(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for s in (side, side.cuda_stream):
        got = run(s)
        junk = [torch.full((1 << 18,), float("nan"), device="cuda") for _ in range(8)]  # may take freed memory on the current stream
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        del junk
