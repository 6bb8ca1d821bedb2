"""A decoder block's step as it is used: norm, projections, rotary positions, prefix-shared attention, gated norms around the feed-forward
block, the vocabulary head and the DPO loss, and all the way back; on other streams, and captured into a graph."""
import pytest
import torch

import paper_2410_20305_amd as ps

pytestmark = pytest.mark.gpu

T, HQ, HK, D, H, N, V = 190, 4, 2, 64, 128, 192, 331
OFF, P, RL = [4, 100], [30, 25], [20, 31, 17, 28]
SCALE, BETA, EPS, RES = 0.125, 0.3, 1e-5, 0.9


class Step:
    """One block between embedding rows and loss, fp32 so that torch's own functions may be held beside it."""

    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *s, k=1.0, at=0.0: torch.randn(*s, generator=g, device="cuda") * k + at
        self.p = dict(X=rn(T, H), w0=rn(H, k=0.2, at=1.0), Wqkv=rn((HQ + 2 * HK) * D, H, k=H ** -0.5), Wo=rn(H, HQ * D, k=0.06), w1=rn(H, k=0.2, at=1.0), g1=rn(H, k=0.3, at=0.5),
                      w2=rn(H, k=0.2, at=1.0), Wg=rn(N, H, k=0.09), Wu=rn(N, H, k=0.09), Wd=rn(H, N, k=0.07), w3=rn(H, k=0.2, at=1.0), g3=rn(T, H, k=0.3, at=0.5),
                      w4=rn(H, k=0.2, at=1.0), W=rn(V, H, k=0.1))
        self.ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        self.ref = rn(4, k=3.0, at=-100.0)
        self.meta = ps.psattn_build_meta(OFF, P, RL[0::2], RL[1::2], T)
        self.plan = ps.LogprobPlan(OFF, P, [0, 2, 4], RL, T)
        f = ps.psattn_rope_frequencies(32, 10000.0, "parts", factor=2.0, original_positions=64, low=1.0, high=8.0)
        self.freqs = torch.from_numpy(f).cuda()
        self.rope = ps.Rope(D, 10000.0, 128, rotary_dim=32, layout="interleaved", frequencies=f, amplitude=1.07)
        self.pos = torch.from_numpy(self.meta.positions()[0]).cuda()

    def library(self, stream=None):
        """Loss and the gradients of everything."""
        p, k = self.p, dict(stream=stream)
        mm = torch.matmul
        n0, _, _, r0 = ps.psattn_gatednorm_fwd(p["X"], None, p["w0"], eps=EPS, **k)
        qkv = mm(n0, p["Wqkv"].T).view(T, HQ + 2 * HK, D)
        q, kk = ps.psattn_rope_apply(self.rope, qkv[:, :HQ], qkv[:, HQ:HQ + HK], meta=self.meta, **k)
        v = qkv[:, HQ + HK:].contiguous()
        O, LSE = ps.psattn_fwd(self.meta, q, kk, v, SCALE, **k)
        b1 = mm(O.view(T, HQ * D), p["Wo"].T)
        n2, s1, rb1, rs1 = ps.psattn_gatednorm_fwd(p["X"], b1, p["w2"], w_post=p["w1"], gate=p["g1"], res_scale=RES, eps=EPS, **k)
        y, kept = ps.psattn_ffn_fwd(n2, p["Wg"], p["Wu"], p["Wd"], **k)
        n4, s3, rb3, rs3 = ps.psattn_gatednorm_fwd(s1, y, p["w4"], w_post=p["w3"], gate=p["g3"], res_scale=RES, eps=EPS, **k)
        lse, logp = ps.psattn_head_logprob_fwd(self.plan, n4, p["W"], self.ids, **k)
        loss, d = ps.psattn_dpo_loss(logp, self.ref, BETA, **k)
        g = {}
        dn4, g["W"] = ps.psattn_head_logprob_bwd(self.plan, n4, p["W"], self.ids, lse, d, **k)
        ds1, dy, g["w4"], g["w3"], g["g3"] = ps.psattn_gatednorm_bwd(y, s3, p["w4"], rb3, rs3, dn4, w_post=p["w3"], gate=p["g3"], res_scale=RES, **k)
        dn2, g["Wg"], g["Wu"], g["Wd"] = ps.psattn_ffn_bwd(n2, p["Wg"], p["Wu"], p["Wd"], kept, dy, **k)
        dx, db1, g["w2"], g["w1"], g["g1"] = ps.psattn_gatednorm_bwd(b1, s1, p["w2"], rb1, rs1, dn2, dS=ds1, w_post=p["w1"], gate=p["g1"], res_scale=RES, **k)
        g["Wo"] = mm(db1.T, O.view(T, HQ * D))
        dq, dk, dv = ps.psattn_bwd(self.meta, q, kk, v, O, mm(db1, p["Wo"]).view(T, HQ, D), LSE, SCALE, **k)
        dqkv = torch.empty_like(qkv)
        ps.psattn_rope_apply_bwd(self.rope, dq, dk, meta=self.meta, dQ=dqkv[:, :HQ], dK=dqkv[:, HQ:HQ + HK], **k)
        dqkv[:, HQ + HK:] = dv
        dqkv = dqkv.view(T, -1)
        g["Wqkv"] = mm(dqkv.T, n0)
        g["X"], _, g["w0"], _, _ = ps.psattn_gatednorm_bwd(None, p["X"], p["w0"], None, r0, mm(dqkv, p["Wqkv"]), dS=dx, **k)
        return loss, g

    def plain(self):
        """The same from torch's functions with autograd, in 64 bits."""
        p = {k: v.double().requires_grad_() for k, v in self.p.items()}
        rms = lambda x, w: x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * w
        turn = self.pos.double()[:, None, None] * self.freqs
        by = torch.polar(torch.full_like(turn, 1.07), turn)

        def rope(x):
            z = torch.view_as_complex(x[..., :32].reshape(T, -1, 16, 2)) * by
            return torch.cat([torch.view_as_real(z).flatten(-2), x[..., 32:]], -1)

        qkv = (rms(p["X"], p["w0"]) @ p["Wqkv"].T).view(T, HQ + 2 * HK, D)
        q, k, v = rope(qkv[:, :HQ]), rope(qkv[:, HQ:HQ + HK]), qkv[:, HQ + HK:]
        t = torch.arange(T, device="cuda")
        ok = torch.zeros(T, T, dtype=torch.bool, device="cuda")
        for i, o in enumerate(OFF):
            c, r = o + P[i], o + P[i] + RL[2 * i]
            end = r + RL[2 * i + 1]
            a, b = t[:, None], t[None, :]
            ok |= (a >= o) & (a < end) & (b >= o) & (b <= a) & ~((a >= r) & (b >= c) & (b < r))
        k, v = (x.repeat_interleave(HQ // HK, 1) for x in (k, v))
        s = (q.transpose(0, 1) @ k.permute(1, 2, 0)) * SCALE
        w = torch.softmax(torch.where(ok, s, torch.full_like(s, -1e300)), -1) * ok.any(1)[:, None]
        O = (w @ v.transpose(0, 1)).transpose(0, 1).reshape(T, HQ * D)
        s1 = RES * p["X"] + p["g1"] * rms(O @ p["Wo"].T, p["w1"])
        n2 = rms(s1, p["w2"])
        y = (torch.nn.functional.silu(n2 @ p["Wg"].T) * (n2 @ p["Wu"].T)) @ p["Wd"].T
        n4 = rms(RES * s1 + p["g3"] * rms(y, p["w3"]), p["w4"])
        lp = torch.log_softmax(n4 @ p["W"].T, 1)
        per = []
        for i, o in enumerate(OFF):
            at = o + P[i]
            for n in RL[2 * i:2 * i + 2]:
                rows = [o + P[i] - 1] + list(range(at, at + n - 1))
                per.append(lp[rows, self.ids[at:at + n].long()].sum())
                at += n
        z = torch.stack(per) - self.ref.double()
        loss = -torch.nn.functional.logsigmoid(BETA * (z[0::2] - z[1::2]))
        loss.sum().backward()
        return loss.detach(), {k: v.grad for k, v in p.items()}


def test_against_torch():
    """fp32 throughout: a chain of some twenty operators, each off by some 2^-24 of sums of up to 331 terms, on values that pass through
    norms; 1e-4 of a tensor's norm leaves room for them and for nothing that is a different formula."""
    s = Step()
    loss, g = s.library()
    want, wg = s.plain()
    assert ((loss.double() - want).abs() <= 1e-4 * (1 + want.abs())).all(), (loss, want)
    assert set(g) == set(wg)
    for k in g:
        off = (g[k].double().reshape(-1) - wg[k].reshape(-1)).norm() / wg[k].norm()
        assert off <= 1e-4, (k, off.item())


def _flat(out):
    return [out[0]] + [out[1][k] for k in sorted(out[1])]


def test_on_another_stream():
    s = Step(1)
    want = [t.clone() for t in _flat(s.library())]
    side = torch.cuda.Stream()
    for turn in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = _flat(s.library())
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(want, got)), turn


def _calls(s, stream=None):
    """The new calls by themselves: products of torch's have a stream of their own choice."""
    p, k = s.p, dict(stream=stream)
    x, b = p["X"], p["g3"]
    y, S, rb, rs = ps.psattn_gatednorm_fwd(x, b, p["w2"], w_post=p["w1"], gate=p["g1"], **k)
    out = [y, S, rb, rs, *ps.psattn_gatednorm_bwd(b, S, p["w2"], rb, rs, y, dS=x, w_post=p["w1"], gate=p["g1"], **k)]
    y, S, rb, rs = ps.psattn_gatednorm_fwd(x, b, p["w2"], w_post=p["w1"], gate=x, **k)
    out += [y, *ps.psattn_gatednorm_bwd(b, S, p["w2"], rb, rs, y, w_post=p["w1"], gate=x, **k)]
    q, kk = ps.psattn_rope_apply(s.rope, x.view(T, 2, D), b.view(T, 2, D), meta=s.meta, **k)
    out += [q, kk, *ps.psattn_rope_apply_bwd(s.rope, q, kk, positions=s.pos, **k)]
    lse, logp = ps.psattn_head_logprob_fwd(s.plan, x, p["W"], s.ids, **k)
    return out + [lse, logp, *ps.psattn_head_logprob_bwd(s.plan, x, p["W"], s.ids, lse, logp, **k)]


@pytest.mark.parametrize("as_handle", [False, True])
def test_memory_that_the_current_stream_has_freed(as_handle):
    """A call on another stream makes what it needs there, not from memory that the current stream has freed and still works on."""
    s = Step(2)
    want = [t.clone() for t in _calls(s)]
    side = torch.cuda.Stream()
    for turn in range(3):
        side.wait_stream(torch.cuda.current_stream())
        used = [torch.empty_like(t) for t in want]
        for _ in range(20):
            for t in used:
                t.fill_(float("nan"))
        del t, used
        got = _calls(s, side.cuda_stream if as_handle else side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(want, got)), turn
        del got
    torch.cuda.synchronize()


def test_two_graphs_replayed_in_turn():
    """Two captures with workspaces of their own, replayed with eager calls between; every replay as the eager calls."""
    steps = [Step(3), Step(4)]
    for s in steps:
        _calls(s)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_calls(s))
        graphs.append(g)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for turn in range(3):
        for s in steps:
            s.p["X"].copy_(torch.randn(T, H, generator=gen, device="cuda"))
            s.p["W"].copy_(torch.randn(V, H, generator=gen, device="cuda") * 0.1)
        want = [[t.clone() for t in _calls(s)] for s in steps]
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for w, o in zip(want, outs):
            assert all(torch.equal(a, b) for a, b in zip(w, o)), turn


def test_workspaces_of_any_contents_and_exact_size():
    s = Step(5)
    p = s.p
    want = _calls(s)
    lib = ps.load_library()
    y, S, rb, rs = want[:4]
    for fill in (0, 255):
        for shift in (0, 1, 64):
            ws = lambda n: torch.full((n + shift,), fill, dtype=torch.uint8, device="cuda")[shift:]
            got = ps.psattn_gatednorm_bwd(p["g3"], S, p["w2"], rb, rs, y, dS=p["X"], w_post=p["w1"], gate=p["g1"], workspace=ws(lib.psattn_gatednorm_bwd_workspace_bytes(T, H)))
            assert all(torch.equal(a, b) for a, b in zip(got, want[4:9]))
            lse, logp = ps.psattn_head_logprob_fwd(s.plan, p["X"], p["W"], s.ids, workspace=ws(lib.psattn_head_logprob_fwd_workspace_bytes(s.plan.handle, 0, V, H)))
            assert torch.equal(lse, want[-4]) and torch.equal(logp, want[-3])
            got = ps.psattn_head_logprob_bwd(s.plan, p["X"], p["W"], s.ids, lse, logp, workspace=ws(lib.psattn_head_logprob_bwd_workspace_bytes(s.plan.handle, 0, V, H)))
            assert torch.equal(got[0], want[-2]) and torch.equal(got[1], want[-1])
    with pytest.raises(ps.PsattnError):
        ps.psattn_head_logprob_fwd(s.plan, p["X"], p["W"], s.ids, workspace=ws(64))
