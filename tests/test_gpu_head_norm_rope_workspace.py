"""Workspaces of the vocabulary head and the gated norms: of exactly the bytes that are asked for, of any contents, with nothing written
behind them, at sizes on either side of each way that a call may take."""
import pytest
import torch

import paper_2410_20305_amd as ps

pytestmark = pytest.mark.gpu

LIB = ps.load_library()
CODE = {torch.float32: 0, torch.bfloat16: 1}


class Room:
    """A workspace between guards."""

    def __init__(self, n, fill, shift=0):
        self.buf = torch.full((n + 1024,), 0x5A, dtype=torch.uint8, device="cuda")
        self.at, self.n = 512 + shift, n
        self.view = self.buf[self.at:self.at + n]
        self.view.fill_(fill)

    def check(self):
        torch.cuda.synchronize()
        assert torch.all(self.buf[:self.at] == 0x5A) and torch.all(self.buf[self.at + self.n:] == 0x5A), "written outside the workspace"


# tokens of one response, vocabulary, hidden: few items and many, logits in parts of k or not, dz twice, both products of dz in one launch
HEADS = [(2, 130, 4096), (2, 40000, 64), (33, 300, 2048), (34, 300, 2048), (60, 513, 72), (66, 513, 72), (70, 1000, 4100), (258, 1000, 520), (259, 1000, 520), (300, 33000, 65),
         (1030, 700, 136), (1030, 300, 1001), (2000, 129, 33)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V,h", HEADS)
def test_head(T, V, h, dtype):
    g = torch.Generator(device="cuda").manual_seed(T + V + h)
    plan = ps.LogprobPlan([0], [1], [0, 1], [T - 1], T)
    X, W = torch.randn(T, h, generator=g, device="cuda").to(dtype), (torch.randn(V, h, generator=g, device="cuda") * h ** -0.5).to(dtype)
    ids, d = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32), torch.ones(1, device="cuda")
    want = None
    for fill, shift in ((0, 0), (255, 16), (127, 3)):
        a = Room(LIB.psattn_head_logprob_fwd_workspace_bytes(plan.handle, CODE[dtype], V, h), fill, shift)
        b = Room(LIB.psattn_head_logprob_bwd_workspace_bytes(plan.handle, CODE[dtype], V, h), fill, shift)
        lse, logp = ps.psattn_head_logprob_fwd(plan, X, W, ids, workspace=a.view)
        got = [lse, logp, *ps.psattn_head_logprob_bwd(plan, X, W, ids, lse, d, workspace=b.view)]
        a.check()
        b.check()
        assert all(bool(torch.isfinite(t).all()) for t in got)
        want = want or got
        assert all(torch.equal(x, y) for x, y in zip(want, got)), (fill, shift)
    with pytest.raises(ps.PsattnError):
        ps.psattn_head_logprob_fwd(plan, X, W, ids, workspace=a.view[1:])
    with pytest.raises(ps.PsattnError):
        ps.psattn_head_logprob_bwd(plan, X, W, ids, lse, d, workspace=b.view[1:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,h", [(1, 1), (3, 64), (600, 130), (700, 2048), (513, 4096), (300, 8192), (9, 8193), (300, 9000), (40, 16384), (2500, 16392), (600, 40000), (27000, 72)])
def test_gatednorm(n, h, dtype):
    g = torch.Generator(device="cuda").manual_seed(n + h)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)
    X, B, dY, w = rn(n, h), rn(n, h), rn(n, h), rn(h)
    for gate in (rn(h), rn(n, h)):
        Y, S, rb, rs = ps.psattn_gatednorm_fwd(X, B, w, w_post=w, gate=gate)
        want = None
        for fill, shift in ((0, 0), (255, 16), (127, 3)):
            room = Room(LIB.psattn_gatednorm_bwd_workspace_bytes(n, h), fill, shift)
            got = ps.psattn_gatednorm_bwd(B, S, w, rb, rs, dY, dS=X, w_post=w, gate=gate, workspace=room.view)
            room.check()
            assert all(bool(torch.isfinite(t).all()) for t in got)
            want = want or got
            assert all(torch.equal(x, y) for x, y in zip(want, got)), (fill, shift)
        with pytest.raises(ps.PsattnError):
            ps.psattn_gatednorm_bwd(B, S, w, rb, rs, dY, w_post=w, gate=gate, workspace=room.view[1:])
