"""Vocabulary head, backward: vocabularies that are taken in several pieces, whose parts of dX add up."""
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import HALF, TINY

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24


def _whole_step(n, V, h, dtype, shift, d=0.5):
    """One prompt token and a response of n: what the two calls take and give."""
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    g = torch.Generator(device="cuda").manual_seed(n + V + h)

    def off_boundary(*shape, scale=1.0):
        buf = torch.empty(shape[0] * shape[1] + shift, dtype=dt, device="cuda")
        t = buf[shift:].view(shape)
        for at in range(0, shape[0], 1 << 22):
            t[at:at + (1 << 22)] = torch.randn((len(t[at:at + (1 << 22)]), shape[1]), generator=g, device="cuda") * scale
        return t

    X, W = off_boundary(n + 1, h), off_boundary(V, h, scale=h ** -0.5)
    ids = torch.randint(0, V, (n + 1,), generator=g, device="cuda", dtype=torch.int32)
    ids[1], ids[n] = 0, V - 1
    plan = ps.LogprobPlan([0], [1], [0, 1], [n], n + 1)
    lse, logp = ps.psattn_head_logprob_fwd(plan, X, W, ids)
    dX, dW = off_boundary(n + 1, h), off_boundary(V, h)
    dX.fill_(float("nan")), dW.fill_(float("nan"))
    ps.psattn_head_logprob_bwd(plan, X, W, ids, lse, torch.tensor([d], device="cuda"), dX=dX, dW=dW)
    return X, W, ids, d, lse[:n].double(), logp.item(), dX, dW


def _check(step, dtype, sums, dx_sums):
    """sums: additions in a chain of the sum of exponentials; dx_sums: of a sum of dX.  The reference takes a part of the vocabulary at a time, of
    which its own products have less than 2^31 elements."""
    X, W, ids, d, lse, logp, dX, dW = step
    n, (V, h), half = len(lse), W.shape, HALF[dtype]
    x, tok, at = X[:n].double(), ids[1:].long(), max(1, min(V, (1 << 27) // n))
    starts = range(0, V, at)
    ref = torch.logsumexp(torch.stack([torch.logsumexp(x @ W[v:v + at].double().T, 1) for v in starts]), 0)
    own = (x * W[tok].double()).sum(1)
    rlogp = (own - ref).sum().item()
    ez = (h + 2) * EPS32 * (x.abs().max(0)[0] @ W.abs().max(0)[0].double()).item()  # of a logit, at most
    e_lse = ez + sums * EPS32 + 8 * EPS32 * ref.abs().max().item()
    assert (lse - ref).abs().max().item() <= e_lse
    assert abs(logp - rlogp) <= n * (2 * e_lse) + (n + 2) * EPS32 * abs(rlogp)
    e = 1.01 * half + 2 * e_lse + 60 * EPS32  # of dz: its rounding, its logit, the log-sum-exp, the exponential
    rX, sX = torch.zeros_like(x), torch.zeros_like(x)
    for v in starts:
        w = W[v:v + at].double()
        G = (x @ w.T).sub_(ref[:, None]).exp_().mul_(-d)
        mine = (tok >= v) & (tok < v + at)
        G[mine.nonzero()[:, 0], tok[mine] - v] += d
        rX += G @ w
        rW = G.T.contiguous() @ x
        G.abs_()
        sX += G @ w.abs()
        off = (dW[v:v + at].double() - rW).abs() - (half * rW.abs() + (e + (n + 8) * EPS32) * (G.T.contiguous() @ x.abs()) + TINY)
        assert off.max().item() <= 0, ("dW", v + off.argmax().item() // h, off.max().item())
    off = (dX[:-1].double() - rX).abs() - (half * rX.abs() + (e + (dx_sums + 8) * EPS32) * sX + TINY)
    assert off.max().item() <= 0, ("dX", off.max().item())
    assert torch.isfinite(dX).all() and torch.isfinite(dW).all() and torch.all(dX[-1] == 0)


@pytest.mark.parametrize("n,V,dtype", [(1, 35_000_000, "bf16"), (63, 35_000_000, "bf16"), (2, 18_000_000, "f32"), (63, 18_000_000, "f32")])
def test_few_items_of_a_large_vocabulary(n, V, dtype):
    """Rows of dz as long as the vocabulary would reach over 4 GiB: as pieces they stay below 512 MiB, and over the same number of pieces the sums of
    exponentials are joined 128 columns at a time by 256 lanes, dX's in parts of at most 2^14."""
    _check(_whole_step(n, V, 8, dtype, 0), dtype, V // (128 * 256) + 160, 1 << 14)
