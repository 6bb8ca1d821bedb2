"""Vocabulary head: vocabularies that the backward takes in several pieces, whose parts of dX add up, and tensors of 2^31 elements and more."""
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import HALF, TINY

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24


def _whole_step(n, V, h, dtype, shift, d=0.5, prompt=1):
    """A prompt and a response of n: what the two calls take and give."""
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    g = torch.Generator(device="cuda").manual_seed(n + V + h)

    def off_boundary(*shape, scale=1.0):
        buf = torch.empty(shape[0] * shape[1] + shift, dtype=dt, device="cuda")
        t = buf[shift:].view(shape)
        for at in range(0, shape[0], 1 << 22):
            t[at:at + (1 << 22)] = torch.randn((len(t[at:at + (1 << 22)]), shape[1]), generator=g, device="cuda") * scale
        return t

    T = n + prompt
    X, W = off_boundary(T, h), off_boundary(V, h, scale=h ** -0.5)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    ids[prompt], ids[T - 1] = 0, V - 1
    plan = ps.LogprobPlan([0], [prompt], [0, 1], [n], T)
    lse, logp = ps.psattn_head_logprob_fwd(plan, X, W, ids)
    dX, dW = off_boundary(T, h), off_boundary(V, h)
    dX.fill_(float("nan")), dW.fill_(float("nan"))
    ps.psattn_head_logprob_bwd(plan, X, W, ids, lse, torch.tensor([d], device="cuda"), dX=dX, dW=dW)
    assert torch.all(dX[:prompt - 1] == 0) and torch.all(dX[-1] == 0)
    rows = slice(prompt - 1, T - 1)
    return X[rows], W, ids[prompt:], d, lse[rows].double(), logp.item(), dX[rows], dW


def _check(step, dtype, sums, dx_sums):
    """sums: additions in a chain of the sum of exponentials; dx_sums: of a sum of dX.  The reference takes a part of the vocabulary at a time, of
    which its own products have less than 2^31 elements."""
    X, W, ids, d, lse, logp, dX, dW = step
    n, (V, h), half = len(lse), W.shape, HALF[dtype]
    x, tok, at = X.double(), ids.long(), max(1, min(V, (1 << 27) // max(n, h)))
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
    off = (dX.double() - rX).abs() - (half * rX.abs() + (e + (dx_sums + 8) * EPS32) * sX + TINY)
    assert off.max().item() <= 0, ("dX", off.max().item())
    assert torch.isfinite(dX).all() and torch.isfinite(dW).all()


@pytest.mark.parametrize("n,V,dtype", [(1, 35_000_000, "bf16"), (63, 35_000_000, "bf16"), (2, 18_000_000, "f32"), (63, 18_000_000, "f32")])
def test_few_items_of_a_large_vocabulary(n, V, dtype):
    """Rows of dz as long as the vocabulary would reach over 4 GiB: as pieces they stay below 512 MiB, and over the same number of pieces the sums of
    exponentials are joined 128 columns at a time by 256 lanes, dX's in parts of at most 2^14."""
    _check(_whole_step(n, V, 8, dtype, 0), dtype, V // (128 * 256) + 160, 1 << 14)


@pytest.mark.parametrize("n,V,h,dtype,shift", [(6001, 30001, 33, "f32", 0), (6001, 30001, 36, "f32", 1), (6001, 30000, 64, "f32", 0), (6001, 60003, 65, "bf16", 0), (6001, 60003, 64, "bf16", 1),
                                               (6001, 60001, 64, "bf16", 0), (60000, 10001, 64, "bf16", 0), (60000, 10001, 41, "bf16", 1), (40000, 5003, 40, "f32", 0)])
def test_parts_of_dx_add_up(n, V, h, dtype, shift):
    """Both types, joint and separate products, whole rows and others, and dW in parts of the items: two and more pieces, the last one smaller"""
    assert n * V * {"bf16": 2, "f32": 4}[dtype] > 512 << 20
    _check(_whole_step(n, V, h, dtype, shift), dtype, V // 64 + 100, V + 70)


def test_tensors_of_more_than_2_31_elements():
    """A short response far into X, and tokens up to the end of W"""
    V, h, prompt = 264000, 8200, 264000
    assert V * h > 1 << 31 and prompt * h > 1 << 31
    _check(_whole_step(40, V, h, "bf16", 0, prompt=prompt), "bf16", V // 64 + 100, 1 << 14)
