"""Vocabulary head, bf16: a frequent token's row of dW, whose two parts, what the items of that token add and what all others take away,
nearly cancel.  It is as exact as its own rounding: neither part is rounded by itself."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import HALF, TINY, Guarded, close, np64, rnd
from oracle import psattn_block_oracle as blk
from oracle import psattn_oracle as orc

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24
MEAN = 2.0  # of all columns of X but the first


def _calibrated(n, V, h, token, most, seed=0):
    """n items, each row of which gives `token` a probability of up to `most`, and that many of them are followed by it as their
    probabilities add up to.  Column 0 of X and W is that token's logit; the others' share of the logits is small."""
    rng = np.random.default_rng(n * 7 + V + h + seed)
    p = rng.uniform(0, most, n)
    X = rnd(rng, n + 1, h, shift=MEAN, dtype="bf16")
    X[:n, 0] = np.log(np.maximum(p, 1e-3) / (1 - p) * (V - 1))
    W = rnd(rng, V, h, scale=0.01 / h ** 0.5, dtype="bf16")
    W[:, 0] = 0
    W[token, 0] = 1
    X = torch.from_numpy(X).bfloat16().double().numpy()
    P = np.exp(X[:n] @ W.T)
    P /= P.sum(1, keepdims=True)
    ids = rng.integers(0, V - 1, n + 1)
    ids += ids >= token
    ids[1 + rng.choice(n, int(round(P[:, token].sum())), replace=False)] = token
    return X, W, ids


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("n,V,h,most", [(40, 300, 64, 0.8), (130, 513, 72, 0.5), (256, 200, 128, 0.5), (300, 520, 264, 0.4), (700, 1000, 101, 0.3), (1100, 1500, 256, 0.2),
                                        (1500, 260, 1003, 0.2), (2900, 300, 64, 0.2), (2900, 3000, 64, 0.2)])
def test_parts_that_cancel(n, V, h, most, shift):
    """dz away from the items' own tokens is rounded to bf16 once, from fp32: the reference has it rounded too, and where the kernel's dz,
    off by what fp32 loses, may round to the other side, a step of it is allowed.  Then the fp32 sum's roundings and the result's one.  What
    the others take away goes through two numbers of bf16, the second what the first one's rounding leaves: 2^-8 of 2^-8 of it is lost."""
    token, d = 17, 0.0371
    X, W, ids = _calibrated(n, V, h, token, most)
    plan = ps.LogprobPlan([0], [1], [0, 1], [n], n + 1)
    dev = Guarded("bf16", shift)
    tX, tW, tid = dev.put(X), dev.put(W), dev.put(ids.astype(np.int32), dtype=torch.int32)
    lse, _ = ps.psattn_head_logprob_fwd(plan, tX, tW, tid)
    d = float(torch.tensor(d))
    _, dW = ps.psattn_head_logprob_bwd(plan, tX, tW, tid, lse, torch.tensor([d], device="cuda"), dX=dev.empty(n + 1, h), dW=dev.empty(V, h))
    dev.check()
    x, own = X[:n], ids[1:] == token
    Z = x @ W.T
    ref = np.log(np.exp(Z - Z.max(1, keepdims=True)).sum(1)) + Z.max(1)
    ez = (h + 2) * EPS32 * (np.abs(x) @ np.abs(W.T))
    P, far = np.exp(Z - ref[:, None]), np.abs(Z - ref[:, None])
    e_lse = (P * (ez + EPS32 * (2 * far + 8))).sum(1) + ez.max(1) * 1e-3 + (V / 64 + 100) * EPS32 + 4 * EPS32 * np.abs(ref)
    p = P[:, token]
    dz = d * (own - p)
    e = d * (p * (ez[:, token] + e_lse + EPS32 * (2 * far[:, token] + 8)) + 2 * EPS32 * own) + 2 * EPS32 * np.abs(dz) + TINY
    bf = lambda a: torch.from_numpy(a).bfloat16().double().numpy()
    held = np.where(own, dz, bf(dz))
    off = np.where(own, e, np.abs(bf(dz - e) - bf(dz)) + np.abs(bf(dz + e) - bf(dz)))
    want, size = held @ x, np.abs(held) @ np.abs(x)
    others = np.where(own, 0, held) @ x
    tol = HALF["bf16"] * np.abs(want) + (1 + HALF["bf16"]) * (off @ np.abs(x) + (n + 4) * EPS32 * size + HALF["bf16"] ** 2 * np.abs(others)) + TINY
    close(dW[token].float().cpu().numpy().astype(np.float64), want, tol, "the frequent token's row")
    # the bound tells a part rounded by itself from a sum rounded once
    assert np.any(np.abs(bf(bf(others) + np.where(own, held, 0) @ x) - want) > 1.5 * tol)
    # and every row as before
    items = orc.prediction_items([0], [1], [0, 1], [n])
    _, rW, G = blk.head_grad(X, W, ids, items, np.array([d]))
    aG = np.abs(G[:n])
    close(dW, rW, HALF["bf16"] * np.abs(rW) + 1.01 * ((HALF["bf16"] + 4 * ez.max() + (V / 64 + 200) * EPS32 + (n + 4) * EPS32) * (aG.T @ np.abs(x))) + TINY, "dW")


def test_a_result_does_not_depend_on_who_comes_first():
    """Many items of few tokens, in three calls with other contents of the workspace: the same bits."""
    n, V, h = 1500, 40, 200
    X, W, ids = _calibrated(n, V, h, 3, 0.3)
    plan = ps.LogprobPlan([0], [1], [0, 1], [n], n + 1)
    tX, tW, tid = torch.from_numpy(X).bfloat16().cuda(), torch.from_numpy(W).bfloat16().cuda(), torch.from_numpy(ids.astype(np.int32)).cuda()
    lse, _ = ps.psattn_head_logprob_fwd(plan, tX, tW, tid)
    d = torch.tensor([0.25], device="cuda")
    bytes_ = ps.load_library().psattn_head_logprob_bwd_workspace_bytes(plan.handle, 1, V, h)
    got = []
    for fill in (0, 255, 1, 0):
        ws = torch.full((bytes_,), fill, dtype=torch.uint8, device="cuda")
        got.append(ps.psattn_head_logprob_bwd(plan, tX, tW, tid, lse, d, workspace=ws))
    for g in got[1:]:
        assert torch.equal(g[0], got[0][0]) and torch.equal(g[1], got[0][1])


@pytest.mark.parametrize("n,V,h", [(40, 300, 64), (300, 520, 72), (1100, 300, 64)])
def test_sums_beyond_the_range_of_bf16(n, V, h):
    """A column of X that holds the largest numbers, a token that many rows find probable and one row is followed by: what the others take away is
    beyond fp32, the one row's part within it, so dW is infinite there, not NaN, and the other columns are as they are without it."""
    X, W, ids = _calibrated(n, V, h, 17, 0.5)
    W[:, 5] = 0
    ids[ids == 17] = 18
    ids[n // 2] = 17
    plan = ps.LogprobPlan([0], [1], [0, 1], [n], n + 1)
    tW, tid, d = torch.from_numpy(W).bfloat16().cuda(), torch.from_numpy(ids.astype(np.int32)).cuda(), torch.tensor([1.0], device="cuda")
    got = []
    for top in (0.0, 3e38):
        X[:, 5] = top
        tX = torch.from_numpy(X).bfloat16().cuda()
        lse, _ = ps.psattn_head_logprob_fwd(plan, tX, tW, tid)
        got.append(ps.psattn_head_logprob_bwd(plan, tX, tW, tid, lse, d))
    (dX, dW), (dX2, dW2) = got
    assert torch.equal(dX, dX2)
    keep = torch.arange(h, device="cuda") != 5
    assert torch.equal(dW[:, keep], dW2[:, keep])
    assert dW2[17, 5] == -float("inf")
