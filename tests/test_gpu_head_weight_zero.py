"""Vocabulary head: a response whose d_resp_logp is 0 gives nothing to the gradients, whatever its rows of X hold."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from oracle import psattn_oracle as orc

pytestmark = pytest.mark.gpu

# offset, prompt lengths, response pointers, response lengths, tokens in all, the response of weight 0
TABLES = {
    "few": ([0], [5], [0, 2], [4, 6], 15, 1),
    "some": ([0, 40, 90], [10, 7, 30], [0, 2, 4, 6], [12, 9, 20, 21, 3, 1], 130, 2),
    "more": ([0, 300], [100, 20], [0, 2, 4], [60, 70, 90, 80], 500, 0),
    "many": ([0], [5], [0, 3], [900, 700, 500], 2105, 1),
}


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("table,V,h", [("few", 333, 104), ("few", 130, 4096), ("some", 700, 96), ("some", 260, 2049), ("more", 520, 72), ("many", 300, 64), ("many", 3000, 33)])
def test_rows_that_are_not_finite(table, V, h, dtype, value):
    off, P, ptr, rl, T, quiet = TABLES[table]
    g = torch.Generator().manual_seed(V + h)
    X, W = torch.randn(T, h, generator=g).to(dtype).cuda(), (torch.randn(V, h, generator=g) * h ** -0.5).to(dtype).cuda()
    ids = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda()
    d = torch.randn(len(rl), generator=g).cuda()
    d[quiet] = 0
    plan = ps.LogprobPlan(off, P, ptr, rl, T)
    items = orc.prediction_items(off, P, ptr, rl)
    own = sorted({r for j, r, _ in items if j == quiet} - {r for j, r, _ in items if j != quiet})  # the prompt's last row is others' too
    assert own
    lse, _ = ps.psattn_head_logprob_fwd(plan, X, W, ids)
    dX, dW = ps.psattn_head_logprob_bwd(plan, X, W, ids, lse, d)
    assert torch.isfinite(dW).all() and torch.all(dX[own] == 0)
    X[own] = value
    lse, logp = ps.psattn_head_logprob_fwd(plan, X, W, ids)
    assert torch.isnan(logp[quiet]) and torch.isnan(lse[own]).all()
    got = ps.psattn_head_logprob_bwd(plan, X, W, ids, lse, d)
    assert torch.equal(got[0], dX) and torch.equal(got[1], dW)
