"""Embedding and layer norm at sizes that take their paths for many rows: long pieces and several passes of the sort, four tokens at a
time, many rows to a workgroup, column sums of wide rows."""
import pytest
import torch

import paper_2410_20305_amd as ps
from test_gpu_layernorm import _check, _run

pytestmark = pytest.mark.gpu


# pieces of 64 tokens; four tokens at a time off 16-byte boundaries; blocks of more than 1 024 tokens in the sort and three passes of
# digits; one id with most of the tokens over many long pieces
@pytest.mark.parametrize("dtype,T,V,h,share", [("bf16", 33000, 5000, 8192, 0.0), ("f32", 8334, 50257, 1001, 0.0), ("bf16", 8334, 50257, 1001, 0.3), ("f32", 70000, 300000, 24, 0.0),
                                               ("bf16", 70001, 300000, 33, 0.2), ("bf16", 34000, 40, 8000, 0.9), ("f32", 200000, 1000, 17, 0.1)])
def test_embedding_on_whole_numbers(dtype, T, V, h, share):
    """Sums of small whole numbers are exact in fp32: each token counted once and at its row."""
    gen = torch.Generator(device="cuda").manual_seed(T)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    ids = torch.randint(-1, V + 1, (T,), generator=gen, device="cuda", dtype=torch.int32)
    ids[torch.rand(T, generator=gen, device="cuda") < share] = V // 2
    W = torch.randint(-128, 129, (V, h), generator=gen, device="cuda").to(dt)
    dX = torch.randint(-3, 4, (T, h), generator=gen, device="cuda").to(dt)
    real = (ids >= 0) & (ids < V)
    at = torch.where(real, ids, 0).long()
    X = ps.psattn_embed_fwd(ids, W, scale=2.0)
    assert torch.equal(X, torch.where(real[:, None], W[at] * 2, torch.zeros((), dtype=dt, device="cuda")))
    del X, W
    want = torch.zeros(V, h, dtype=torch.float64, device="cuda")
    for i in range(0, T, 10000):
        want.index_add_(0, at[i:i + 10000], torch.where(real[i:i + 10000, None], dX[i:i + 10000].double(), 0.0))
    assert torch.equal(ps.psattn_embed_bwd(ids, dX, V, scale=2.0), (want * 2).to(dt))


# rows of one workgroup each, many to a workgroup in the backward, aligned and not; rows whose columns are summed in a pass of their own
# (the last row of each type: too wide for registers)
@pytest.mark.parametrize("dtype,n,h", [("bf16", 3000, 4096), ("bf16", 2999, 2050), ("bf16", 2500, 5001), ("f32", 3000, 1030), ("f32", 1700, 4100), ("f32", 1500, 6001),
                                       ("bf16", 1100, 9001), ("bf16", 1100, 9000), ("f32", 1100, 9001), ("bf16", 900, 20001), ("f32", 900, 17002)])
def test_layer_norm_of_many_rows(dtype, n, h):
    _check(*_run(n, h, dtype, residual=h % 2 == 0, bias=True), dtype)
