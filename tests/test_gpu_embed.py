"""Embedding and its gradient against the 64-bit oracle, and what the calls promise about ids, edges and order."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import DTYPES, HALF, Guarded, close, np64, rnd, same
from oracle import psattn_block_oracle as blk

pytestmark = pytest.mark.gpu


def _ids(rng, T, V, kind):
    if kind == "log":        # few frequent ids, many rare ones, some padding
        ids = np.exp(rng.uniform(0, np.log(V + 1.0), T)).astype(np.int64) - 1
        ids[rng.uniform(size=T) < 0.1] = -1
    elif kind == "one":      # every token the same
        ids = np.full(T, V // 2)
    elif kind == "none":     # nothing but padding
        ids = np.where(np.arange(T) % 2, -1, V)
    elif kind == "falling":
        ids = (V - 1 - np.arange(T)) % V
    else:                    # ids at and outside the ends
        ids = rng.choice([0, V - 1, V, -1, -2 ** 31, 2 ** 31 - 1, V // 2], T)
    return ids.astype(np.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,h,kind,shift", [
    (1, 1, 1, "one", 0), (1, 100, 4096, "log", 0), (2, 7, 3, "ends", 1), (63, 50, 64, "log", 0), (64, 1, 33, "one", 0), (257, 1000, 130, "falling", 0),
    (1000, 300, 200, "log", 3), (1025, 5, 65, "log", 0), (2048, 4096, 96, "falling", 0), (3000, 70001, 17, "log", 0), (5000, 33, 40, "one", 0),
    (700, 12, 129, "none", 0), (4097, 513, 24, "ends", 1), (20000, 900, 8, "log", 0), (9000, 257, 1032, "log", 0),
])
def test_rows_and_gradient(dtype, T, V, h, kind, shift):
    rng = np.random.default_rng(T * 31 + V)
    ids, scale = _ids(rng, T, V, kind), 1.375
    W, dX = rnd(rng, V, h, dtype=dtype), rnd(rng, T, h, dtype=dtype)
    dev = Guarded(dtype, shift)
    tids = dev.put(ids, dtype=torch.int32)
    X = ps.psattn_embed_fwd(tids, dev.put(W), scale=scale, X=dev.empty(T, h))
    dW = ps.psattn_embed_bwd(tids, dev.put(dX), V, scale=scale, dW=dev.empty(V, h))
    dev.check()
    close(X, blk.embed(ids, W, scale), HALF[dtype] * np.abs(blk.embed(ids, W, scale)) * (1 + 2 ** -8), "X")
    ref, mag = blk.embed_grad(ids, dX, V, scale), blk.embed_grad(ids, np.abs(dX), V, scale)
    # one rounding per addition, one for the scale
    n = np.zeros(V)
    np.add.at(n, ids[(ids >= 0) & (ids < V)], 1)
    close(dW, ref, HALF[dtype] * np.abs(ref) + (n[:, None] + 2) * 2.0 ** -24 * mag * (1 + HALF[dtype]), "dW")
    assert np.all(np64(dW)[n == 0] == 0)


@pytest.mark.parametrize("T,V,kind", [(3001, 97, "log"), (4000, 2, "one"), (600, 70000, "falling")])
def test_gradient_is_exact_on_whole_numbers(T, V, kind):
    """Small whole numbers add up without rounding: every token is counted once and at its row."""
    rng = np.random.default_rng(11)
    ids = _ids(rng, T, V, kind)
    dX = rng.integers(-3, 4, (T, 72)).astype(np.float64)
    dev = Guarded("f32")
    same(ps.psattn_embed_bwd(dev.put(ids, dtype=torch.int32), dev.put(dX), V, scale=2.0), blk.embed_grad(ids, dX, V, 2.0), "dW")


def test_gradient_repeats_bit_for_bit_and_leaves_no_trace():
    """Same bits again, on a workspace that held something else, and after a call of another size on it."""
    rng = np.random.default_rng(3)
    T, V, h = 7000, 500, 264
    ids = torch.from_numpy(_ids(rng, T, V, "log")).cuda()
    dX = torch.from_numpy(rng.standard_normal((T, h))).to(torch.bfloat16).cuda()
    need = ps.load_library().psattn_embed_bwd_workspace_bytes(ps.BF16, T, V, h)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    first = ps.psattn_embed_bwd(ids, dX, V, workspace=ws)
    ps.psattn_embed_bwd(ids[:100], dX[:100], V, workspace=ws)
    for _ in range(3):
        assert torch.equal(ps.psattn_embed_bwd(ids, dX, V, workspace=ws), first)


def test_order_of_a_rows_sum_is_that_of_the_tokens():
    """fp32 addition keeps what it is given first: 1 + 2^-24 ... in the order of the tokens, whatever else is in the batch."""
    h, V = 8, 40
    dX = np.zeros((300, h))
    ids = np.arange(300) % V
    mine = np.nonzero(ids == 7)[0]
    dX[mine] = (2.0 ** -24)
    dX[mine[0]] = 1.0   # first: every later 2^-24 is half a step of 1 and is dropped
    got = np64(ps.psattn_embed_bwd(torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(dX).float().cuda(), V))
    assert np.all(got[7] == 1.0)


def test_rows_without_tokens_are_not_read():
    """NaN in rows of padding, and in other ids' rows, reach nothing."""
    ids = torch.tensor([1, -1, 2, 9, 1], dtype=torch.int32, device="cuda")
    dX = torch.ones(5, 24, dtype=torch.bfloat16, device="cuda")
    dX[1] = float("nan")
    dX[3] = float("inf")
    dX[2, 5] = float("nan")
    dW = ps.psattn_embed_bwd(ids, dX, 9)
    assert torch.all(dW[1] == 2) and torch.isnan(dW[2, 5]) and torch.isfinite(dW).sum() == dW.numel() - 1
    W = torch.full((9, 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    W[1], W[2] = 1, 3
    X = ps.psattn_embed_fwd(ids, W, scale=0.5)
    assert X[:, 0].tolist() == [0.5, 0.0, 1.5, 0.0, 0.5]


def test_no_tokens():
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert ps.psattn_embed_fwd(none, torch.ones(3, 4, device="cuda")).shape == (0, 4)
    dW = torch.full((3, 5), float("nan"), device="cuda")
    ps.psattn_embed_bwd(none, torch.empty(0, 5, device="cuda"), 3, dW=dW)
    assert torch.all(dW == 0)


def test_table_past_32_bits():
    """Rows whose byte offset passes 2^32: 40 000 rows of 65 000 bf16 (5.2 GB)."""
    V, h = 40000, 65000
    W = torch.zeros(V, h, dtype=torch.bfloat16, device="cuda")
    W[V - 1] = 3.0
    W[1] = 2.0
    ids = torch.tensor([V - 1, 1, -1, V - 1], dtype=torch.int32, device="cuda")
    X = ps.psattn_embed_fwd(ids, W)
    assert X[:, 0].tolist() == [3, 2, 0, 3] and X[:, h - 1].tolist() == [3, 2, 0, 3]
    W.fill_(float("nan"))
    ps.psattn_embed_bwd(ids, X, V, dW=W)
    assert torch.all(W[V - 1] == 6) and torch.all(W[1] == 2) and torch.all(W[0] == 0) and torch.all(W[V - 2] == 0) and torch.all(W[V // 2] == 0)


def test_refusals_on_the_device():
    ids, W = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(8, 16, device="cuda")
    with pytest.raises(TypeError):
        ps.psattn_embed_fwd(ids.long(), W)
    with pytest.raises(TypeError):
        ps.psattn_embed_fwd(ids, W.half())
    with pytest.raises(ValueError):
        ps.psattn_embed_fwd(ids, W.T)
    with pytest.raises(ValueError):
        ps.psattn_embed_bwd(ids, W, 8)          # eight rows for four ids
    with pytest.raises(ValueError):
        ps.psattn_embed_bwd(ids, W[:4], 0)
    with pytest.raises(ps.PsattnError):
        ps.psattn_embed_bwd(ids, W[:4], 8, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert DTYPES["bf16"] == torch.bfloat16
