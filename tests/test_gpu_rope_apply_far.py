"""Rotary positions: rows turned at positions near 2^20, whose angles are made in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import close, np64
from oracle import psattn_block_oracle as blk

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("transposed", [False, True])
def test_rows_at_far_positions(layout, transposed):
    n = 1 << 20
    rope = ps.Rope(4, 10000.0, n, layout=layout)
    f = ps.psattn_rope_frequencies(4, 10000.0)
    pos = np.array([n - 1, n - 2, 999983])
    x = np.random.default_rng(1).standard_normal((3, 2, 4)).astype(np.float32).astype(np.float64)
    call = ps.psattn_rope_apply_bwd if transposed else ps.psattn_rope_apply
    y = call(rope, torch.from_numpy(x).float().cuda(), positions=torch.from_numpy(pos.astype(np.int32)).cuda())[0]
    ref = blk.rotary(x, pos, f, interleaved=layout == "interleaved", transposed=transposed)
    partner = [1, 0, 3, 2] if layout == "interleaved" else [2, 3, 0, 1]
    size = np.abs(x) + np.abs(x[..., partner])
    # 2^20 times a frequency's 2^-53 is 2^-33: nothing beside fp32
    close(np64(y), ref, 5 * EPS32 * size, "far")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_tensors_of_more_than_2_31_elements(layout):
    """Q and K out of one buffer: the last tokens as a call of their own gives them, bit for bit."""
    T, last = (1 << 31) // (20 * 128) + 100, 64
    whole = torch.empty(T, 20, 128, dtype=torch.bfloat16, device="cuda")
    assert whole.numel() > 1 << 31
    for at in range(0, T, 1 << 15):
        whole[at:at + (1 << 15)] = torch.randn(whole[at:at + (1 << 15)].shape, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda") % 4096
    rope = ps.Rope(128, 10000.0, 4096, layout=layout)
    for call in (ps.psattn_rope_apply, ps.psattn_rope_apply_bwd):
        Q, K = call(rope, whole[:, :16], whole[:, 16:], positions=pos)
        for some in (slice(T - last, T), slice(0, last)):
            q, k = call(rope, whole[some, :16].clone(), whole[some, 16:].clone(), positions=pos[some].clone())
            assert torch.equal(Q[some], q) and torch.equal(K[some], k)
