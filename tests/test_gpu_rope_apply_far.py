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
