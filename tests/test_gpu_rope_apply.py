"""Rotary positions of any layout on Q and K in memory, and the transposed turn, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import DTYPES, HALF, Guarded, close, np64, rnd
from oracle import psattn_block_oracle as blk

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24
MOST = 300  # positions of a table


def _bound(x, pos, f, inter, amp, transposed, dtype):
    """A cosine and a sine are held in fp32, and two products and a sum follow: four roundings of the two terms' magnitudes."""
    n = len(f)
    y = blk.rotary(x, pos, f, inter, amp, transposed, MOST)
    size = np.zeros_like(y)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + n)
        size[..., [a, b]] = abs(amp) * (np.abs(x[..., [a]]) + np.abs(x[..., [b]]))
    return y, np.where(size > 0, HALF[dtype] * np.abs(y) + (1 + HALF[dtype]) * 4 * EPS32 * size, 0.0)


def _run(T, hq, hk, d, rotary, layout, dtype, scaling="none", amp=1.0, shift=0, pos=None, fused=False, in_place=False):
    rng = np.random.default_rng(T * 7 + hq * 5 + d + rotary)
    f = ps.psattn_rope_frequencies(rotary, 10000.0, scaling, factor=4.0, original_positions=128, low=1.0, high=8.0)
    rope = ps.Rope(d, 10000.0, MOST, rotary_dim=rotary, layout=layout, frequencies=f, amplitude=amp)
    pos = rng.integers(0, MOST, T) if pos is None else np.asarray(pos)
    dev = Guarded(dtype, shift)
    tp = dev.put(pos.astype(np.int32), dtype=torch.int32)
    inter = layout == "interleaved"
    for transposed, call in ((False, ps.psattn_rope_apply), (True, ps.psattn_rope_apply_bwd)):
        Q, K = rnd(rng, T, hq, d, dtype=dtype), rnd(rng, T, hk, d, dtype=dtype) if hk else None
        if fused:
            whole = dev.put(np.concatenate([Q, K, K], 1))
            tQ, tK = whole[:, :hq], whole[:, hq:hq + hk]
        else:
            tQ, tK = dev.put(Q), dev.put(K) if hk else None
        out = (tQ, tK) if in_place else (dev.empty(T, hq, d), dev.empty(T, hk, d) if hk else None)
        rQ, rK = call(rope, tQ, tK, tp, None, *out)
        dev.check()
        for got, x, what in ((rQ, Q, "Q"), (rK, K, "K")):
            if x is not None:
                close(np64(got), *_bound(x, pos, f, inter, amp, transposed, dtype), (what, transposed))
        if fused:
            assert np.array_equal(np64(whole[:, hq + hk:]), K), "what stands behind Q and K"
    return rope


HEADS = [(64, 64), (128, 128), (128, 64), (64, 32), (80, 80), (80, 40), (96, 24), (256, 256), (40, 20), (2, 2), (3, 2), (65, 64), (66, 64), (10, 4), (512, 512), (512, 2), (512, 16), (130, 6)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rotary", HEADS)
def test_heads(d, rotary, layout, dtype):
    _run(13, 3, 2, d, rotary, layout, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,hq,hk", [(1, 1, 0), (1, 32, 8), (2, 1, 1), (5, 7, 3), (33, 16, 16), (260, 9, 1), (1000, 8, 2), (4099, 5, 4)])
def test_tokens_and_head_counts(T, hq, hk, dtype):
    _run(T, hq, hk, 64, 64, "half", dtype)
    _run(T, hq, hk, 32, 16, "interleaved", dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("scaling,amp", [("linear", 1.0), ("base", 1.0), ("parts", 1.1386), ("none", -0.5), ("none", 0.0)])
def test_frequencies_and_amplitudes(scaling, amp, layout, dtype):
    _run(50, 4, 1, 64, 48, layout, dtype, scaling=scaling, amp=amp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [1, 2, 3, 4])
def test_unaligned(shift, dtype):
    _run(20, 3, 2, 64, 64, "half", dtype, shift=shift)
    _run(20, 3, 2, 64, 32, "interleaved", dtype, shift=shift)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rotary", [(64, 64), (80, 20), (33, 30)])
@pytest.mark.parametrize("in_place", [False, True])
def test_slices_of_one_buffer_and_in_place(d, rotary, in_place, dtype):
    for layout in ("half", "interleaved"):
        _run(37, 4, 2, d, rotary, layout, dtype, fused=True, in_place=in_place)
        _run(1, 4, 2, d, rotary, layout, dtype, fused=True, in_place=in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_positions_outside_the_table_give_zeros(in_place):
    pos = [0, -1, MOST - 1, MOST, 5, 2 ** 31 - 1, -2 ** 31, 7, MOST + 1]
    for layout in ("half", "interleaved"):
        _run(9, 3, 1, 40, 24, layout, "bf16", pos=pos, in_place=in_place)
        _run(9, 3, 1, 40, 24, layout, "f32", pos=pos, in_place=in_place)


@pytest.mark.parametrize("T", [60, 1500])
def test_positions_of_a_mask(T):
    """The mask's own positions, small (in the kernels' arguments) and large, as an array of the same numbers gives them."""
    off, P, c, r = [3, 30], [7, 5], [5, 8], [9, T - 60 + 6]
    meta = ps.psattn_build_meta(off, P, c, r, T)
    pos, n = meta.positions()
    rope = ps.Rope(64, 500.0, n, layout="interleaved", rotary_dim=32)
    Q, K = torch.randn(T, 4, 64, device="cuda").bfloat16(), torch.randn(T, 2, 64, device="cuda").bfloat16()
    tp = torch.from_numpy(pos).cuda()
    for call in (ps.psattn_rope_apply, ps.psattn_rope_apply_bwd):
        a, b = call(rope, Q, K, meta=meta), call(rope, Q, K, positions=tp)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    with pytest.raises(ps.PsattnError) as e:
        ps.psattn_rope_apply(ps.Rope(64, 500.0, n - 1, layout="half"), Q, K, meta=meta)
    assert e.value.status == -8


def test_the_same_rotation_as_inside_attention():
    """head_dim 128, half layout: Kr of psattn_fwd_rope bit for bit, from a table of either kind; one with other frequencies serves
    attention too."""
    T = 90
    meta = ps.psattn_build_meta([2], [20], [30], [35], T)
    Q, K, V = (torch.randn(T, h, 128, device="cuda").bfloat16() for h in (4, 2, 2))
    f = ps.psattn_rope_frequencies(128, 10000.0, "parts", factor=4.0, original_positions=32, low=1.0, high=4.0)
    for rope in (ps.Rope(128, 10000.0, 64), ps.Rope(128, 10000.0, 64, layout="half"), ps.Rope(128, 10000.0, 64, frequencies=f, amplitude=1.125)):
        O, LSE, Qr, Kr = ps.psattn_fwd_rope(meta, rope, Q, K, V, 0.1)
        q, k = ps.psattn_rope_apply(rope, Q, K, meta=meta)
        assert torch.equal(k, Kr) and torch.equal(q, Qr)
        O2, LSE2 = ps.psattn_fwd(meta, q, k, V, 0.1)
        assert torch.equal(O, O2) and torch.equal(LSE, LSE2)


def test_far_positions():
    """Angles of positions near 2^20: made in 64 bits."""
    n = 1 << 20
    rope = ps.Rope(4, 10000.0, n, layout="half")
    f = ps.psattn_rope_frequencies(4, 10000.0)
    pos = np.array([n - 1, n - 2, 999983])
    x = np.random.default_rng(1).standard_normal((3, 2, 4)).astype(np.float32).astype(np.float64)
    y = ps.psattn_rope_apply(rope, torch.from_numpy(x).float().cuda(), positions=torch.from_numpy(pos.astype(np.int32)).cuda())[0]
    ref = blk.rotary(x, pos, f)
    size = np.abs(x) + np.abs(np.roll(x, 2, -1))
    # 2^20 times a frequency's 2^-53 is 2^-33: nothing beside fp32
    close(np64(y), ref, 5 * EPS32 * size, "far")


def test_not_finite_stays_in_its_pair():
    rope = ps.Rope(64, 10000.0, 8, rotary_dim=32, layout="half")
    x = torch.ones(4, 2, 64, device="cuda")
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    good = ps.psattn_rope_apply(rope, x, positions=pos)[0]
    x[1, 0, 3], x[2, 1, 50] = float("nan"), float("inf")
    got = ps.psattn_rope_apply(rope, x, positions=pos)[0]
    bad = ~(got == good)
    assert {tuple(i) for i in bad.nonzero().tolist()} == {(1, 0, 3), (1, 0, 19), (2, 1, 50)}


def test_no_tokens():
    rope = ps.Rope(64, 10000.0, 8, layout="half")
    q = torch.empty(0, 3, 64, device="cuda")
    assert ps.psattn_rope_apply(rope, q, q, positions=torch.empty(0, dtype=torch.int32, device="cuda"))[0].shape == (0, 3, 64)


def test_refusals_of_the_binding():
    rope = ps.Rope(64, 10000.0, 8, layout="half")
    x, pos = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="contiguous"):
        ps.psattn_rope_apply(rope, x.transpose(0, 1).contiguous().transpose(0, 1), positions=pos)
    with pytest.raises(ValueError, match="contiguous"):
        ps.psattn_rope_apply(rope, x[:1].expand(4, 2, 64), positions=pos)
    with pytest.raises(ValueError, match="positions"):
        ps.psattn_rope_apply(rope, x, positions=pos[:3])
    with pytest.raises(TypeError, match="positions"):
        ps.psattn_rope_apply(rope, x, positions=pos.long())
    with pytest.raises(TypeError, match="K has dtype"):
        ps.psattn_rope_apply(rope, x, x.bfloat16(), positions=pos)
    with pytest.raises(ValueError, match="no K"):
        ps.psattn_rope_apply(rope, x, positions=pos, Kr=x)


@pytest.mark.parametrize("rotary,scaling,amp", [(128, "none", 1.0), (64, "base", 1.5), (6, "parts", -0.25)])
def test_far_positions(rotary, scaling, amp):
    """Cosines and sines as they stand in the table: half a step of fp32, and of an angle up to 2^20 in 64 bits, rounded once, 2^-33"""
    most = 1 << 20
    f = ps.psattn_rope_frequencies(rotary, 500000.0, scaling, factor=8.0, original_positions=8192, low=1.0, high=4.0)
    rope = ps.Rope(rotary, 500000.0, most, rotary_dim=rotary, layout="half", frequencies=f, amplitude=amp)
    pos = np.concatenate([np.arange(300), np.random.default_rng(rotary).integers(0, most, 3000), np.arange(most - 50, most)])
    x = torch.zeros(len(pos), 1, rotary, device="cuda")
    x[..., : rotary // 2] = 1.0
    got, _ = ps.psattn_rope_apply(rope, x, x, torch.from_numpy(pos.astype(np.int32)).cuda())
    a = pos[:, None].astype(np.float64) * f[None, :]
    want = amp * np.concatenate([np.cos(a), np.sin(a)], 1)
    close(np64(got)[:, 0], want, EPS32 * np.abs(want) + abs(amp) * 2.0 ** -32, "table")


@pytest.mark.parametrize("theta", [10000.0, 500000.0])
def test_tables_of_both_kinds_are_the_same(theta):
    n = 20011
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    x = torch.zeros(n, 1, 128, device="cuda")
    x[..., :64] = 1.0
    a, b = (ps.psattn_rope_apply(r, x, x, pos)[0] for r in (ps.Rope(128, theta, n), ps.Rope(128, theta, n, layout="half")))
    assert torch.equal(a, b)
