"""The feed-forward block's workspaces hold what a call uses (CPU: sizes alone)."""
import pytest

import paper_2410_20305_amd as ps

LIB = ps.load_library()
F32, BF16 = 0, 1
MB = 1 << 20


def _sizes(dt, T, h, n):
    return [f(dt, T, h, n) for f in (LIB.psattn_ffn_fwd_workspace_bytes, LIB.psattn_ffn_bwd_workspace_bytes, LIB.psattn_ffn_fwd_unaligned_workspace_bytes,
                                     LIB.psattn_ffn_bwd_unaligned_workspace_bytes)]


@pytest.mark.parametrize("T,h,n", [(320, 4096, 14336), (16384, 4096, 14336), (1037, 1008, 2736), (70000, 8, 16)])
def test_no_room_for_copies_that_are_not_made(T, h, n):
    fwd, bwd, fwd_off, bwd_off = _sizes(BF16, T, h, n)
    copies = 2 * (T * h + 3 * h * n + T * n)
    assert fwd_off - fwd >= copies and bwd_off - bwd >= copies + 2 * T * h
    assert _sizes(BF16, 319, h, n)[2] - _sizes(BF16, 319, h, n)[0] < 2 * 3 * h * n   # no copies below 320 tokens
    if T == 16384:   # nothing is split: dG and dU alone
        assert fwd <= 1024 and bwd <= 2 * 2 * T * n + 2048


@pytest.mark.parametrize("T,h,n", [(320, 4095, 14336), (1037, 1001, 2731), (640, 64, 77), (500, 33, 80)])
def test_room_for_widths_that_are_not_whole(T, h, n):
    up8 = lambda x: (x + 7) // 8 * 8
    fwd, bwd, fwd_off, bwd_off = _sizes(BF16, T, h, n)
    copies = (2 * (T + 2 * n) * up8(h) if h % 8 else 0) + (2 * (T + h) * up8(n) if n % 8 else 0)
    assert fwd >= copies and bwd >= copies + 2 * T * up8(h) * (h % 8 > 0) + 2 * 2 * T * up8(n)
    assert fwd_off >= fwd and bwd_off >= bwd
    if h % 8 and n % 8:
        assert fwd_off == fwd and bwd_off == bwd


def test_fp32_needs_none_and_nonsense_has_none():
    a = _sizes(F32, 1000, 100, 300)
    assert a[0] == a[2] and a[1] == a[3]
    for bad in ((2, 5, 7, 9), (BF16, -1, 7, 9), (BF16, 5, 0, 9), (BF16, 5, 7, -9)):
        assert _sizes(*bad) == [0, 0, 0, 0]
    assert all(x > 0 for x in _sizes(BF16, 0, 7, 9))
