"""Vocabulary head, gated norms, rotary positions: what the calls refuse (CPU only: they refuse before they touch the device).  Plans and
rotary tables live on a device: these stand for them, in the library's layout, with addresses that are never looked at."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from oracle import psattn_block_oracle as blk

LIB = ps.load_library()
P = 4096  # an address that is never looked at
F32, BF16, BAD = 0, 1, 2
INF, NAN = float("inf"), float("nan")


class _Plan(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("T", "n_samples", "n_resp", "n_rows")] + [("n_items", C.c_int64), ("device", C.c_int)] + [("p%d" % i, C.c_void_p) for i in range(11)]


class _Rope(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("head_dim", "rotary_dim", "layout", "max_positions")] + [("device", C.c_int), ("table", C.c_void_p)]


PLAN = _Plan(T=10, n_samples=1, n_resp=2, n_rows=5, n_items=6)
HUGE = _Plan(T=1 << 24, n_samples=1, n_resp=2, n_rows=1 << 23, n_items=1 << 23)
NONE = _Plan(T=10)
ROPE = _Rope(128, 128, 0, 64)
a_plan, a_rope = C.addressof, C.addressof


def _head_fwd(plan=PLAN, dt=BF16, V=100, h=64, X=P, W=P, ids=P, lse=P, logp=P, ws=P, n=1 << 40):
    return LIB.psattn_head_logprob_fwd(None if plan is None else a_plan(plan), dt, V, h, X, W, ids, lse, logp, ws, n, None)


def _head_bwd(plan=PLAN, dt=BF16, V=100, h=64, X=P, W=P, ids=P, lse=P, d=P, dX=P, dW=P, ws=P, n=1 << 40):
    return LIB.psattn_head_logprob_bwd(None if plan is None else a_plan(plan), dt, V, h, X, W, ids, lse, d, dX, dW, ws, n, None)


def _gn_fwd(dt=BF16, n=4, h=16, eps=1e-6, res=1.0, X=P, B=P, w_post=P, gate=P, rows=1, w_pre=P, S=P, Y=P, rb=P, rs=P):
    return LIB.psattn_gatednorm_fwd(dt, n, h, eps, res, X, B, w_post, gate, rows, w_pre, S, Y, rb, rs, None)


def _gn_bwd(dt=BF16, n=4, h=16, res=1.0, B=P, w_post=P, gate=P, rows=1, w_pre=P, S=P, rb=P, rs=P, dY=P, dS=None, dX=P, dB=P, dw_post=P, dgate=P, dw_pre=P, ws=P,
            size=1 << 40):
    return LIB.psattn_gatednorm_bwd(dt, n, h, res, B, w_post, gate, rows, w_pre, S, rb, rs, dY, dS, dX, dB, dw_post, dgate, dw_pre, ws, size, None)


def _apply(rope=ROPE, dt=BF16, tr=0, T=3, pos=P, meta=None, hq=4, Q=P, q=512, Qr=P, qr=512, hk=2, K=P, k=256, Kr=P, kr=256):
    return LIB.psattn_rope_apply(None if rope is None else a_rope(rope), dt, tr, T, pos, meta, hq, Q, q, Qr, qr, hk, K, k, Kr, kr, None)


def _create(d=128, r=128, layout=0, f=None, amp=1.0, n=8):
    out = C.c_void_p(1)
    if f is None:
        f = np.ones(64)
    rc = LIB.psattn_rope_create_layout(d, r, layout, f.__array_interface__["data"][0] if isinstance(f, np.ndarray) else None, amp, n, None, C.byref(out))
    assert out.value is None
    return rc


def _freq(n=32, theta=1e4, kind=0, factor=8.0, L=4096.0, low=1.0, high=32.0, out=True):
    x = np.zeros(max(1, n))
    return LIB.psattn_rope_frequencies(n, theta, kind, factor, L, low, high, x.__array_interface__["data"][0] if out else None)


@pytest.mark.parametrize("call,args", [
    *[(_head_fwd, {k: None}) for k in ("plan", "X", "W", "ids", "lse", "logp", "ws")],
    *[(_head_bwd, {k: None}) for k in ("plan", "X", "W", "ids", "lse", "d", "dX", "dW", "ws")],
    *[(c, a) for c in (_head_fwd, _head_bwd) for a in (dict(dt=BAD), dict(dt=-1), dict(V=0), dict(h=0), dict(V=-4), dict(n=64))],
    *[(_gn_fwd, {k: None}) for k in ("X", "B", "w_pre", "S", "Y", "rb", "rs")],
    *[(_gn_bwd, {k: None}) for k in ("B", "w_post", "gate", "w_pre", "S", "rb", "rs", "dY", "dX", "dB", "dw_post", "dgate", "dw_pre", "ws")],
    *[(c, a) for c in (_gn_fwd, _gn_bwd) for a in (dict(dt=BAD), dict(n=-1), dict(h=0), dict(res=NAN), dict(res=INF), dict(rows=0), dict(rows=2), dict(rows=5), dict(rows=-1),
                                                  dict(gate=None, rows=1))],
    (_gn_fwd, dict(eps=-1.0)), (_gn_fwd, dict(eps=NAN)), (_gn_fwd, dict(eps=INF)), (_gn_fwd, dict(B=None, S=None)), (_gn_fwd, dict(B=None, S=None, gate=None, rows=0)),
    (_gn_bwd, dict(size=100)), (_gn_bwd, dict(B=None, dB=None)),
    (_apply, dict(rope=None)), (_apply, dict(dt=BAD)), (_apply, dict(T=-1)), (_apply, dict(hq=-1)), (_apply, dict(hk=-1)), (_apply, dict(pos=None)),
    (_apply, dict(meta=P)), (_apply, dict(q=511)), (_apply, dict(qr=0)), (_apply, dict(k=255)), (_apply, dict(kr=-256)),
    *[(_apply, {k: None}) for k in ("Q", "Qr", "K", "Kr")],
    (_create, dict(d=0)), (_create, dict(r=0)), (_create, dict(r=63)), (_create, dict(r=130)), (_create, dict(layout=2)), (_create, dict(layout=-1)), (_create, dict(f=0)),
    (_create, dict(amp=NAN)), (_create, dict(amp=INF)), (_create, dict(n=0)), (_create, dict(f=np.full(64, NAN))), (_create, dict(f=np.full(64, INF))),
    (_freq, dict(out=False)), (_freq, dict(n=0)), (_freq, dict(n=7)), (_freq, dict(theta=0.0)), (_freq, dict(theta=NAN)), (_freq, dict(theta=INF)), (_freq, dict(kind=4)),
    (_freq, dict(kind=-1)), (_freq, dict(kind=1, factor=0.0)), (_freq, dict(kind=2, factor=NAN)), (_freq, dict(kind=3, factor=INF)), (_freq, dict(kind=3, L=0.0)),
    (_freq, dict(kind=3, low=4.0, high=4.0)), (_freq, dict(kind=3, high=NAN)), (_freq, dict(kind=3, low=-INF)),
])
def test_library_refuses(call, args):
    assert call(**args) == -1, args


@pytest.mark.parametrize("call,args", [
    (_head_fwd, dict(plan=HUGE)), (_head_bwd, dict(plan=HUGE)), (_head_fwd, dict(h=1 << 22)), (_head_bwd, dict(h=1 << 22)), (_head_fwd, dict(dt=F32, h=1 << 21)),
    (_head_fwd, dict(V=(1 << 31) - 1)), (_head_bwd, dict(V=(1 << 31) - 1)), (_head_fwd, dict(plan=_Plan(T=1 << 23, n_samples=1, n_resp=1, n_rows=4000000, n_items=4000000), V=1 << 20)),
    (_gn_fwd, dict(n=1 << 21)), (_gn_fwd, dict(h=(1 << 24) + 1)), (_gn_bwd, dict(n=1 << 21, size=1 << 62)), (_gn_bwd, dict(h=(1 << 24) + 1, size=1 << 62)),
    (_create, dict(d=513)), (_create, dict(d=1024)), (_apply, dict(hq=(1 << 20) + 1, q=1 << 40, qr=1 << 40)),
    (_apply, dict(T=(1 << 31) - 1)), (_apply, dict(rope=_Rope(512, 2, 0, 4), T=1 << 25, hq=1, hk=0, Q=P + 2, q=512, qr=512)),
])
def test_library_has_no_kernel_for(call, args):
    assert call(**args) == -6, args


def test_a_mask_without_a_device_and_of_another_size():
    meta = ps.psattn_build_meta([0], [2], [1], [1], 6, host_only=True)
    assert _apply(pos=None, meta=meta.handle, T=6) == -7
    assert _apply(pos=None, meta=meta.handle, T=5) == -1


def test_attention_refuses_tables_of_other_layouts():
    meta = ps.psattn_build_meta([0], [2], [1], [1], 6, host_only=True)
    for rope in (_Rope(128, 64, 0, 8), _Rope(128, 128, 1, 8), _Rope(64, 64, 0, 8)):
        assert LIB.psattn_rope_k(meta.handle, a_rope(rope), BF16, 2, 128, P, P, None) == -6
    assert LIB.psattn_rope_k(meta.handle, a_rope(_Rope(128, 128, 0, 8)), BF16, 2, 128, P, P, None) == -7  # the mask has no device


def test_nothing_to_do_is_no_error():
    assert _head_fwd(plan=NONE, X=None, W=None, ids=None, lse=None, logp=None, ws=None) == 0
    assert _gn_fwd(n=0, X=None, B=None, S=None, Y=None, rs=None, w_post=None, gate=None, rows=0) == 0
    assert _apply(T=0, pos=None, Q=None, K=None, Qr=None, Kr=None) == 0
    assert _apply(hq=0, hk=0, Q=None, K=None, Qr=None, Kr=None) == 0


def test_workspace_sizes():
    for f in (LIB.psattn_head_logprob_fwd_workspace_bytes, LIB.psattn_head_logprob_bwd_workspace_bytes):
        assert f(a_plan(PLAN), BF16, 7, 9) > 0 and f(a_plan(NONE), F32, 7, 9) > 0
        assert f(None, BF16, 7, 9) == 0 and f(a_plan(PLAN), BAD, 7, 9) == 0 and f(a_plan(PLAN), BF16, 0, 9) == 0 and f(a_plan(PLAN), BF16, 7, -9) == 0
    many = _Plan(T=50000, n_samples=1, n_resp=2, n_rows=40000, n_items=40000)
    # a piece of the logits' gradient, not all of it (10 GB), beside the rows and dX's sums
    assert LIB.psattn_head_logprob_bwd_workspace_bytes(a_plan(many), BF16, 128000, 4096) < (1 << 29) + 40000 * 4096 * 6 + (1 << 21)
    assert LIB.psattn_gatednorm_bwd_workspace_bytes(5, 7) > 0 and LIB.psattn_gatednorm_bwd_workspace_bytes(0, 7) > 0
    assert LIB.psattn_gatednorm_bwd_workspace_bytes(-1, 7) == 0 and LIB.psattn_gatednorm_bwd_workspace_bytes(5, 0) == 0


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
@pytest.mark.parametrize("n", [2, 4, 32, 128])
def test_frequencies(scaling, n):
    """Powers, products and quotients in 64 bits: a few roundings each, and a power's argument error of 2^-53 times log(theta)."""
    got = ps.psattn_rope_frequencies(n, 10000.0, scaling, factor=8.0, original_positions=4096, low=1.0, high=32.0)
    ref = blk.rotary_frequencies(n, 10000.0, scaling, 8.0, 4096.0, 1.0, 32.0)
    assert got.shape == (n // 2,) and np.all(np.abs(got - ref) <= 64 * 2.0 ** -53 * ref)


def test_binding_refuses():
    X, w, ids = torch.zeros(4, 16), torch.zeros(16), torch.zeros(4, dtype=torch.int32)

    class Table:
        handle, head_dim = None, 16
    Q = torch.zeros(4, 2, 16)
    plan = type("Plan", (), dict(handle=None, total_tokens=4, n_responses=2))()
    for call in (lambda: ps.psattn_gatednorm_fwd(X, X, w), lambda: ps.psattn_gatednorm_bwd(X, X, w, None, w[:4], X), lambda: ps.psattn_rope_apply(Table, Q, positions=ids),
                 lambda: ps.psattn_rope_apply_bwd(Table, Q, Q, positions=ids), lambda: ps.psattn_head_logprob_fwd(plan, X, X, ids),
                 lambda: ps.psattn_head_logprob_bwd(plan, X, X, ids, w[:4], w[:2])):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="one of them"):
        ps.psattn_rope_apply(Table, Q)
    with pytest.raises(ValueError, match="three dimensions"):
        ps.psattn_rope_apply(Table, X, positions=ids)
    with pytest.raises(ValueError, match="the rotary table of 16"):
        ps.psattn_rope_apply(Table, Q[..., :8], positions=ids)
    with pytest.raises(ValueError, match="layout must be"):
        ps.Rope(16, 1e4, 8, layout="quarter")
    with pytest.raises(ValueError, match="frequencies has shape"):
        ps.Rope(16, 1e4, 8, frequencies=np.ones(4))
    with pytest.raises(ValueError, match="scaling must be"):
        ps.psattn_rope_frequencies(16, 1e4, "yes")
    with pytest.raises(ps.PsattnError):
        ps.psattn_rope_frequencies(15, 1e4)
