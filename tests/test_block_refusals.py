"""Embedding, layer norm, feed-forward block: what the calls refuse (CPU only: they refuse before they touch the device)."""
import ctypes as C

import pytest
import torch

import paper_2410_20305_amd as ps

LIB = ps.load_library()
P = 4096  # an address that is never looked at
F32, BF16, BAD = 0, 1, 2


def _embed_fwd(dt=BF16, T=4, V=8, h=16, scale=1.0, ids=P, W=P, X=P):
    return LIB.psattn_embed_fwd(dt, T, V, h, scale, ids, W, X, None)


def _embed_bwd(dt=BF16, T=4, V=8, h=16, scale=1.0, ids=P, dX=P, dW=P, ws=P, n=1 << 30):
    return LIB.psattn_embed_bwd(dt, T, V, h, scale, ids, dX, dW, ws, n, None)


def _ln_fwd(dt=BF16, n=4, h=16, eps=1e-5, X=P, R=None, w=P, b=None, S=None, Y=P, mean=P, rstd=P):
    return LIB.psattn_layernorm_fwd(dt, n, h, eps, X, R, w, b, S, Y, mean, rstd, None)


def _ln_bwd(dt=BF16, n=4, h=16, S=P, w=P, mean=P, rstd=P, dY=P, dS=None, dX=P, dw=P, db=None, ws=P, size=1 << 30):
    return LIB.psattn_layernorm_bwd(dt, n, h, S, w, mean, rstd, dY, dS, dX, dw, db, ws, size, None)


def _ffn_fwd(dt=BF16, act=0, T=4, h=16, n=32, X=P, Wg=P, Wu=P, Wd=P, G=P, U=P, H=P, Y=P, ws=P, size=1 << 30):
    return LIB.psattn_ffn_fwd(dt, act, T, h, n, X, Wg, Wu, Wd, G, U, H, Y, ws, size, None)


def _ffn_bwd(dt=BF16, act=0, T=4, h=16, n=32, X=P, Wg=P, Wu=P, Wd=P, G=P, U=P, H=P, dY=P, dX=P, dWg=P, dWu=P, dWd=P, ws=P, size=1 << 30):
    return LIB.psattn_ffn_bwd(dt, act, T, h, n, X, Wg, Wu, Wd, G, U, H, dY, dX, dWg, dWu, dWd, ws, size, None)


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("call,args", [
    (_embed_fwd, dict(dt=BAD)), (_embed_fwd, dict(T=-1)), (_embed_fwd, dict(V=0)), (_embed_fwd, dict(h=0)), (_embed_fwd, dict(scale=NAN)),
    (_embed_fwd, dict(scale=INF)), (_embed_fwd, dict(ids=None)), (_embed_fwd, dict(W=None)), (_embed_fwd, dict(X=None)),
    (_embed_bwd, dict(dt=-1)), (_embed_bwd, dict(T=-1)), (_embed_bwd, dict(V=-2)), (_embed_bwd, dict(h=0)), (_embed_bwd, dict(scale=NAN)),
    (_embed_bwd, dict(ids=None)), (_embed_bwd, dict(dX=None)), (_embed_bwd, dict(dW=None)), (_embed_bwd, dict(ws=None)), (_embed_bwd, dict(n=0)),
    (_ln_fwd, dict(dt=BAD)), (_ln_fwd, dict(n=-1)), (_ln_fwd, dict(h=0)), (_ln_fwd, dict(eps=-1e-6)), (_ln_fwd, dict(eps=NAN)),
    (_ln_fwd, dict(eps=INF)), (_ln_fwd, dict(X=None)), (_ln_fwd, dict(w=None)), (_ln_fwd, dict(Y=None)), (_ln_fwd, dict(mean=None)),
    (_ln_fwd, dict(rstd=None)), (_ln_fwd, dict(R=P)), (_ln_fwd, dict(S=P)),
    (_ln_bwd, dict(dt=BAD)), (_ln_bwd, dict(n=-1)), (_ln_bwd, dict(h=-5)), (_ln_bwd, dict(S=None)), (_ln_bwd, dict(w=None)),
    (_ln_bwd, dict(mean=None)), (_ln_bwd, dict(rstd=None)), (_ln_bwd, dict(dY=None)), (_ln_bwd, dict(dX=None)), (_ln_bwd, dict(dw=None)),
    (_ln_bwd, dict(ws=None)), (_ln_bwd, dict(size=16)),
    (_ffn_fwd, dict(dt=BAD)), (_ffn_fwd, dict(act=2)), (_ffn_fwd, dict(act=-1)), (_ffn_fwd, dict(T=-1)), (_ffn_fwd, dict(h=0)), (_ffn_fwd, dict(n=0)),
    (_ffn_fwd, dict(X=None)), (_ffn_fwd, dict(Wg=None)), (_ffn_fwd, dict(Wu=None)), (_ffn_fwd, dict(Wd=None)), (_ffn_fwd, dict(H=None)),
    (_ffn_fwd, dict(Y=None)), (_ffn_fwd, dict(G=None)), (_ffn_fwd, dict(U=None)), (_ffn_fwd, dict(ws=None)), (_ffn_fwd, dict(size=0)),
    (_ffn_bwd, dict(dt=BAD)), (_ffn_bwd, dict(act=7)), (_ffn_bwd, dict(T=-1)), (_ffn_bwd, dict(h=0)), (_ffn_bwd, dict(n=-3)),
    *[(_ffn_bwd, {k: None}) for k in ("X", "Wg", "Wu", "Wd", "G", "U", "H", "dY", "dX", "dWg", "dWu", "dWd", "ws")], (_ffn_bwd, dict(size=64)),
])
def test_library_refuses(call, args):
    assert call(**args) == -1, args


@pytest.mark.parametrize("call,args", [
    (_embed_fwd, dict(T=(1 << 24) + 1)), (_embed_fwd, dict(h=(1 << 23) + 1)), (_embed_bwd, dict(T=(1 << 24) + 1, n=1 << 62)), (_embed_bwd, dict(V=(1 << 31) - 1, n=1 << 62)),
    (_embed_bwd, dict(V=1 << 28, n=1 << 62)), (_ln_fwd, dict(n=1 << 21)), (_ln_fwd, dict(h=(1 << 24) + 1)), (_ln_bwd, dict(n=1 << 21, size=1 << 62)),
    (_ln_bwd, dict(h=(1 << 24) + 8, size=1 << 62)), (_ffn_fwd, dict(h=1 << 22, size=1 << 62)), (_ffn_fwd, dict(dt=F32, h=1 << 21, size=1 << 62)),
    (_ffn_bwd, dict(h=1 << 22, size=1 << 62)), (_ffn_bwd, dict(n=1 << 22, size=1 << 62)),
])
def test_library_has_no_kernel_for(call, args):
    assert call(**args) == -6, args


def test_no_rows_is_no_error_forward():
    assert _embed_fwd(T=0, ids=None, X=None) == 0
    assert _ln_fwd(n=0, X=None, Y=None, mean=None, rstd=None) == 0
    assert _ffn_fwd(T=0, X=None, G=None, U=None, H=None, Y=None, ws=None) == 0


def test_workspace_sizes():
    for f in (LIB.psattn_embed_bwd_workspace_bytes, LIB.psattn_ffn_fwd_workspace_bytes, LIB.psattn_ffn_bwd_workspace_bytes):
        assert f(BF16, 5, 7, 9) > 0 and f(BF16, 0, 7, 9) > 0
        assert f(BAD, 5, 7, 9) == 0 and f(BF16, -1, 7, 9) == 0 and f(BF16, 5, 0, 9) == 0 and f(BF16, 5, 7, -9) == 0
    f = LIB.psattn_layernorm_bwd_workspace_bytes
    assert f(5, 7) > 0 and f(0, 7) > 0 and f(-1, 7) == 0 and f(5, 0) == 0
    # sizes past 32 bits
    assert LIB.psattn_ffn_bwd_workspace_bytes(BF16, 1 << 20, 8192, 28672) >= 4 * (1 << 20) * 28672
    assert LIB.psattn_layernorm_bwd_workspace_bytes(1 << 22, 1 << 14) < 1 << 34


def test_binding_refuses_host_tensors_and_wrong_shapes():
    X, W, ids = torch.zeros(4, 16), torch.zeros(8, 16), torch.zeros(4, dtype=torch.int32)
    w = torch.zeros(16)
    for call in (lambda: ps.psattn_embed_fwd(ids, W), lambda: ps.psattn_embed_bwd(ids, X, 8), lambda: ps.psattn_layernorm_fwd(X, w),
                 lambda: ps.psattn_layernorm_bwd(X, w, w[:4], w[:4], X), lambda: ps.psattn_ffn_fwd(X, W, W, W.T.contiguous()),
                 lambda: ps.psattn_ffn_bwd(X, W, W, W.T.contiguous(), (X, X, X), X)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="two dimensions"):
        ps.psattn_layernorm_fwd(X[0], w)
    with pytest.raises(ValueError, match="two dimensions"):
        ps.psattn_embed_fwd(ids, W[0])
