"""RMS norms before and after a block with its gate and residual scale, and their gradients, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import HALF, Guarded, close, hold, np64, rnd
from oracle import psattn_block_oracle as blk

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24


def _run(n, h, dtype, post=True, gate="row", block=True, ds=True, seed=0, shift=0, eps=1e-6, res=0.875):
    rng = np.random.default_rng(n * 13 + h + seed)
    a = dict(X=rnd(rng, n, h, scale=2.0, dtype=dtype), B=None, w_pre=rnd(rng, h, scale=0.3, shift=1.0, dtype=dtype), w_post=None, gate=None,
             dY=rnd(rng, n, h, dtype=dtype), dS=rnd(rng, n, h, dtype=dtype) if ds else None, eps=float(np.float32(eps)), res=float(np.float32(res)))
    if block:
        a["B"] = rnd(rng, n, h, scale=0.5, shift=0.05, dtype=dtype)
        a["w_post"] = rnd(rng, h, scale=0.3, shift=0.7, dtype=dtype) if post else None
        a["gate"] = None if gate is None else rnd(rng, *(dict(row=(h,), one=(1, h), all=(n, h))[gate]), scale=0.4, shift=0.4, dtype=dtype)
    dev = Guarded(dtype, shift)
    put = lambda x: None if x is None else dev.put(x)
    f32 = lambda: dev.empty(n, dtype=torch.float32)
    t = {k: put(a[k]) for k in ("X", "B", "w_pre", "w_post", "gate", "dY", "dS")}
    form = dict(w_post=t["w_post"], gate=t["gate"], res_scale=res)
    has_b, has_p = t["B"] is not None, t["w_post"] is not None
    Y, S, rb, rs = ps.psattn_gatednorm_fwd(t["X"], t["B"], t["w_pre"], eps=eps, S=dev.empty(n, h) if has_b else None, Y=dev.empty(n, h), rstd_b=f32() if has_p else None,
                                           rstd_s=f32(), **form)
    dX, dB, dwp, dwo, dg = ps.psattn_gatednorm_bwd(t["B"], S, t["w_pre"], rb, rs, t["dY"], dS=t["dS"], dX=dev.empty(n, h), dB=dev.empty(n, h) if has_b else None,
                                                   dw_pre=dev.empty(h), dw_post=dev.empty(h) if has_p else None,
                                                   dgate=dev.empty(*a["gate"].shape) if a["gate"] is not None else None, **form)
    dev.check()
    return a, dict(Y=Y, S=S, rb=rb, rs=rs, dX=dX, dB=dB, dw_pre=dwp, dw_post=dwo, dgate=dg)


def _check(a, got, dtype):
    """Error bounds.  A row's sums of h terms run in chains of at most c = h / 64 + 24 additions (64 lanes and more, then a tree),
    so that a reciprocal root is off by r = (c + 4) 2^-24 relatively.  From there on products and sums add up.  The second norm's and the
    gradients' references start from the held S."""
    X, B, w_pre, w_post, g, dY, dS, eps, res = (a[k] for k in ("X", "B", "w_pre", "w_post", "gate", "dY", "dS", "eps", "res"))
    n, h = X.shape
    half, c, E = HALF[dtype], h / 64 + 24, EPS32
    r = (c + 4) * E
    _, S64, rb, _ = blk.gatednorm(X, B, w_pre, w_post, g, res, eps)
    if B is not None:
        if w_post is not None:
            close(got["rb"], rb, rb * (r + E), "rstd_b")
        close(got["S"], S64, half * np.abs(S64) + (1 + half) * (np.abs(S64 - res * X) * (r + 6 * E) + 2 * E * (np.abs(res * X) + np.abs(S64))), "S")
    S = np64(got["S"])
    Y, _, _, rs = blk.gatednorm(S, None, w_pre, None, None, 1.0, eps)
    close(got["rs"], rs, rs * (r + E), "rstd_s")
    close(got["Y"], Y, (half + (1 + half) * (r + 4 * E)) * np.abs(Y), "Y")
    rs = rs[:, None]
    sh, q = S * rs, dY * w_pre
    ds0 = 0 if dS is None else dS
    t = ds0 + rs * q
    e_t = 2 * E * np.abs(t) + np.abs(rs * q) * (r + 4 * E)
    m = rs[:, 0] * (q * sh).mean(1)
    e_m = rs[:, 0] * np.abs(q * sh).mean(1) * ((c + 8) * E + 2 * r)
    m, e_m = m[:, None], e_m[:, None]
    ds = t - m * sh
    e_ds = e_t + e_m * np.abs(sh) + np.abs(m * sh) * (r + 4 * E) + 2 * E * np.abs(ds)
    dX, dB, dw_pre, dw_post, dgate = blk.gatednorm_grad(B, S, w_pre, w_post, g, res, eps, dY, dS)
    k = 1.0 if B is None else abs(res)
    close(got["dX"], dX, half * np.abs(dX) + (1 + half) * (k * e_ds + 2 * E * np.abs(dX)), "dX")
    chain = (min(n, 600) + 8) * E  # sums over rows: one rounding per addition, never more than some hundreds in a chain
    close(got["dw_pre"], dw_pre, half * np.abs(dw_pre) + (1 + half) * (np.abs(dY * sh) * (r + 3 * E + chain)).sum(0), "dw_pre")
    if B is None:
        return
    bh = B if rb is None else B * rb[:, None]
    r_b = 0 if rb is None else r
    one_g, one_w = np.ones(()) if g is None else g, np.ones(()) if w_post is None else w_post
    gw = np.broadcast_to(one_g * one_w, S.shape)
    e_c = e_ds * np.abs(bh) + np.abs(ds * bh) * (r_b + 3 * E)
    if g is not None:
        e = np.abs(one_w) * (e_c + np.abs(ds * bh) * 3 * E)
        if dgate.shape == S.shape and n > 1:
            close(got["dgate"], dgate, half * np.abs(dgate) + (1 + half) * e, "dgate")
        else:
            e = (e + chain * np.abs(one_w * ds * bh)).sum(0)
            close(np64(got["dgate"]).reshape(-1), dgate.reshape(-1), half * np.abs(dgate.reshape(-1)) + (1 + half) * e, "dgate")
    if w_post is not None:
        e = (np.abs(one_g) * (e_c + np.abs(ds * bh) * (3 * E + chain))).sum(0)
        close(got["dw_post"], dw_post, half * np.abs(dw_post) + (1 + half) * e, "dw_post")
        mb = (ds * gw * bh).mean(1)[:, None]
        e_mb = (np.abs(t * gw * bh) * ((c + 6) * E + r_b) + e_t * np.abs(gw * bh)).mean(1)[:, None] + \
            (e_m + np.abs(m) * ((c + 8) * E + r + r_b)) * np.abs(sh * gw * bh).mean(1)[:, None] + 4 * E * np.abs(mb)
        e = rb[:, None] * (e_ds * np.abs(gw) + 4 * E * np.abs(ds * gw) + np.abs(bh) * e_mb + np.abs(bh * mb) * (r_b + 4 * E)) + np.abs(dB) * (r_b + 3 * E)
    else:
        e = e_ds * np.abs(gw) + 3 * E * np.abs(ds * gw)
    close(got["dB"], dB, half * np.abs(dB) + (1 + half) * e, "dB")


SHAPES = [(1, 1), (1, 2), (3, 7), (1, 64), (5, 63), (2, 65), (70, 128), (33, 130), (129, 256), (64, 257), (9, 511), (300, 512), (7, 1000), (40, 1001), (17, 1024), (3, 1026),
          (19, 2048), (5, 2050), (11, 4096), (2, 4104), (3, 8192), (2, 8200), (2, 16384), (3, 16392), (2, 20001), (1, 65536)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,h", SHAPES)
def test_shapes(n, h, dtype):
    _check(*_run(n, h, dtype, post=(n + h) % 3 != 0, gate=("row", "all", None, "one")[(n + h) % 4], ds=h % 2 == 0), dtype)
    _check(*_run(n, h, dtype, gate="all"), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", [None, "row", "one", "all"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("ds", [False, True])
def test_every_form(dtype, gate, post, ds):
    _check(*_run(37, 768, dtype, post, gate, ds=ds), dtype)
    _check(*_run(5, 9000, dtype, post, gate, ds=ds), dtype)
    _check(*_run(3, 17000, dtype, post, gate, ds=ds), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,h", [(1, 5), (20, 100), (9, 4096), (3, 9001), (2, 17000)])
def test_norm_alone(n, h, dtype):
    """Without a block's output: Y is the norm of X, whose gradient takes dS along."""
    _check(*_run(n, h, dtype, block=False, ds=h != 100), dtype)


@pytest.mark.parametrize("n,h,shift", [(5, 256, 1), (9, 4096, 3), (4, 1000, 2), (3, 8192, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unaligned_rows(n, h, shift, dtype):
    _check(*_run(n, h, dtype, gate="all", shift=shift), dtype)
    _check(*_run(n, h, dtype, gate="row", shift=shift), dtype)


@pytest.mark.parametrize("n", [2, 255, 1023, 4096, 20011])
def test_many_rows(n):
    _check(*_run(n, 96, "bf16"), "bf16")
    _check(*_run(n, 40, "f32", gate="all"), "f32")


@pytest.mark.parametrize("n,h,dtype,shift", [(600, 8200, "bf16", 1), (523, 8193, "bf16", 0), (300, 16383, "bf16", 3), (270, 16379, "bf16", 0), (301, 8196, "f32", 0), (280, 9001, "f32", 1),
                                             (265, 16381, "f32", 2), (400, 4097, "f32", 0), (300, 8191, "f32", 0), (530, 4095, "bf16", 0), (520, 4090, "bf16", 5), (1100, 1001, "bf16", 0),
                                             (257, 127, "bf16", 1), (263, 255, "bf16", 7), (261, 1021, "f32", 3)])
def test_more_rows_than_workgroups(n, h, dtype, shift):
    """Widths about the places where a row's lanes or its kernel change, several rows to a workgroup and to its columns' sums"""
    _check(*_run(n, h, dtype, gate="all", shift=shift), dtype)
    _check(*_run(n, h, dtype, gate=None if h % 2 else "row", post=h % 3 != 0, ds=False, shift=shift), dtype)


def test_scale_zero_and_eps():
    _check(*_run(6, 300, "f32", res=0.0), "f32")
    _check(*_run(6, 300, "bf16", res=-2.5, eps=0.5), "bf16")
    x = torch.zeros(3, 320, device="cuda")
    Y, S, _, rs = ps.psattn_gatednorm_fwd(x, x, x[0] + 1, eps=0.25)
    assert torch.all(Y == 0) and torch.all(S == 0) and torch.all(rs == 2.0)


@pytest.mark.parametrize("h", [64, 1001, 4096, 20000])
def test_not_finite_keeps_to_its_row(h):
    rng = np.random.default_rng(1)
    t = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(torch.bfloat16).cuda()
    X, B, g, dY, w = t(6, h), t(6, h), t(6, h), t(6, h), t(h)

    def rows(X, B, g):
        Y, S, rb, rs = ps.psattn_gatednorm_fwd(X, B, w, w_post=w, gate=g)
        dX, dB, _, _, dg = ps.psattn_gatednorm_bwd(B, S, w, rb, rs, dY, w_post=w, gate=g)
        return Y, S, dX, dB, dg

    good = rows(X, B, g)
    X2, B2, g2 = X.clone(), B.clone(), g.clone()
    X2[1, h // 2], B2[2, 0], g2[4, h - 1] = float("nan"), float("inf"), float("nan")
    for a, b in zip(good, rows(X2, B2, g2)):
        keep = [0, 3, 5]
        assert torch.equal(a[keep], b[keep])
        assert not torch.isfinite(b[[1, 2, 4]]).all()


def test_no_rows():
    x, w = torch.empty(0, 24, device="cuda"), torch.ones(24, device="cuda")
    Y, S, rb, rs = ps.psattn_gatednorm_fwd(x, x, w, w_post=w, gate=w)
    assert Y.shape == (0, 24)
    dX, dB, dwp, dwo, dg = ps.psattn_gatednorm_bwd(x, S, w, rb, rs, x, w_post=w, gate=w * float("inf"), dw_pre=w + 1, dw_post=w + 1, dgate=w + 1)
    assert torch.all(dwp == 0) and torch.all(dwo == 0) and torch.all(dg == 0)


def test_repeated_calls_and_rows_by_themselves():
    """The same bits again, and a row's results whatever rows stand beside it."""
    a, got = _run(64, 520, "bf16", gate="all")
    _, again = _run(64, 520, "bf16", gate="all")
    for k in got:
        assert torch.equal(got[k], again[k]), k
    t = lambda k, r=slice(None): torch.from_numpy(a[k][r] if a[k].ndim == 2 else a[k]).to(torch.bfloat16).cuda()
    Y, S, rb, rs = ps.psattn_gatednorm_fwd(t("X", slice(9, 10)), t("B", slice(9, 10)), t("w_pre"), w_post=t("w_post"), gate=t("gate", slice(9, 10)), res_scale=0.875)
    assert torch.equal(Y, got["Y"][9:10]) and torch.equal(S, got["S"][9:10]) and torch.equal(rs, got["rs"][9:10])


def test_refusals_of_the_binding():
    x, w = torch.zeros(4, 16, device="cuda"), torch.ones(16, device="cuda")
    fwd, bwd = ps.psattn_gatednorm_fwd, ps.psattn_gatednorm_bwd
    for call in (lambda: fwd(x, None, w, w_post=w), lambda: fwd(x, None, w, gate=w), lambda: fwd(x, None, w, S=x), lambda: fwd(x, x, None),
                 lambda: fwd(x, x, w, gate=torch.ones(3, 16, device="cuda")), lambda: fwd(x, x, w, rstd_b=w[:4]), lambda: fwd(x, x[:3], w), lambda: fwd(x, x, w[:8]),
                 lambda: bwd(x, x, w, None, w[:4], x, w_post=w), lambda: bwd(x, x, w, w[:4], w[:4], x), lambda: bwd(None, x, w, None, w[:4], x, gate=w),
                 lambda: bwd(x, x, w, None, w[:4], None), lambda: bwd(x, x, w, None, w[:4], x, dgate=w), lambda: fwd(x.T, x.T, w[:4])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        fwd(x, x, w.bfloat16())
