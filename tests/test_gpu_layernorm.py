"""Layer norm (with the residual sum) and its gradients against the 64-bit oracle."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import HALF, Guarded, close, hold, np64, rnd
from oracle import psattn_block_oracle as blk

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24


def _run(n, h, dtype, residual, bias, seed=0, shift=0, eps=1e-5, offset=0.1, scale=1.0):
    rng = np.random.default_rng(n * 13 + h + seed)
    X = rnd(rng, n, h, scale=scale, shift=offset, dtype=dtype)
    R = rnd(rng, n, h, scale=2.0, dtype=dtype) if residual else None
    w, b = rnd(rng, h, scale=0.3, shift=1.0, dtype=dtype), rnd(rng, h, scale=0.5, dtype=dtype) if bias else None
    dY, dS = rnd(rng, n, h, dtype=dtype), rnd(rng, n, h, dtype=dtype) if residual else None
    dev = Guarded(dtype, shift)
    put = lambda x: None if x is None else dev.put(x)
    f32 = lambda: dev.empty(n, dtype=torch.float32)
    tw = put(w)
    Y, S, mean, rstd = ps.psattn_layernorm_fwd(put(X), tw, put(b), eps, residual=put(R), S=dev.empty(n, h) if residual else None,
                                               Y=dev.empty(n, h), mean=f32(), rstd=f32())
    dX, dw, db = ps.psattn_layernorm_bwd(S, tw, mean, rstd, put(dY), dS=put(dS), bias=bias, dX=dev.empty(n, h), dweight=dev.empty(h),
                                         dbias=dev.empty(h) if bias else None)
    dev.check()
    held = X if R is None else hold(dtype)(X + R)
    return dict(X=X, S=held, w=w, b=b, dY=dY, dS=dS, eps=eps), dict(Y=Y, S=S, mean=mean, rstd=rstd, dX=dX, dw=dw, db=db)


def _check(a, got, dtype):
    """Error bounds.  A row's sums of h terms run in chains of at most c = h / 64 + 24 additions (64 lanes and more, then a
    tree).  d_mean <= c 2^-24 mean|s|; a centred value is off by d = d_mean + 2^-24 |s - mean|; rstd by r (c + 4) 2^-24 + r^2 d
    relatively, as the variance's terms are off by 2 d each.  From there on products and sums add up."""
    S, w, b, dY, dS, eps = (a[k] for k in ("S", "w", "b", "dY", "dS", "eps"))
    n, h = S.shape
    half, c = HALF[dtype], h / 64 + 24
    if "X" in a and got["S"] is not None:
        assert np.array_equal(np64(got["S"]), S)
    Y, mean, rstd = blk.layernorm(S, w, b, eps)
    cen = S - mean[:, None]
    d_mean = c * EPS32 * np.abs(S).mean(1)
    d = d_mean[:, None] + EPS32 * np.abs(cen)
    close(got["mean"], mean, d_mean + EPS32 * np.abs(mean), "mean")
    r_rel = (c + 4) * EPS32 + rstd ** 2 * (2 * np.abs(cen) * d).mean(1)
    close(got["rstd"], rstd, rstd * r_rel, "rstd")
    xh = cen * rstd[:, None]
    d_xh = rstd[:, None] * d + np.abs(xh) * (r_rel[:, None] + 2 * EPS32)
    close(got["Y"], Y, half * np.abs(Y) + (1 + half) * (np.abs(w) * d_xh + 3 * EPS32 * (np.abs(xh * w) + (0 if b is None else np.abs(b)))), "Y")
    dX, dw, db = blk.layernorm_grad(S, w, eps, dY, dS)
    q = dY * w
    m1, m2 = np.abs(q).mean(1)[:, None], np.abs(q * xh).mean(1)[:, None]
    d1 = (c + 2) * EPS32 * m1
    d2 = (c + 4) * EPS32 * m2 + (np.abs(q) * d_xh).mean(1)[:, None]
    inner = np.abs(q) + m1 + np.abs(xh) * m2
    d_in = d1 + d_xh * m2 + np.abs(xh) * d2 + 6 * EPS32 * inner
    tol = rstd[:, None] * (d_in + inner * r_rel[:, None]) + (0 if dS is None else 2 * EPS32 * (np.abs(dS) + rstd[:, None] * inner))
    close(got["dX"], dX, half * np.abs(dX) + (1 + half) * tol, "dX")
    # sums over rows: one rounding per addition, at most n of them, never more than some hundreds in a chain
    chain = min(n, 600) + 8
    close(got["dw"], dw, half * np.abs(dw) + (1 + half) * ((np.abs(dY) * d_xh).sum(0) + chain * EPS32 * np.abs(dY * xh).sum(0)), "dw")
    if b is not None:
        close(got["db"], db, half * np.abs(db) + (1 + half) * chain * EPS32 * np.abs(dY).sum(0), "db")


SHAPES = [(1, 1), (1, 2), (3, 7), (1, 64), (5, 63), (2, 65), (70, 128), (33, 130), (129, 256), (64, 257), (9, 511), (300, 512), (7, 1000), (40, 1001),
          (17, 1024), (3, 1026), (19, 2048), (5, 2050), (11, 4096), (2, 4104), (3, 8192), (2, 8200), (2, 16384), (3, 16392), (2, 20001), (1, 65536)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,h", SHAPES)
def test_against_oracle(n, h, dtype):
    _check(*_run(n, h, dtype, residual=(n + h) % 2 == 0, bias=h % 3 != 0), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("bias", [False, True])
def test_every_form(dtype, residual, bias):
    _check(*_run(37, 768, dtype, residual, bias), dtype)


@pytest.mark.parametrize("n,h,shift", [(5, 256, 1), (9, 4096, 3), (4, 1000, 2), (3, 8192, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unaligned_rows(n, h, shift, dtype):
    _check(*_run(n, h, dtype, True, True, shift=shift), dtype)


@pytest.mark.parametrize("n", [2, 255, 1023, 4096, 20011])
def test_many_rows(n):
    _check(*_run(n, 96, "bf16", True, True), "bf16")
    _check(*_run(n, 40, "f32", False, True), "f32")


def test_far_from_zero():
    """Rows whose mean is 1 000 times their spread: the squares are those of the centred values."""
    _check(*_run(20, 1024, "f32", False, True, offset=1000.0), "f32")


def test_constant_rows_and_eps():
    x = torch.full((3, 320), 2.5, device="cuda")
    w, b = torch.full((320,), 3.0, device="cuda"), torch.full((320,), 0.25, device="cuda")
    Y, _, mean, rstd = ps.psattn_layernorm_fwd(x, w, b, eps=0.25)
    assert torch.all(Y == 0.25) and torch.all(mean == 2.5) and torch.all(rstd == 2.0)
    assert torch.isnan(ps.psattn_layernorm_fwd(x, w, b, eps=0.0)[0]).all()  # 0 times infinity, as the formula has it


@pytest.mark.parametrize("h", [64, 1001, 4096, 20000])
def test_not_finite_keeps_to_its_row(h):
    rng = np.random.default_rng(1)
    X = torch.from_numpy(rng.standard_normal((6, h))).to(torch.bfloat16).cuda()
    w = torch.ones(h, dtype=torch.bfloat16, device="cuda")
    dY = torch.ones_like(X)
    good = ps.psattn_layernorm_fwd(X, w)
    g = ps.psattn_layernorm_bwd(X, w, good[2], good[3], dY, bias=False)[0]
    bad = X.clone()
    bad[2, h // 2], bad[4, 0] = float("nan"), float("inf")
    Y, _, mean, rstd = ps.psattn_layernorm_fwd(bad, w)
    dX = ps.psattn_layernorm_bwd(bad, w, mean, rstd, dY, bias=False)[0]
    keep = [0, 1, 3, 5]
    assert torch.equal(Y[keep], good[0][keep]) and torch.equal(dX[keep], g[keep])
    assert torch.isnan(Y[2]).all() and torch.isnan(Y[4]).all() and torch.isnan(dX[2]).all()


def test_repeats_bit_for_bit():
    rng = np.random.default_rng(2)
    X = torch.from_numpy(rng.standard_normal((5000, 520))).to(torch.bfloat16).cuda()
    w = torch.ones(520, dtype=torch.bfloat16, device="cuda")
    Y, _, mean, rstd = ps.psattn_layernorm_fwd(X, w, w)
    need = ps.load_library().psattn_layernorm_bwd_workspace_bytes(5000, 520)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    first = ps.psattn_layernorm_bwd(X, w, mean, rstd, Y, workspace=ws)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, ps.psattn_layernorm_bwd(X, w, mean, rstd, Y, workspace=ws)))


def test_no_rows():
    w = torch.ones(12, device="cuda")
    none = torch.empty(0, 12, device="cuda")
    Y, S, mean, rstd = ps.psattn_layernorm_fwd(none, w)
    assert Y.shape == (0, 12) and mean.shape == (0,)
    dw, db = torch.full((12,), float("nan"), device="cuda"), torch.full((12,), float("nan"), device="cuda")
    ps.psattn_layernorm_bwd(none, w, mean, rstd, none, dweight=dw, dbias=db)
    assert torch.all(dw == 0) and torch.all(db == 0)


def test_refusals_on_the_device():
    X, w = torch.zeros(4, 16, device="cuda"), torch.zeros(16, device="cuda")
    st = torch.zeros(4, device="cuda")
    with pytest.raises(ValueError):
        ps.psattn_layernorm_fwd(X, w[:8])
    with pytest.raises(TypeError):
        ps.psattn_layernorm_fwd(X, w.bfloat16())
    with pytest.raises(ValueError):
        ps.psattn_layernorm_fwd(X[:, ::2], w[:8])
    with pytest.raises(ValueError):
        ps.psattn_layernorm_fwd(X, w, S=torch.empty_like(X))
    with pytest.raises(ps.PsattnError):
        ps.psattn_layernorm_fwd(X, w, eps=-1.0)
    with pytest.raises(ValueError):
        ps.psattn_layernorm_bwd(X, w, st, st, X, bias=False, dbias=w)
    with pytest.raises(ValueError):
        ps.psattn_layernorm_bwd(X, w, st[:3], st, X)
