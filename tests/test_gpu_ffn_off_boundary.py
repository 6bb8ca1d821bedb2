"""The feed-forward block on tensors of which some start off a 16-byte boundary, with the workspace that copies them and with the one
that does not; and with one width that is whole and one that is not.  Whole numbers: every way gives the same bits."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps

pytestmark = pytest.mark.gpu

OPERANDS = ("X", "Wg", "Wu", "Wd", "H", "dY")
RESULTS = ("Y", "G", "U", "dX", "dWg", "dWu", "dWd")


def _tensors(T, h, n):
    rng = np.random.default_rng(T + h + n)
    whole = lambda *s: np.where(rng.uniform(size=s) < 0.25, rng.integers(-1, 2, s), 0)
    X, Wg, Wu, Wd, dY = np.abs(whole(T, h)), np.abs(whole(n, h)) * 64, whole(n, h), whole(h, n), whole(T, h)
    return dict(X=X, Wg=Wg, Wu=Wu, Wd=Wd, dY=dY)


def _place(shape, dtype, off, guard):
    n = int(np.prod(shape))
    buf = torch.full((n + 80,), 7.0, dtype=dtype, device="cuda")
    at = 32 + (3 if off else 0)
    guard.append((buf, at, n))
    return buf[at:at + n].view(shape)


def _run(d, off, roomy):
    """Forward and backward with the tensors named in `off` off a boundary, on workspaces of just the bytes asked for."""
    guard = []
    (T, h), n = d["X"].shape, d["Wg"].shape[0]
    bf = torch.bfloat16
    place = lambda name, shape, dt=bf: _place(shape, dt, name in off, guard)
    ins = {}
    for k, v in d.items():
        ins[k] = place(k, v.shape)
        ins[k].copy_(torch.from_numpy(v))
    lib, out = ps.load_library(), []
    ws = lambda f: torch.full((f(ps.BF16, T, h, n) + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    fwd, bwd = (lib.psattn_ffn_fwd_unaligned_workspace_bytes, lib.psattn_ffn_bwd_unaligned_workspace_bytes) if roomy else (lib.psattn_ffn_fwd_workspace_bytes, lib.psattn_ffn_bwd_workspace_bytes)
    wf, wb = ws(fwd), ws(bwd)
    W = (ins["X"], ins["Wg"], ins["Wu"], ins["Wd"])
    kept = (place("G", (T, n), torch.float32), place("U", (T, n), torch.float32), place("H", (T, n)))
    Y, kept = ps.psattn_ffn_fwd(*W, kept=kept, Y=place("Y", (T, h)), workspace=wf[:-512])
    kept[0].clamp_(max=64.0)   # gates of 64 and 0
    grads = ps.psattn_ffn_bwd(*W, kept, ins["dY"], dX=place("dX", (T, h)), dWg=place("dWg", (n, h)), dWu=place("dWu", (n, h)), dWd=place("dWd", (h, n)), workspace=wb[:-512])
    assert bool((wf[-512:] == 0xFF).all()) and bool((wb[-512:] == 0xFF).all()), "written behind the workspace"
    for buf, at, m in guard:
        assert bool((buf[:at] == 7.0).all()) and bool((buf[at + m:] == 7.0).all()), "written outside a tensor"
    return [t.clone() for t in (Y, *kept, *grads)]


def _expected(d):
    x, wg, wu, wd, dy = (torch.from_numpy(d[k]).double().cuda() for k in ("X", "Wg", "Wu", "Wd", "dY"))
    bf = lambda t: t.to(torch.bfloat16)
    g, u = x @ wg.T, x @ wu.T
    H = bf(g * u)
    G = g.clamp(max=64.0)
    dH = dy @ wd
    dG, dU = bf(dH * u * torch.where(G > 0, 1.0, 0.5)).double(), bf(dH * G).double()
    return [bf(H.double() @ wd.T), G.float(), u.float(), H, bf(dG @ wg + dU @ wu), bf(dG.T.contiguous() @ x), bf(dU.T.contiguous() @ x), bf(dy.T.contiguous() @ H.double())]


@pytest.mark.parametrize("roomy", [False, True])
@pytest.mark.parametrize("T,h,n", [(1, 64, 136), (50, 256, 136), (200, 72, 520), (321, 136, 264), (700, 520, 1032), (2100, 264, 2056)])
def test_each_tensor_off_a_boundary(T, h, n, roomy):
    d = _tensors(T, h, n)
    want = _expected(d)
    for off in [(), *[(k,) for k in OPERANDS + RESULTS], OPERANDS, RESULTS, OPERANDS + RESULTS]:
        for a, b in zip(want, _run(d, off, roomy)):
            assert torch.equal(a, b), off


@pytest.mark.parametrize("off", [(), ("Wd", "H"), OPERANDS + RESULTS])
@pytest.mark.parametrize("roomy", [False, True])
@pytest.mark.parametrize("T,h,n", [(1, 256, 131), (20, 131, 256), (50, 256, 131), (60, 77, 520), (130, 264, 333), (319, 333, 264), (330, 264, 131), (700, 131, 520), (1500, 1001, 264)])
def test_one_width_whole(T, h, n, roomy, off):
    d = _tensors(T, h, n)
    for a, b in zip(_expected(d), _run(d, off, roomy)):
        assert torch.equal(a, b)


def test_the_binding_asks_for_the_copies_room():
    """Workspaces that the binding makes: from a tensor off a boundary on, those that copy."""
    d = _tensors(400, 64, 136)
    (T, h), n, bf = d["X"].shape, d["Wg"].shape[0], torch.bfloat16
    lib, guard = ps.load_library(), []
    for off in ((), ("Wu",)):
        t = [_place(d[k].shape, bf, k in off, guard).copy_(torch.from_numpy(d[k])) for k in ("X", "Wg", "Wu", "Wd")]
        torch.cuda.synchronize()
        before = torch.cuda.memory_stats()["requested_bytes.all.allocated"]
        ps.psattn_ffn_fwd(*t)
        asked = torch.cuda.memory_stats()["requested_bytes.all.allocated"] - before
        need = lib.psattn_ffn_fwd_unaligned_workspace_bytes if off else lib.psattn_ffn_fwd_workspace_bytes
        assert asked == 2 * T * h + (4 + 4 + 2) * T * n + need(ps.BF16, T, h, n)
