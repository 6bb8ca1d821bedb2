"""Workspaces of the embedding's, layer norm's and feed-forward block's calls: whatever they hold on entry, wherever they start, nothing
behind their end is written."""
import pytest
import torch

import paper_2410_20305_amd as ps

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GUARD = 4096
F32, BF16 = 0, 1


def _code(dtype):
    return BF16 if dtype == torch.bfloat16 else F32


def _same_whatever_it_holds(need, call):
    """`call(workspace)` gives the same bits with workspaces of zeros and of NaN, on a boundary and off it, of just `need` bytes."""
    want = None
    for fill, shift in ((0x00, 0), (0xFF, 0), (0xFF, 8), (0x7F, 4)):
        buf = torch.full((GUARD + need + GUARD,), fill, dtype=torch.uint8, device="cuda")
        ends = [buf[:GUARD + shift], buf[GUARD + shift + need:]]
        for e in ends:
            e.fill_(0xA5)
        got = call(buf[GUARD + shift:GUARD + shift + need])
        assert all(bool((e == 0xA5).all()) for e in ends), "written outside"
        assert all(bool(torch.isfinite(t).all()) for t in got)
        if want is None:
            want = got
        for a, b in zip(want, got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,h,n", [(1, 64, 128), (3, 4096, 520), (40, 65, 131), (221, 512, 1000), (330, 33, 65), (700, 129, 1000), (1037, 1001, 331),
                                   (4100, 520, 1032)])
def test_feed_forward(T, h, n, dtype):
    g = torch.Generator(device="cuda").manual_seed(T + h)
    X, Wg, Wu, Wd, dY = (torch.randn(*s, generator=g, device="cuda").to(DTYPES[dtype]) for s in ((T, h), (n, h), (n, h), (h, n), (T, h)))
    lib, dt = ps.load_library(), _code(X.dtype)

    def forward(ws):
        Y, kept = ps.psattn_ffn_fwd(X, Wg, Wu, Wd, workspace=ws)
        return (Y, *kept)

    _same_whatever_it_holds(lib.psattn_ffn_fwd_workspace_bytes(dt, T, h, n), forward)
    kept = ps.psattn_ffn_fwd(X, Wg, Wu, Wd)[1]
    _same_whatever_it_holds(lib.psattn_ffn_bwd_workspace_bytes(dt, T, h, n), lambda ws: ps.psattn_ffn_bwd(X, Wg, Wu, Wd, kept, dY, workspace=ws))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,h", [(1, 1, 1), (63, 5, 40), (6144, 100, 17), (6145, 7, 130), (9000, 70000, 33)])
def test_embedding_gradient(T, V, h, dtype):
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    dX = torch.randn(T, h, generator=g, device="cuda").to(DTYPES[dtype])
    need = ps.load_library().psattn_embed_bwd_workspace_bytes(_code(dX.dtype), T, V, h)
    _same_whatever_it_holds(need, lambda ws: (ps.psattn_embed_bwd(ids, dX, V, workspace=ws),))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,h", [(1, 1), (5, 1001), (300, 64), (2331, 1001), (70, 9001), (9, 20000)])
def test_layer_norm_gradient(T, h, dtype):
    g = torch.Generator(device="cuda").manual_seed(h)
    X, dY = (torch.randn(T, h, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    w = torch.randn(h, generator=g, device="cuda").to(DTYPES[dtype])
    _, S, mean, rstd = ps.psattn_layernorm_fwd(X, w, w)
    need = ps.load_library().psattn_layernorm_bwd_workspace_bytes(T, h)
    _same_whatever_it_holds(need, lambda ws: ps.psattn_layernorm_bwd(S, w, mean, rstd, dY, workspace=ws))


def test_backward_without_what_the_forward_keeps():
    X, W, Wd = torch.zeros(4, 16, device="cuda"), torch.zeros(32, 16, device="cuda"), torch.zeros(16, 32, device="cuda")
    kept = ps.psattn_ffn_fwd(X, W, W, Wd, keep=False)[1]
    with pytest.raises(ValueError, match="keep"):
        ps.psattn_ffn_bwd(X, W, W, Wd, kept, X)
