"""The feed-forward block on sizes that take many workgroups of the largest tiles, tiles at both edges and k in parts: whole numbers, whose
sums are exact, against torch's products in fp64."""
import pytest
import torch

import paper_2410_20305_amd as ps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,h,n,shift", [(4099, 1544, 4104, 0), (2048, 2048, 8192, 0), (1500, 776, 6152, 0), (2309, 1031, 3007, 0), (1024, 1024, 4096, 1), (90, 2056, 7000, 0),
                                         (300, 4096, 520, 0), (9000, 264, 264, 0)])
def test_whole_numbers_are_exact(T, h, n, shift):
    gen = torch.Generator(device="cuda").manual_seed(T)

    def whole(rows, cols, factor=1):
        buf = torch.zeros(rows * cols + 8, dtype=torch.bfloat16, device="cuda")
        t = buf[shift:shift + rows * cols].view(rows, cols)
        t.copy_(torch.randint(-1, 2, (rows, cols), generator=gen, device="cuda") * (torch.rand(rows, cols, generator=gen, device="cuda") < 0.25) * factor)
        return t

    X, Wg, Wu, Wd, dY = whole(T, h), whole(n, h, 64), whole(n, h), whole(h, n), whole(T, h)
    bf = lambda x: x.to(torch.bfloat16)
    x, wg, wu, wd, dy = (t.double() for t in (X, Wg, Wu, Wd, dY))
    Y, (G, U, H) = ps.psattn_ffn_fwd(X, Wg, Wu, Wd)
    g, u = x @ wg.T, x @ wu.T
    assert torch.equal(G.double(), g) and torch.equal(U.double(), u)
    want = torch.where(g > 0, g * u, 0.0)
    assert torch.equal(torch.where(H.abs() < 1e-20, 0.0, H.double()), bf(want).double())
    # the backward's own inputs: gates of 64 are open (their derivative is 1), gates of 0 have 1/2
    kG = torch.where(torch.rand(T, n, generator=gen, device="cuda") < 0.5, 64.0, 0.0)
    kU = torch.where(torch.rand(T, n, generator=gen, device="cuda") < 0.5, 2.0, -2.0)
    kH = whole(T, n, 2)
    dX, dWg, dWu, dWd = ps.psattn_ffn_bwd(X, Wg, Wu, Wd, (kG, kU, kH), dY)
    dH = dy @ wd
    dG, dU = bf(dH * kU * torch.where(kG > 0, 1.0, 0.5)).double(), bf(dH * kG).double()
    assert torch.equal(dWd, bf(dy.T.contiguous() @ kH.double()))
    assert torch.equal(dWg, bf(dG.T.contiguous() @ x)) and torch.equal(dWu, bf(dU.T.contiguous() @ x))
    assert torch.equal(dX, bf(dG @ wg + dU @ wu))
    # Y from an H of whole numbers: all gates open or shut at exactly 0
    Wp = Wg.abs()
    Xp = X.abs()
    Y, (G, _, H) = ps.psattn_ffn_fwd(Xp, Wp, Wu, Wd)
    g, u = Xp.double() @ wg.abs().T, Xp.double() @ wu.T
    assert torch.equal(H, bf(g * u)) and torch.equal(Y, bf(bf(g * u).double() @ wd.T))


def test_offsets_past_32_bits():
    """G, U, H of 70 000 x 31 000: 4.3 GB in bf16, 8.7 in fp32."""
    T, h, n = 70000, 64, 31000
    gen = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randint(0, 2, (T, h), generator=gen, device="cuda").bfloat16()
    W = torch.randint(0, 2, (n, h), generator=gen, device="cuda").bfloat16()
    Wd = torch.zeros(h, n, dtype=torch.bfloat16, device="cuda")
    Wd[:, n - 1] = 1
    Wd[:, 0] = 1
    Y, (G, U, H) = ps.psattn_ffn_fwd(X, W * 64, W, Wd)
    rows = torch.tensor([0, 1, T // 2, T - 2, T - 1], device="cuda")
    u = X[rows].double() @ W.double().T
    assert torch.equal(U[rows].double(), u) and torch.equal(G[rows].double(), u * 64)
    h0 = (u * u * 64).bfloat16()
    assert torch.equal(H[rows], h0)
    assert torch.equal(Y[rows], (h0[:, :1].double() + h0[:, -1:].double()).bfloat16().expand(-1, h))
    del G, U, H


def test_few_columns_and_rows():
    """Sizes below one 16-byte group, and one token beside a large block."""
    for T, h, n in ((5, 3, 2), (1, 1, 9000), (70, 2, 3), (1, 9000, 1), (130, 5, 1)):
        gen = torch.Generator(device="cuda").manual_seed(T)
        X, W, Wd = (torch.randint(0, 2, s, generator=gen, device="cuda").bfloat16() for s in ((T, h), (n, h), (h, n)))
        Y, (G, U, H) = ps.psattn_ffn_fwd(X, W * 64, W, Wd)
        u = X.double() @ W.double().T
        assert torch.equal(U.double(), u) and torch.equal(H, (u * u * 64).bfloat16()) and torch.equal(Y, (H.double() @ Wd.double().T).bfloat16())
