"""The feed-forward block's largest tiles where operands go through registers: bf16 widths that are no whole 16-byte groups with few
tokens, and fp32.  Whole numbers, whose sums are exact, against torch's products in fp64."""
import pytest
import torch

import paper_2410_20305_amd as ps

pytestmark = pytest.mark.gpu

# sizes for which the launch model takes tiles of 256 x 256, with k in parts and without, in each product: bf16 gate and up, dG and dU (132,
# 583, 59268 unsplit), dX, Y and the gradients of weights; fp32 gate and up, dG and dU, dWg and dWu, Y and dX, dWd
CASES = [("bf16", 221, 2371, 27776), ("bf16", 300, 2047, 6001), ("bf16", 132, 583, 59268), ("bf16", 134, 8699, 1044), ("bf16", 65, 135, 20781), ("bf16", 67, 298, 22095),
         ("f32", 138, 495, 8663), ("f32", 770, 384, 4614), ("f32", 76, 769, 7013), ("f32", 471, 139, 8214), ("f32", 2691, 4447, 106), ("f32", 774, 4722, 487),
         ("f32", 65, 3778, 3284), ("f32", 506, 403, 8193), ("f32", 2048, 2048, 4104)]


@pytest.mark.parametrize("dtype,T,h,n", CASES)
def test_whole_numbers_are_exact(dtype, T, h, n):
    gen = torch.Generator(device="cuda").manual_seed(T + n)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def whole(rows, cols, factor=1, least=-1):
        few = torch.rand(rows, cols, generator=gen, device="cuda") < 0.25
        return (torch.randint(least, 2, (rows, cols), generator=gen, device="cuda") * few * factor).to(dt)

    hold = lambda x: x.to(dt)
    # gates are open (64 and more: SiLU is the identity there) or exactly 0
    X, Wg, Wu, Wd, dY = whole(T, h, least=0), whole(n, h, 64, least=0), whole(n, h), whole(h, n), whole(T, h)
    x, wg, wu, wd, dy = (t.double() for t in (X, Wg, Wu, Wd, dY))
    Y, (G, U, H) = ps.psattn_ffn_fwd(X, Wg, Wu, Wd)
    g, u = x @ wg.T, x @ wu.T
    assert torch.equal(G.double(), g) and torch.equal(U.double(), u)
    assert torch.equal(H, hold(g * u)) and torch.equal(Y, hold(H.double() @ wd.T))
    kG = torch.where(torch.rand(T, n, generator=gen, device="cuda") < 0.5, 64.0, 0.0)   # derivatives 1 and 1/2
    kU = torch.where(torch.rand(T, n, generator=gen, device="cuda") < 0.5, 2.0, -2.0)
    kH = whole(T, n, 2)
    dX, dWg, dWu, dWd = ps.psattn_ffn_bwd(X, Wg, Wu, Wd, (kG, kU, kH), dY)
    dH = dy @ wd
    dG, dU = hold(dH * kU * torch.where(kG > 0, 1.0, 0.5)).double(), hold(dH * kG).double()
    assert torch.equal(dWd, hold(dy.T.contiguous() @ kH.double()))
    assert torch.equal(dWg, hold(dG.T.contiguous() @ x)) and torch.equal(dWu, hold(dU.T.contiguous() @ x))
    assert torch.equal(dX, hold(dG @ wg + dU @ wu))
