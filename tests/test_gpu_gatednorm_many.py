"""RMS norms before and after a block: as many rows as take another number of workgroups in the backward, and tensors of 2^31 elements and more."""
import pytest
import torch

import paper_2410_20305_amd as ps
from block_util import HALF
from test_gpu_gatednorm import _check, _run

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24


@pytest.mark.parametrize("n,h,dtype,gate,shift", [(26623, 72, "bf16", "row", 0), (26624, 72, "bf16", "row", 0), (27001, 300, "bf16", "all", 0), (26699, 1001, "bf16", "row", 1), (27003, 129, "f32", "all", 3),
                                                  (27001, 600, "f32", None, 0), (26627, 2053, "f32", "row", 0), (26630, 4104, "bf16", "row", 0)])
def test_more_rows_than_one_round_of_workgroups(n, h, dtype, gate, shift):
    _check(*_run(n, h, dtype, gate=gate, shift=shift), dtype)


@pytest.mark.parametrize("h", [8200, 8203])
def test_tensors_of_more_than_2_31_elements(h):
    """The last rows as a call of their own gives them, bit for bit; the weight's gradient against its sum in 64 bits."""
    n, last = (1 << 31) // h + 300, 100
    g = torch.Generator(device="cuda").manual_seed(h)

    def rnd(*shape):
        t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        for at in range(0, shape[0], 1 << 14):
            t[at:at + (1 << 14)] = torch.randn(t[at:at + (1 << 14)].shape, generator=g, device="cuda")
        return t

    X, B, gate, dY, w_pre, w_post = rnd(n, h), rnd(n, h), rnd(n, h), rnd(n, h), rnd(h), rnd(h)
    form = dict(w_post=w_post, res_scale=0.5)
    Y, S, rb, rs = ps.psattn_gatednorm_fwd(X, B, w_pre, gate=gate, **form)
    dX, dB, dw_pre, _, dgate = ps.psattn_gatednorm_bwd(B, S, w_pre, rb, rs, dY, gate=gate, **form)
    x, b, k, dy = (t[-last:].clone() for t in (X, B, gate, dY))
    y, s, rb2, rs2 = ps.psattn_gatednorm_fwd(x, b, w_pre, gate=k, **form)
    dx, db, _, _, dk = ps.psattn_gatednorm_bwd(b, s, w_pre, rb2, rs2, dy, gate=k, **form)
    for whole, part in ((Y, y), (S, s), (dX, dx), (dB, db), (dgate, dk), (rb, rb2), (rs, rs2)):
        assert torch.equal(whole[-last:], part)
    want, size = torch.zeros(h, dtype=torch.float64, device="cuda"), torch.zeros(h, dtype=torch.float64, device="cuda")
    for at in range(0, n, 1 << 13):
        part = dY[at:at + (1 << 13)].double() * S[at:at + (1 << 13)].double() * rs[at:at + (1 << 13), None].double()
        want += part.sum(0)
        size += part.abs().sum(0)
    # at most 1 024 workgroups' rows in a chain of each, then 64 of those: n / 256 + 80 additions and more than there are
    tol = HALF["bf16"] * want.abs() + (n / 256 + 80) * EPS32 * size
    assert ((dw_pre.double() - want).abs() <= tol).all()
