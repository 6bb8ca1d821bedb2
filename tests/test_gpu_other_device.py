"""Plans and rotary tables of another device than the current one are refused.  There may be one device only: the handle's own number is changed,
and what it holds stays where it is."""
import ctypes as C

import pytest
import torch

import paper_2410_20305_amd as ps
from test_head_norm_rope_refusals import _Plan, _Rope

pytestmark = pytest.mark.gpu


class _Elsewhere:
    def __init__(self, kind, owner):
        h = owner.handle
        self.at = kind.from_address(h.value if isinstance(h, C.c_void_p) else h)

    def __enter__(self):
        assert self.at.device == torch.cuda.current_device()
        self.at.device += 1

    def __exit__(self, *e):
        self.at.device -= 1


def test_a_plan():
    plan = ps.LogprobPlan([0], [2], [0, 2], [3, 4], 9)
    X, W, ids = torch.randn(9, 32, device="cuda"), torch.randn(40, 32, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda")
    lse, logp = ps.psattn_head_logprob_fwd(plan, X, W, ids)
    dX, dW = torch.full_like(X, 7.0), torch.full_like(W, 7.0)
    with _Elsewhere(_Plan, plan):
        for call in (lambda: ps.psattn_head_logprob_fwd(plan, X, W, ids), lambda: ps.psattn_head_logprob_bwd(plan, X, W, ids, lse, logp, dX=dX, dW=dW)):
            with pytest.raises(ps.PsattnError) as e:
                call()
            assert e.value.status == -1
    torch.cuda.synchronize()
    assert torch.all(dX == 7) and torch.all(dW == 7)
    again, _ = ps.psattn_head_logprob_fwd(plan, X, W, ids)
    assert torch.equal(lse, again)


def test_a_rotary_table():
    rope = ps.Rope(64, 10000.0, 16, layout="half")
    Q, pos = torch.randn(4, 2, 64, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")
    out = torch.full_like(Q, 7.0)
    with _Elsewhere(_Rope, rope):
        for call in (ps.psattn_rope_apply, ps.psattn_rope_apply_bwd):
            with pytest.raises(ps.PsattnError) as e:
                call(rope, Q, None, pos, None, out)
            assert e.value.status == -1
    torch.cuda.synchronize()
    assert torch.all(out == 7)
