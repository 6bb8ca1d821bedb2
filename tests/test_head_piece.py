"""Vocabulary head, backward: the workspace of few predicted tokens and a vocabulary of many millions (CPU only).  dz stands there in rows of a piece of
the vocabulary, 64 of them at least, which the products' copies reach by 32-bit offsets."""
import pytest

import paper_2410_20305_amd as ps
from test_head_norm_rope_refusals import BF16, F32, _Plan, a_plan

LIB = ps.load_library()


@pytest.mark.parametrize("dt,size", [(BF16, 2), (F32, 4)])
@pytest.mark.parametrize("n", [0, 1, 2, 31, 32, 33, 63, 64, 65, 200])
@pytest.mark.parametrize("vocab", [3_000_000, 34_100_000, 200_000_000, 2_000_000_000])
def test_few_items_of_a_large_vocabulary(dt, size, n, vocab):
    plan = _Plan(T=1000, n_samples=1, n_resp=2, n_rows=n, n_items=n)
    room = LIB.psattn_head_logprob_bwd_workspace_bytes(a_plan(plan), dt, vocab, 8)
    # a piece of dz, dX's and the logits' and dW's sums in parts (64 MiB each at most), an item of each token, the rest small
    assert 0 < room <= (512 << 20) + 4 * (64 << 20) + (4 * vocab if dt == BF16 and n > 32 else 0), room / 2 ** 20
