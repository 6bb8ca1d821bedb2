"""Plans of the log-probability heads: what they hold, and items found among many responses, empty ones and empty prompts too."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps
import test_gpu_head as head

pytestmark = pytest.mark.gpu


def test_a_plan_holds_two_numbers_to_a_token():
    """A descriptor of each token and the rows that predict: a plan is made for each batch, and what only one of the heads would read is not in it."""
    T = 32 << 20
    ps.LogprobPlan([0], [1], [0, 1], [1], 2)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    plan = ps.LogprobPlan([0], [1], [0, 1], [T - 1], T)
    held = free - torch.cuda.mem_get_info()[0]
    assert 2 * 4 * T - (1 << 20) <= held <= 2 * 4 * T + (16 << 20), held
    del plan


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seed,samples", [(0, 1), (1, 3), (2, 40), (3, 150)])
def test_items_of_many_responses(seed, samples, dtype, monkeypatch):
    rng = np.random.default_rng(seed)
    off, prompt, ptr, lens, at = [], [], [0], [], 0
    for _ in range(samples):
        at += int(rng.integers(0, 3))
        off.append(at)
        p = int(rng.choice([0, 1, 2, 9]))
        more = [int(n) for n in rng.choice([0, 0, 1, 1, 2, 7], int(rng.integers(0, 9)))]
        if p + sum(more) == 0:
            p = 1
        prompt.append(p)
        lens += more
        ptr.append(len(lens))
        at += p + sum(more)
    lens[-1:] = [lens[-1] + 5]
    monkeypatch.setitem(head.TABLES, "random", (off, prompt, ptr, lens, at + 9))
    a = head._inputs("random", 150, 72, dtype)
    assert len(a[3]) > 0
    head._check(*a, head._call("random", *a[:3], a[4], dtype), dtype)
