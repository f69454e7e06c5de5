"""Top-k of key lists longer than the final block sorts at once (16,384 keys): pass 1 of the reduction prunes in every block."""
from __future__ import annotations

import numpy as np
import pytest

from helpers import variant

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,k", [(40_000, 1024), (70_000, 1000), (33_000, 512)])
def test_long_key_lists_rank_alike_call_after_call(n, k):
    """A survivor list that repeats a few thousand plans: the simulator's scores of n entries leave more than 16,384 keys,
    2 to 5 tiles a block.  The ranking is (score falling, position rising) of the call's own scores, every time."""
    import torch
    from paper_2607_18631_b200 import Plan
    plan = Plan(variant("mid", cluster=dict(budget_bytes=10 ** 15), rules=dict(enforce_realizability=0)))
    out = plan.score(k=0)
    sel = plan.select_survivors(out["reason"], out["tput"], 3000)
    base = sel["surv_idx"][:int(sel["surv_count"].item())]
    surv = base.repeat(-(-n // base.numel()))[:n].contiguous()
    first = plan.simulate(surv, n, 4, k=k)
    torch.cuda.synchronize()
    score = first["tput_sim"][:n].cpu().numpy()
    order = np.argsort(-score, kind="stable")[:k]
    assert int(first["topk_count"].item()) == k and score[order[-1]] > 0
    np.testing.assert_array_equal(first["topk_score"][:k].cpu().numpy(), score[order])
    np.testing.assert_array_equal(first["topk_idx"][:k].cpu().numpy(), surv.cpu().numpy()[order])
    for _ in range(100):
        again = plan.simulate(surv, n, 4, k=k)
        assert torch.equal(again["topk_idx"][:k], first["topk_idx"][:k]) and torch.equal(again["topk_score"][:k], first["topk_score"][:k])
    plan.close()
