"""pf_prefix_attention: what its other tests say and leave open: rows under offsets that make no sense, and a query that holds an infinity."""
from __future__ import annotations

import pytest

from test_gpu_prefix_attention import build, compare, run

pytestmark = pytest.mark.gpu


def test_offsets_that_make_no_sense_give_what_they_say():
    """Offsets below 0 and past the end are moved there, and a group that ends before it begins has no sequence: rows, against the reference of those groups."""
    q, cache, own, table, plen, ptable, _ = build(2, 64, 16, [4, 4], [100, 90], [9] * 8, 4)
    for cu, sound in (([0, 8, 0], [0, 8, 8]), ([-5, 4, 1 << 30], [0, 4, 8]), ([7, 3, 1], [8, 8, 8]), ([1 << 30, 0, -1], [8, 8, 8])):
        compare(run(q, cache, own, table, plen, ptable, cu), q, cache, own, table, plen, ptable, sound, 0.125)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_becomes_of_a_head_whose_query_is_not_finite(bad):
    """NaN: the prefix's keys have both signs, so a score is an infinity of the one or of the other, or no number."""
    import torch
    args = build(2, 128, 64, [10], [500], [40] * 10, 8)
    q = args[0]
    good = run(*args)
    q[8, 5, 0] = bad
    got = run(*args)
    same = torch.ones(10, 8, dtype=torch.bool, device="cuda")
    same[8, 5] = False
    assert torch.isnan(got["out"][8, 5].float()).all() and torch.isnan(got["lse"][8, 5])
    assert torch.equal(got["out"][same], good["out"][same]) and torch.equal(got["lse"][same], good["lse"][same])
