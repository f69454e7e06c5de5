"""Shared prefixes where a wait inside the kernel runs out: the call ends, and the rows that it concerns are NaN.

The wait is one for something that does not come, with a short limit."""
from __future__ import annotations

import pytest

from test_gpu_prefix_attention import build, run

pytestmark = pytest.mark.gpu


@pytest.fixture
def lost_wait():
    """While it lasts a block of the kernel waits in vain, 500 polls (a millisecond) long."""
    from paper_2607_18631_b200.binding import load_library
    L = load_library()
    yield lambda: L.pf_prefix_waits(500, 1)
    assert L.pf_prefix_waits(0, 0) == 0


@pytest.mark.parametrize("B,heads,n_kv,length,hd", [(3, 8, 2, 600, 128), (200, 8, 2, 4000, 64), (40, 16, 4, 30000, 128)])
def test_a_wait_that_runs_out_leaves_nan(B, heads, n_kv, length, hd, lost_wait):
    import torch
    args = build(n_kv, hd, 64, [B], [length], [i % 50 for i in range(B)], heads)
    want = run(*args)
    assert torch.isfinite(want["out"].float()).all()
    assert lost_wait() == 0
    got = run(*args)
    torch.cuda.synchronize()
    from paper_2607_18631_b200.binding import load_library
    assert load_library().pf_prefix_waits(0, 0) == 0
    again = run(*args)
    # the block takes the list's first tiles: rows of the first key head
    bad = torch.isnan(got["out"].float()).all(-1)
    assert bad[0, 0] and torch.equal(bad, torch.isnan(got["out"].float()).any(-1)) and torch.equal(bad, torch.isnan(got["lse"]))
    assert torch.equal(got["out"][~bad], want["out"][~bad]) and not bad[:, heads // n_kv:].any()
    assert torch.equal(again["out"], want["out"]) and torch.equal(again["lse"], want["lse"])


def test_limits_are_checked():
    from paper_2607_18631_b200.binding import PF_ERANGE, load_library
    L = load_library()
    assert L.pf_prefix_waits((1 << 21) + 1, 0) == PF_ERANGE and L.pf_prefix_waits(0, 2) == PF_ERANGE and L.pf_prefix_waits(0, 0) == 0
