"""The mixture-of-experts layer where a wait between its blocks runs out: the call ends, says so and leaves no number behind.

The wait is one for an arrival that nobody makes, with a short limit."""
from __future__ import annotations

import pytest

from test_gpu_moe import layer_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture
def lost_block():
    """While it lasts every meeting waits for a block too many, 2,000 polls (some milliseconds) long."""
    from paper_2607_18631_b200.binding import load_library
    L = load_library()
    yield lambda: L.pf_moe_meeting(2000, 1)
    assert L.pf_moe_meeting(0, 0) == 0


@pytest.mark.parametrize("T", [1, 16, 17, 130])      # up to 16 tokens each block chooses by itself: two meetings, else three
@pytest.mark.parametrize("wtype", ["bf16", "e4m3"])
def test_a_wait_that_runs_out_is_reported_and_leaves_nan(T, wtype, lost_block):
    import torch
    from paper_2607_18631_b200 import ops
    x, router, ws, sc = layer_inputs(T, 512, 200, 16, 16, 1, wtype, seed=T)
    layer = ops.MoeLayer(router, *ws, top_k=4, n_shared=1, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2])
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    want = layer.forward(x, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.isfinite(want["out"].float()).all()
    assert lost_block() == 0
    out = torch.zeros_like(x)
    layer.forward(x, out=out, status=status)
    unasked = layer.forward(x)["out"]                  # nobody reads a status
    torch.cuda.synchronize()
    assert int(status) == 1
    assert torch.isnan(out.float()).all() and torch.isnan(unasked.float()).all()
    from paper_2607_18631_b200.binding import load_library
    assert load_library().pf_moe_meeting(0, 0) == 0
    got = layer.forward(x, status=status)              # the next call is whole again
    assert int(status) == 0 and all(torch.equal(got[n], want[n]) for n in want)


def test_limits_are_checked():
    from paper_2607_18631_b200.binding import PF_ERANGE
    from paper_2607_18631_b200.binding import load_library
    L = load_library()
    assert L.pf_moe_meeting(0, 2) == PF_ERANGE and L.pf_moe_meeting((1 << 21) + 1, 0) == PF_ERANGE
    assert L.pf_moe_meeting(0, 0) == 0
