"""pf_prefix_attention with scores so large that fp32 is coarse at their size: weights stay finite and the largest one counts, as in pf_decode_attention."""
from __future__ import annotations

import pytest

from test_gpu_kv_attention import make_cache, reference_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score", [3.0e3, 1.0e5, 1.0e6, 2.0e7, 3.0e8, 1.0e15, 1.0e30])
@pytest.mark.parametrize("low", [False, True])
@pytest.mark.parametrize("B", [1, 40])
def test_large_scores_stay_finite(score, low, B):
    """Keys that differ little in front of a few that do (low: the scores are far below 0), value scales that are no powers of two."""
    import torch
    from paper_2607_18631_b200 import ops
    n, hd, page = 5000, 128, 16
    kc, vc, ks, vs = make_cache(320, 1, page, hd, 2)
    vs.copy_(torch.rand_like(vs) * 2.0 ** -6 + 2.0 ** -9)
    ks[0] = ks[5] = ks.max()
    kc[:320] = kc[:1]                                  # all pages alike: scores of a few sizes, many ties but for the scales
    table = torch.arange(320, dtype=torch.int32, device="cuda").reshape(1, 320)
    q = torch.randn(1, 8, hd, device="cuda", generator=torch.Generator(device="cuda").manual_seed(B)).to(torch.bfloat16)
    if low:
        kc.copy_((kc.float().abs() + 100).clamp(max=448).to(kc.dtype))
        q = -q.abs()
    top = reference_attention(q, kc, vc, ks, vs, [n], table, 1.0)[3].amax()
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    sm = float(score / top)
    got = ops.pf_prefix_attention(q.repeat(B, 1, 1), kc, vc, ks, vs, zero, zero[:, None].contiguous(), zero[:1] + n, table, sm_scale=sm, lse=True)
    assert torch.isfinite(got["out"].float()).all() and torch.isfinite(got["lse"]).all()
    # a mean of values
    v = vc.float() * vs[:, :, None, None]
    low_, high = v.amin((0, 1, 2)), v.amax((0, 1, 2))
    room = 2.0 ** -6 * torch.maximum(low_.abs(), high.abs())
    assert torch.all(got["out"].float() >= low_ - room) and torch.all(got["out"].float() <= high + room)
    # the log of the sum is the largest score but for log n and the scores' own rounding
    s = (q.double() @ (kc.double() * ks.double()[:, :, None, None])[:, 0].reshape(-1, hd)[:n].T * sm)[0].amax(-1)
    assert torch.all((got["lse"].double() - s).abs() <= 10 + s.abs() * 2.0 ** -18)
