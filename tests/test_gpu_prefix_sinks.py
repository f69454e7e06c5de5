"""pf_prefix_attention where weights span many binary orders: behind a token that holds nearly all the weight, the others keep theirs.

Values are positive, so that weights that are lost do not cancel.  Tolerance: weights as in pf_decode_attention, 2^-11 relative down to 2^-29 of the largest, and
below it an absolute 2^-40 of the largest a token, against values of at most 448 times the page's scale; sums of 16 products one behind the other over
at most 65536 tokens, 4096 steps of 2^-23; the exponent's argument 2^-20 (2 + max|s| / ln 2).  With W = sum w |V| / sum w:
|out - ref| <= W (2^-11 + 2^-11 + 2^-20 (2 + max|s| / ln 2)) + n 2^-40 448 max vs + half a unit of the output."""
from __future__ import annotations

import math

import pytest

from test_gpu_attention_range import with_a_sink
from test_gpu_kv_attention import reference_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("share", [0.992, 0.9999, 0.99999, 0.999997])
@pytest.mark.parametrize("nh,nkv,hd,page,each", [(3, 3, 128, 64, 1), (4, 1, 64, 16, 1), (16, 1, 128, 128, 17), (8, 2, 64, 32, 40)])
@pytest.mark.parametrize("at", [0, 0.4])
def test_a_sink_leaves_the_others_their_share(share, nh, nkv, hd, page, each, at):
    import torch
    from paper_2607_18631_b200 import ops
    n = 100_000 - 100_000 % page                                          # whole pages, which may then be in any order
    q, cache, table, sm = with_a_sink(n, share, nh, nkv, hd, page, nh + hd, 1.0)
    cache[1].copy_(cache[1].float().abs().to(torch.float8_e4m3fn))
    table = table.roll(int(at * table.shape[1]), 1)
    # so many groups that a block goes through the whole prefix (with few, most blocks never see the sink)
    groups = -(-150 // nkv)
    none = torch.zeros(groups * each, dtype=torch.int32, device="cuda")
    got = ops.pf_prefix_attention(q.repeat(groups * each, 1, 1), *cache, none, none[:, None].contiguous(), none[:groups] + n, table.repeat(groups, 1),
                                  torch.arange(groups + 1, dtype=torch.int32, device="cuda") * each, sm_scale=sm, lse=True)
    out, W, lse, top = reference_attention(q, *cache, [n], table, sm)
    bound = W * (2.0 ** -10 + 2.0 ** -20 * (2 + top[..., None] / math.log(2))) + n * 2.0 ** -40 * 448 * float(cache[3].max()) + (out.abs() + W * 2.0 ** -10) * 2.0 ** -8
    err = (got["out"].double() - out).abs()
    assert torch.all(err <= bound), float((err / bound).max())
    assert torch.all((got["lse"].double() - lse).abs() <= 2.0 ** -20 * (4 + top * 2))
