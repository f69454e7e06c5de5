"""pf_decode_attention where weights span many binary orders: a token that holds nearly all the weight and a value near zero.

Tolerance.  Weights enter the second product as fp16 numbers of at most 2^15: 2^-11 relative down to 2^-29 of the largest, and below it an absolute
2^-40 of the largest a token, against values of at most 448 times the page's scale.  The rest as in test_gpu_kv_attention: with W = sum w |V| / sum w,
|out - ref| <= W (2^-11 + 2^-20 (2 + max|s| / ln 2)) + n 2^-40 448 max vs + half a unit of the output.
The log-sum-exp is held to what it is for short rows, 2^-20 (4 + 2 max|s|): its sum is added up in two levels."""
from __future__ import annotations

import math

import pytest

from test_gpu_kv_attention import make_cache, reference_attention

pytestmark = pytest.mark.gpu


def with_a_sink(n, share, nh, nkv, hd, page, seed, lift):
    """One sequence whose first token has `share` of every head's weight; its page holds no
    other key and no value, and a value scale `lift` times as large.  Heads that
    share a key head are multiples (0.95 .. 1) of one query."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    cols = -(-n // page)
    kc, vc, ks, vs = make_cache(cols + 2, nkv, page, hd, seed)
    table = torch.randperm(cols + 2, generator=g, device="cuda")[:cols].reshape(1, cols).to(torch.int32)
    G = nh // nkv
    base = torch.randn(nkv, 1, hd, generator=g, device="cuda")
    q = (base * torch.linspace(1.0, 0.95, G, device="cuda")[:, None]).reshape(1, nh, hd).to(torch.bfloat16)
    sm = 0.5 / math.sqrt(hd)
    first = int(table[0, 0])
    kc.view(torch.uint8)[first] = 0
    _, _, lse, _ = reference_attention(q, kc, vc, ks, vs, [n], table, sm)
    for h in range(nkv):
        # the sink's score is sm * scale * 448 * sum |q|: the scale of its page follows from the share
        kc[first, h, 0] = (torch.sign(q[0, h * G].float()) * 448).to(torch.float8_e4m3fn)
        want = float(lse[0, h * G]) + math.log(share / (1 - share))
        ks[first, h] = want / (sm * 448 * float(q[0, h * G].float().abs().sum()))
    vs[first] *= lift
    vc.view(torch.uint8)[first] = 0
    return q, (kc, vc, ks, vs), table, sm


@pytest.mark.parametrize("share", [0.9, 0.992, 0.998, 0.9999, 1 - 2.0 ** -20])
@pytest.mark.parametrize("nh,nkv,hd,page", [(3, 3, 128, 64), (4, 4, 64, 16), (16, 1, 128, 128), (8, 2, 64, 32)])
def test_a_sink_leaves_the_others_their_share(share, nh, nkv, hd, page):
    check(share, nh, nkv, hd, page, 1.0)


def check(share, nh, nkv, hd, page, lift):
    import torch
    from paper_2607_18631_b200 import ops
    n = 100_000
    q, cache, table, sm = with_a_sink(n, share, nh, nkv, hd, page, nh + hd, lift)
    # so many rows over the same pages that a warp goes through whole sequences (with few, most warps never see the sink)
    rows = -(-148 * 8 // nkv) + 1
    got = ops.pf_decode_attention(q.repeat(rows, 1, 1), *cache, torch.full((rows,), n, dtype=torch.int32, device="cuda"), table.repeat(rows, 1), sm_scale=sm, lse=True)
    out, W, lse, top = reference_attention(q, *cache, [n], table, sm)
    bound = W * (2.0 ** -11 + 2.0 ** -20 * (2 + top[..., None] / math.log(2))) + n * 2.0 ** -40 * 448 * float(cache[3].max()) + (out.abs() + W * 2.0 ** -10) * 2.0 ** -8
    err = (got["out"].double() - out).abs()
    assert torch.all(err <= bound), float((err / bound).max())
    assert torch.all((got["lse"].double() - lse).abs() <= 2.0 ** -20 * (4 + top * 2))


@pytest.mark.parametrize("lift", [2.0 ** 6, 2.0 ** 10])
def test_a_sink_on_a_page_of_large_values(lift):
    """The reference of the weights is taken over score + log2 of the page's value scale: such a page takes its orders off the range."""
    check(0.992, 4, 4, 128, 64, lift)


@pytest.mark.parametrize("score", [3.0e3, 1.0e6, 3.0e8])
def test_large_scores_stay_finite(score):
    """The largest weight is 2^15 at most, however coarse fp32 is at the scores' size."""
    import torch
    from paper_2607_18631_b200 import ops
    n, hd, page = 1000, 128, 16
    kc, vc, ks, vs = make_cache(64, 1, page, hd, 2)
    table = torch.arange(64, dtype=torch.int32, device="cuda").reshape(1, 64)
    q = torch.randn(1, 8, hd, device="cuda").to(torch.bfloat16)
    top = reference_attention(q, kc, vc, ks, vs, [n], table, 1.0)[3].amax()
    got = ops.pf_decode_attention(q, kc, vc, ks, vs, torch.tensor([n], dtype=torch.int32, device="cuda"), table, sm_scale=float(score / top), lse=True)
    assert torch.isfinite(got["out"].float()).all() and torch.isfinite(got["lse"]).all()
    assert torch.all(got["out"].float().abs() <= 448 * vs.max() * 1.01)


@pytest.mark.parametrize("nh,nkv,hd", [(8, 1, 128), (16, 1, 64), (12, 3, 128), (40, 2, 64)])
@pytest.mark.parametrize("lens", [[300, 40, 1], [20_000]])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_a_query_that_is_not_finite_spoils_its_own_head_only(nh, nkv, hd, lens, bad):
    import torch
    from paper_2607_18631_b200 import ops
    B, page = len(lens), 32
    cols = -(-max(lens) // page)
    cache = make_cache(B * cols, nkv, page, hd, nh)
    table = torch.arange(B * cols, dtype=torch.int32, device="cuda").reshape(B, cols)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = (torch.randn(B, nh, hd, device="cuda") * 20).to(torch.bfloat16)
    want = ops.pf_decode_attention(q, *cache, ln, table, sm_scale=0.01, lse=True)
    heads = [1, nh - 1]
    q[:, heads[0], 5] = bad
    q[:, heads[1], hd - 1] = bad
    got = ops.pf_decode_attention(q, *cache, ln, table, sm_scale=0.01, lse=True)
    ok = [h for h in range(nh) if h not in heads]
    assert torch.equal(got["out"][:, ok], want["out"][:, ok]) and torch.equal(got["lse"][:, ok], want["lse"][:, ok])
    many = ln > 30                                          # enough tokens for scores of either sign
    assert torch.isnan(got["out"][many][:, heads].float()).all() and torch.isnan(got["lse"][many][:, heads]).all()


def test_heads_of_very_different_size_share_a_key_head():
    import torch
    from test_gpu_kv_attention import attend

    def edit(q, cache, table):
        q[:, 0] *= 2.0 ** 40
        q[:, 3] *= 2.0 ** 20
        q[:, 6] *= 2.0 ** -20
    attend(3, 8, 1, 128, 64, [200, 33, 900], edit=edit)
    attend(3, 16, 1, 64, 16, [200, 33, 900], edit=edit)
