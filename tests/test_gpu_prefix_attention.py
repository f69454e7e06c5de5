"""pf_prefix_attention against a plain implementation in 64 bits.

Tolerance.  Weights enter the second product as fp16 numbers (2^-11; an absolute 2^-32 of the row's largest below 2^-21 of it), the exponent's
argument carries 2^-20 (2 + max|s|) as in pf_decode_attention, and sums of 16 products are added up one behind the other in 32 bits, cut off: up to 65536 / 16
steps of 2^-23.  With W = sum w |V| / sum w:
|out - ref| <= W (2^-11 + steps 2^-23 + 2^-20 (2 + max|s|)) + n 2^-32 max|V| + half a step of the output type."""
from __future__ import annotations

import pytest

from test_gpu_kv_attention import make_cache

pytestmark = pytest.mark.gpu

PART = dict(bfloat16=2.0 ** -8, float16=2.0 ** -11)


def d32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def tokens_of(cache, scale, row, n, h):
    """The first n tokens of a table row, in 64 bits, without those whose page is not there."""
    import torch
    n_pages, _, P, hd = cache.shape
    n = max(0, min(n, len(row) * P))
    pages = torch.tensor(row[:-(-n // P)], dtype=torch.long)
    ok = (pages >= 0) & (pages < n_pages)
    at = torch.where(ok, pages, 0)
    x = cache[at, h].double() * scale[at, h].double()[:, None, None]
    return x.reshape(-1, hd)[:n][ok.repeat_interleave(P)[:n]]


def reference(q, cache, lengths, table, plen, ptable, cu, sm_scale):
    import torch
    kc, vc, ks, vs = (t.cpu() for t in cache)
    kc, vc = kc.float(), vc.float()
    B, nh, hd = q.shape
    G = nh // kc.shape[1]
    out, lse = torch.zeros(B, nh, hd, dtype=torch.float64), torch.full((B, nh), -float("inf"), dtype=torch.float64)
    tol = torch.zeros(B, nh, hd, dtype=torch.float64)
    tables, ptables = table.cpu().tolist(), ptable.cpu().tolist()
    shared = {}
    for b in range(B):
        group = next((g for g in range(len(plen)) if cu[g] <= b < cu[g + 1]), None)
        for h in range(kc.shape[1]):
            k, v = (tokens_of(c, s, tables[b], lengths[b], h) for c, s in ((kc, ks), (vc, vs)))
            if group is not None:
                if (group, h) not in shared:
                    shared[group, h] = [tokens_of(c, s, ptables[group], plen[group], h) for c, s in ((kc, ks), (vc, vs))]
                k, v = (torch.cat([p, x]) for p, x in zip(shared[group, h], (k, v)))
            if len(k) == 0:
                continue
            rows = slice(h * G, (h + 1) * G)
            s = q[b, rows].cpu().double() @ k.T * sm_scale
            lse[b, rows] = torch.logsumexp(s, -1)
            w = torch.softmax(s, -1)
            out[b, rows] = w @ v
            steps = min(len(k), 65536) / 16
            tol[b, rows] = (w @ v.abs()) * (2.0 ** -11 + steps * 2.0 ** -23 + 2.0 ** -20 * (2 + 1.4427 * s.abs().amax(-1, keepdim=True))) + len(k) * 2.0 ** -32 * v.abs().max()
    return out, lse, tol


def build(n_kv, hd, page, groups, plen, own, heads, dtype="bfloat16", seed=0, loose=0):
    """groups: sequences of each; loose: sequences behind the last group."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    B = sum(groups) + loose
    cols, pcols = (max(1, -(-max(max(n, default=0), 1) // page)) for n in (own, plen))
    n_pages = B * cols + len(groups) * pcols + 2
    cache = make_cache(n_pages, n_kv, page, hd, seed)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table, ptable = order[:B * cols].reshape(B, cols).contiguous(), order[B * cols:B * cols + len(groups) * pcols].reshape(len(groups), pcols).contiguous()
    cu = [sum(groups[:i]) for i in range(len(groups) + 1)]
    q = torch.randn(B, heads, hd, generator=g, device="cuda").to(getattr(torch, dtype))
    return q, cache, list(own), table, list(plen), ptable, cu


def compare(got, q, cache, own, table, plen, ptable, cu, sm_scale):
    import torch
    out, lse, tol = reference(q, cache, own, table, plen, ptable, cu, sm_scale)
    err = (got["out"].cpu().double() - out).abs()
    half = PART[str(q.dtype).split(".")[1]]
    assert torch.all(err <= tol + (out.abs() + tol) * half + 2.0 ** -25), float((err - tol).max())
    none = torch.isinf(lse)
    assert torch.equal(torch.isinf(got["lse"].cpu()), none) and torch.all(got["out"].cpu()[none] == 0)
    rel = (got["lse"].cpu().double() - lse)[~none].abs()
    assert torch.all(rel <= 2.0 ** -16 + 2.0 ** -20 * lse[~none].abs())


def run(q, cache, own, table, plen, ptable, cu, sm_scale=None, **kw):
    from paper_2607_18631_b200 import ops
    return ops.pf_prefix_attention(q, *cache, d32(own), table, d32(plen), ptable, d32(cu), sm_scale=sm_scale, lse=True, **kw)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_kv,heads", [(1, 1), (2, 10), (3, 24), (2, 32)])
def test_one_group(page, hd, n_kv, heads):
    for B, length in ((1, 1), (2, 127), (5, 128), (3, 129), (7, 515), (33, 1000)):
        args = build(n_kv, hd, page, [B], [length], [(37 * i + 5) % 150 for i in range(B)], heads, seed=length)
        compare(run(*args), *args, hd ** -0.5)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("hd", [64, 128])
def test_groups_of_all_kinds(hd, dtype):
    """Empty groups, groups without a prefix, sequences without tokens, sequences in no group."""
    import torch
    groups, plen = [3, 0, 5, 1, 40, 2], [700, 50, 0, 1, 333, 2049]
    B = sum(groups) + 4
    own = [(91 * i) % 400 if i % 3 else 0 for i in range(B)]
    args = build(2, hd, 32, groups, plen, own, 16, dtype=dtype, loose=4)
    compare(run(*args), *args, hd ** -0.5)
    q, cache, own, table, plen, ptable, cu = args
    cu = [2] + cu[1:]                                     # the first two sequences too
    compare(run(q, cache, own, table, plen, ptable, cu), q, cache, own, table, plen, ptable, cu, hd ** -0.5)
    none = run(q, cache, [0] * B, table, [0] * len(plen), ptable, cu)
    assert torch.all(none["out"] == 0) and torch.all(none["lse"] == -float("inf"))


@pytest.mark.parametrize("B,heads,n_kv,length", [(2, 8, 1, 30001), (70, 8, 2, 2500), (129, 2, 1, 1300), (300, 5, 1, 700), (64, 64, 8, 400), (1, 16, 16, 9000)])
def test_many_rows_and_long_prefixes(B, heads, n_kv, length):
    args = build(n_kv, 128, 64, [B], [length], [i % 70 for i in range(B)], heads, seed=B)
    compare(run(*args), *args, 128 ** -0.5)


def test_it_is_attention_over_both_parts():
    """One table row with the prefix's pages and the own ones gives what pf_decode_attention gives (prefixes that fill their pages)."""
    import torch
    from paper_2607_18631_b200 import ops
    q, cache, own, table, plen, ptable, cu = build(4, 128, 64, [9], [640], [30 * i for i in range(9)], 16)
    got = run(q, cache, own, table, plen, ptable, cu)
    joint = torch.cat([ptable.expand(9, -1), table], 1).contiguous()
    want = ops.pf_decode_attention(q, *cache, d32([640 + n for n in own]), joint, lse=True)
    assert torch.allclose(got["out"].float(), want["out"].float(), rtol=2.0 ** -7, atol=2.0 ** -10)
    assert torch.allclose(got["lse"], want["lse"], rtol=0, atol=1e-4)
    alone = ops.pf_prefix_attention(q, *cache, d32(own), table, d32(plen), ptable, lse=True)      # without offsets: one group of all
    assert torch.equal(alone["out"], got["out"]) and torch.equal(alone["lse"], got["lse"])
    no = ops.pf_prefix_attention(q, *cache, d32(own), table, d32([]), ptable[:0], d32([0]), lse=True)
    ref = ops.pf_decode_attention(q, *cache, d32(own), table, lse=True)
    assert torch.equal(no["out"], ref["out"]) and torch.equal(no["lse"], ref["lse"])


def test_pages_that_are_not_there_and_what_lies_behind_the_length():
    import torch
    args = build(2, 64, 16, [6, 5], [200, 77], [3 * i for i in range(11)], 8)
    q, cache, own, table, plen, ptable, cu = args
    ptable[0, 2], ptable[0, 5], ptable[1, 0] = -1, 1 << 30, cache[0].shape[0]
    compare(run(*args), *args, 0.125)
    kc, vc, ks, vs = cache
    last = int(ptable[0, 12])                             # 200 = 12 pages and 8 tokens
    kc.view(torch.uint8)[last, :, 8:] = 0x7F              # NaN behind the prefix's end
    vc.view(torch.uint8)[last, :, 8:] = 0x7F
    compare(run(*args), *args, 0.125)
    plen[1] = 1 << 30                                     # longer than the table
    want = run(q, cache, own, table, [200, ptable.shape[1] * 16], ptable, cu)
    got = run(*args)
    assert torch.equal(got["out"], want["out"])


def test_scores_of_all_sizes():
    """sm_scale of both signs and zero, large scores, one token with nearly all the weight in front of many."""
    import torch
    for sm in (-0.3, 0.0, 2.0, 1e-3):
        args = build(1, 64, 32, [20], [700], [i for i in range(20)], 4, seed=3)
        compare(run(*args, sm_scale=sm), *args, sm)
    q, cache, own, table, plen, ptable, cu = build(1, 128, 64, [3], [20000], [5, 0, 9], 4)
    kc, vc, ks, vs = cache
    ks.fill_(2.0 ** -9)
    first = int(ptable[0, 0])
    q[:] = 0
    q[..., 0] = 8.0
    kc.view(torch.uint8)[:, :, :, 0] = 0
    for lead in (6.0, 12.0, 16.0):                        # bits that the first token is ahead of the others
        kc[first, 0, 0, 0] = min(448.0, lead / 1.4427 / 8.0 / (128 ** -0.5) * 512)
        ks[first] = 2.0 ** -9 if kc[first, 0, 0, 0].float() < 448 else 2.0 ** -9 * (lead / 1.4427 / 8.0 / (128 ** -0.5) * 512) / 448
        args = q, cache, own, table, plen, ptable, cu
        compare(run(*args), *args, 128 ** -0.5)


def test_values_of_very_different_pages():
    import torch
    args = build(1, 128, 16, [12], [900], [20] * 12, 3, seed=5)
    vs = args[1][3]
    vs.copy_(torch.exp2(torch.randint(-30, 10, vs.shape, device="cuda").float()))
    compare(run(*args), *args, 128 ** -0.5)


def test_a_query_that_is_not_finite_spoils_its_own_head():
    import torch
    args = build(2, 128, 64, [10], [500], [40] * 10, 8)
    q = args[0]
    good = run(*args)
    q[3, 2, 7], q[8, 5, 0] = float("nan"), float("inf")
    got = run(*args)
    same = torch.ones(10, 8, dtype=torch.bool, device="cuda")
    same[3, 2] = same[8, 5] = False
    assert torch.equal(got["out"][same], good["out"][same]) and torch.equal(got["lse"][same], good["lse"][same])
    assert torch.isnan(got["out"][3, 2].float()).all() and torch.isnan(got["lse"][3, 2])


def test_nan_in_the_cache_reaches_the_rows_that_see_it():
    import torch
    args = build(2, 64, 16, [4, 3], [100, 90], [9] * 7, 4)
    kc = args[1][0]
    kc.view(torch.uint8)[int(args[5][0, 1]), 1, 3, 5] = 0x7F       # of the first group's prefix, key head 1
    got = run(*args)["out"].float()
    assert torch.isnan(got[:4, 2:]).all() and not torch.isnan(got[:4, :2]).any() and not torch.isnan(got[4:]).any()


def test_strides_streams_and_captured_calls():
    import torch
    from paper_2607_18631_b200 import ops
    args = build(2, 128, 64, [30], [1500], [11 * i for i in range(30)], 16)
    q, cache, own, table, plen, ptable, cu = args
    want = run(*args)
    wide = torch.zeros(30, 20, 128, dtype=q.dtype, device="cuda")
    wide[:, 2:18] = q
    into = torch.zeros(30, 18, 128, dtype=q.dtype, device="cuda")
    got = run(wide[:, 2:18], cache, own, table, plen, ptable, cu, out=into[:, 1:17])
    assert torch.equal(into[:, 1:17], want["out"]) and torch.all(into[:, 0] == 0) and torch.all(into[:, 17] == 0) and torch.equal(got["lse"], want["lse"])
    side = torch.cuda.Stream()
    mine = q.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    dev = [d32(own), table, d32(plen), ptable, d32(cu)]
    torch.cuda.synchronize()
    got = ops.pf_prefix_attention(mine, *cache, *dev, lse=True, stream=side)
    del mine
    rubbish = [torch.full_like(q, float("nan")) for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got["out"], want["out"]), len(rubbish)
    # two captured calls that share a workspace, replayed one behind the other with other lengths
    size = ops._lib()[0].pf_prefix_attention_workspace(ops._cache(torch, "", *cache), 30, 16, 1, ptable.shape[1])
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(ops.pf_prefix_attention(q, *cache, *dev, lse=True, workspace=ws))
        graphs.append(g)
    ws.view(torch.uint8).fill_(0xFF)
    for g in graphs:
        g.replay()
    assert all(torch.equal(o["out"], want["out"]) and torch.equal(o["lse"], want["lse"]) for o in outs)
    dev[0].fill_(7)
    dev[2].fill_(801)
    graphs[0].replay()
    compare(outs[0], q, cache, [7] * 30, table, [801], ptable, cu, 128 ** -0.5)


def test_offsets_that_make_no_sense_stay_in_range():
    """Decreasing or outlying offsets: rows of sequences in sound groups are right, and nothing else is touched."""
    import torch
    args = build(2, 64, 16, [4, 4], [100, 90], [9] * 8, 4)
    q, cache, own, table, plen, ptable, _ = args
    out = torch.full((10, 4, 64), 5.0, dtype=q.dtype, device="cuda")
    for cu in ([0, 8, 0], [-5, 4, 1 << 30], [7, 3, 1], [1 << 30, 0, -1]):
        run(q, cache, own, table, plen, ptable, cu, out=out[1:9])
        assert torch.all(out[0] == 5.0) and torch.all(out[9] == 5.0)


def test_same_call_same_bits():
    import torch
    args = build(4, 128, 64, [50], [5000], [13 * i for i in range(50)], 32)
    a = run(*args)
    for _ in range(5):
        b = run(*args)
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])
