"""pf_kv_append and pf_decode_attention against plain implementations in 64 bits.

The append is exact arithmetic (powers of two, one rounding to e4m3), so its bytes are compared bit for bit with a
reference that walks page by page.

Attention tolerances.  Weights are rounded to fp16 (2^-11) before the second product while the denominator keeps them in fp32; the
exponent's argument, up to |s| in base 2, carries 2^-22 |s| from fp32 sums over 64 or 128 products and the exponential 2^-22; sums over
n tokens run in at most 32-token tiles joined in fp32.  With W = sum w |V| / sum w:
|out - ref| <= W (2^-11 + 2^-20 (2 + max|s|)) + half a unit of the output type."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu


def make_cache(n_pages, n_kv, page, hd, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    kc, vc = (torch.randn(n_pages, n_kv, page, hd, generator=g, device="cuda").mul(110).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.exp2(torch.randint(lo, lo + 4, (n_pages, n_kv), generator=g, device="cuda").float()) for lo in (-8, -9))
    return kc, vc, ks, vs


# ------------------------------------------------------------------ append
def reference_append(kc, vc, ks, vs, k, v, cu, lens, table, max_new):
    """Page by page, head by head, on the CPU."""
    import torch
    for cache, scale, x in ((kc, ks, k), (vc, vs, v)):
        n_pages, n_kv, P, hd = cache.shape
        for b in range(len(lens)):
            n = max(0, min(cu[b + 1] - cu[b], max_new, x.shape[0] - cu[b])) if cu[b] >= 0 else 0
            j = 0
            start = max(0, lens[b])
            while j < n:
                pos = start + j
                slot, m = pos % P, min(P - pos % P, n - j)
                col = pos // P
                page = int(table[b, col]) if col < table.shape[1] else -1
                if 0 <= page < n_pages:
                    for h in range(n_kv):
                        part = x[cu[b] + j:cu[b] + j + m, h].double()
                        fin = part[~torch.isnan(part)]
                        amax = float(fin.abs().max()) if fin.numel() else 0.0
                        e = -100
                        if amax > 0:
                            e = 118 if math.isinf(amax) else max(-100, min(118, math.frexp(amax)[1] - 9 + (math.frexp(amax)[0] > 0.875)))
                        s = 2.0 ** e
                        if slot:
                            old = float(scale[page, h])
                            s = max(s, old)
                            if s > old:
                                cache[page, h, :slot] = (cache[page, h, :slot].double() * (old / s)).float().to(torch.float8_e4m3fn)
                        scale[page, h] = s
                        q = (part / s).clamp(-448, 448)
                        cache[page, h, slot:slot + m] = q.float().to(torch.float8_e4m3fn)
                j += m


def append_case(n_kv, hd, page, new, past, dtype="bfloat16", seed=0, edit=None, spare=2):
    import torch
    from paper_2607_18631_b200 import ops
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    B = len(new)
    cols = max(-(-(max(p, 0) + n) // page) for p, n in zip(past, new)) + 1
    n_pages = B * cols + spare
    cache = make_cache(n_pages, n_kv, page, hd, seed)
    table = torch.randperm(n_pages, generator=g, device="cuda")[:B * cols].reshape(B, cols).to(torch.int32)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    dt = getattr(torch, dtype)
    k, v = (torch.randn(cu[-1], n_kv, hd, generator=g, device="cuda").mul(s).to(dt) for s in (3.0, 0.01))
    if edit:
        edit(k, v, table)
    want = [t.cpu().clone() for t in cache]
    reference_append(*want, k.cpu(), v.cpu(), cu, past, table.cpu(), max(new))
    d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ops.pf_kv_append(*cache, k, v, d(cu), d(past), table, max_new=max(new))
    for got, ref, name in zip(cache, want, ("k", "v", "k_scale", "v_scale")):
        a, b = (t.cpu().contiguous().view(torch.uint8) for t in (got, ref))
        if got.dtype == torch.float8_e4m3fn:      # any NaN byte is as good as another
            nan = torch.isnan(got.cpu().float())
            assert torch.equal(nan, torch.isnan(ref.float())), name
            assert torch.equal(a[~nan], b[~nan]), name
        else:
            assert torch.equal(a, b), name
    return cache


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_kv", [1, 3])
def test_append_single_tokens(page, hd, n_kv):
    append_case(n_kv, hd, page, [1] * 9, [0, 1, page - 1, page, page + 1, 2 * page - 1, 5, 15, 3 * page + 7])


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_append_ragged_prompts(page, hd, dtype):
    append_case(2, hd, page, [1, 0, page, page + 1, 3 * page - 1, 4, 77], [0, 5, 0, page - 1, 3, 2 * page, 9], dtype=dtype)


def test_append_few_tokens_cross_a_page():
    append_case(4, 128, 16, [4, 3, 2, 4], [14, 15, 13, 12])


def test_append_scale_grows_exactly_and_extremes():
    import torch

    def edit(k, v, table):
        k[0] = 0                                   # zeros: the least scale
        k[1] = 448.0                               # exactly representable at scale 1
        k[2, 0, 0] = 449.0
        v[3] = float("inf")
        v[4, :, 3] = float("nan")
        k[5] = 2.0 ** -120
        v[6] = -3.0e38
    append_case(2, 64, 32, [1] * 8, [0, 0, 3, 4, 31, 32, 40, 63], edit=edit)
    append_case(2, 64, 32, [9, 8, 1], [3, 0, 2], edit=lambda k, v, t: (k[4].fill_(1e4), v[9].fill_(0)))
    # a token after a token: the first keeps its value while the scale grows by 2^6
    from paper_2607_18631_b200 import ops
    kc, vc, ks, vs = make_cache(1, 1, 16, 64)
    table, d = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    first = torch.full((1, 1, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    ops.pf_kv_append(kc, vc, ks, vs, first, first, d(0, 1), d(0), table, max_new=1)
    assert float(ks) == 2.0 ** -6
    ops.pf_kv_append(kc, vc, ks, vs, first * 64, first, d(0, 1), d(1), table, max_new=1)
    assert float(ks) == 1.0 and torch.all(kc[0, 0, 0].float() == 7.0) and torch.all(kc[0, 0, 1].float() == 448.0)


def test_append_drops_what_has_no_place():
    """Pages outside the cache, positions past the table, rows past the tokens, more tokens than max_new."""
    def edit(k, v, table):
        table[0, 0] = -1
        table[1, 1] = 1 << 30
        table[2, 2] = table.numel() + 2
    for new in ([40, 40, 40], [3, 3, 3]):
        append_case(2, 64, 16, new, [0, 14, 30], edit=edit)
    import torch
    from paper_2607_18631_b200 import ops
    cache = make_cache(6, 1, 16, 64)
    k = torch.randn(8, 1, 64, device="cuda").to(torch.bfloat16)
    for cu, lens, max_new in (([0, 8], [30], 8), ([-3, 5], [0], 8), ([4, 20], [0], 16), ([0, 8], [0], 3), ([5, 2], [0], 8), ([0, 8], [-4], 8)):
        table = torch.tensor([[3, 1]], dtype=torch.int32, device="cuda")
        want = [t.cpu().clone() for t in cache]
        reference_append(*want, k.cpu(), k.cpu(), cu, lens, table.cpu(), max_new)
        d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        ops.pf_kv_append(*cache, k, k, d(cu), d(lens), table, max_new=max_new)
        assert all(torch.equal(a.cpu().contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(cache, want)), (cu, lens, max_new)


def test_append_strided_tokens_and_empty_calls():
    import torch
    from paper_2607_18631_b200 import PlanfrontError, ops
    qkv = torch.randn(5, 10 * 64, device="cuda").to(torch.bfloat16)            # fused projections: q, k, v side by side
    k, v = qkv[:, 6 * 64:8 * 64].unflatten(1, (2, 64)), qkv[:, 8 * 64:].unflatten(1, (2, 64))
    a, b = make_cache(8, 2, 16, 64), make_cache(8, 2, 16, 64)
    d = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(4, dtype=torch.int32, device="cuda").reshape(2, 2)
    ops.pf_kv_append(*a, k, v, d(0, 2, 5), d(0, 9), table, max_new=3)
    ops.pf_kv_append(*b, k.contiguous(), v.contiguous(), d(0, 2, 5), d(0, 9), table, max_new=3)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))
    before = [t.clone() for t in a]
    ops.pf_kv_append(*a, k[:0], v[:0], d(0, 0, 0), d(0, 9), table, max_new=3)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, before))
    for bad in (lambda: ops.pf_kv_append(*a, k.float(), v.float(), d(0, 2, 5), d(0, 9), table, max_new=3),
                lambda: ops.pf_kv_append(*a, k, v[:3], d(0, 2, 5), d(0, 9), table, max_new=3),
                lambda: ops.pf_kv_append(*a, k, v, d(0, 2), d(0, 9), table, max_new=3),
                lambda: ops.pf_kv_append(*a, k, v, d(0, 2, 5).long(), d(0, 9), table, max_new=3),
                lambda: ops.pf_kv_append(*a, k, v, d(0, 2, 5), d(0, 9), table, max_new=-1),
                lambda: ops.pf_kv_append(a[0][:, :, :8], a[1][:, :, :8], a[2], a[3], k, v, d(0, 2, 5), d(0, 9), table, max_new=3),
                lambda: ops.pf_kv_append(*a, k.cpu(), v, d(0, 2, 5), d(0, 9), table, max_new=3)):
        with pytest.raises(PlanfrontError):
            bad()


# ------------------------------------------------------------------ attention
def reference_attention(q, kc, vc, ks, vs, lens, table, sm):
    import torch
    B, nh, hd = q.shape
    n_pages, nkv, P, _ = kc.shape
    G = nh // nkv
    out, W = (torch.zeros(B, nh, hd, dtype=torch.float64, device=q.device) for _ in range(2))
    lse = torch.full((B, nh), -math.inf, dtype=torch.float64, device=q.device)
    top = torch.zeros(B, nh, dtype=torch.float64, device=q.device)
    for b in range(B):
        n = min(max(0, lens[b]), table.shape[1] * P)
        pages = table[b, :-(-n // P)].long()
        seen = ((pages >= 0) & (pages < n_pages)).repeat_interleave(P)[:n]
        pages = pages.clamp(0, n_pages - 1)
        for h in range(nkv):
            k, v = ((c[pages, h].double() * s[pages, h].double()[:, None, None]).reshape(-1, hd)[:n][seen] for c, s in ((kc, ks), (vc, vs)))
            if not k.shape[0]:
                continue
            rows = slice(h * G, (h + 1) * G)
            s = q[b, rows].double() @ k.T * sm
            p = torch.softmax(s, 1)
            out[b, rows], W[b, rows], lse[b, rows], top[b, rows] = p @ v, p @ v.abs(), torch.logsumexp(s, 1), s.abs().amax(1)
    return out, W, lse, top


def attend(B, nh, nkv, hd, page, lens, dtype="bfloat16", seed=0, q_mul=1.0, sm=None, edit=None, extra_cols=0, n_pages=None):
    import torch
    from paper_2607_18631_b200 import ops
    g = torch.Generator(device="cuda").manual_seed(seed + 5)
    cols = max(1, -(-max(lens) // page)) + extra_cols
    n_pages = n_pages or B * cols + 2
    cache = make_cache(n_pages, nkv, page, hd, seed)
    table = (torch.randperm(max(n_pages, B * cols), generator=g, device="cuda")[:B * cols] % n_pages).reshape(B, cols).to(torch.int32)
    q = (torch.randn(B, nh, hd, generator=g, device="cuda") * q_mul).to(getattr(torch, dtype))
    sm = 1.0 / math.sqrt(hd) if sm is None else sm
    if edit:
        edit(q, cache, table)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = ops.pf_decode_attention(q, *cache, ln, table, sm_scale=sm, lse=True)
    out, W, lse, top = reference_attention(q, *cache, lens, table, sm)
    half = 2.0 ** -8 if dtype == "bfloat16" else 2.0 ** -11
    bound = W * (2.0 ** -11 + 2.0 ** -20 * (2 + top[..., None] / math.log(2))) + (out.abs() + W * 2.0 ** -10) * half + 2.0 ** -25
    err = (got["out"].double() - out).abs()
    assert torch.all(err <= bound), (float((err / bound.clamp(min=1e-30)).max()), (err > bound).nonzero()[:4].tolist())
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(got["lse"]), empty) and torch.all(got["lse"][empty] < 0)
    assert torch.all((got["lse"].double() - lse)[~empty].abs() <= 2.0 ** -20 * (4 + top[~empty] * 2))
    assert torch.all(got["out"][empty] == 0)
    again = ops.pf_decode_attention(q, *cache, ln, table, sm_scale=sm, lse=True)
    assert torch.equal(again["out"], got["out"]) and torch.equal(again["lse"], got["lse"])
    return got


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("nh,nkv", [(1, 1), (8, 8), (8, 1), (12, 3), (20, 4), (16, 1), (40, 2), (136, 8)])
def test_attention_heads_and_pages(hd, page, nh, nkv):
    attend(5, nh, nkv, hd, page, [1, 0, page, 3 * page + 5, 200])


@pytest.mark.parametrize("lens", [[1], [31], [32], [33], [0], [0, 0, 7, 0], [257, 1, 1, 1, 64], [5000], [1] * 300, [0, 3] * 150, [20000, 3, 0, 900]])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_attention_lengths(lens, dtype):
    attend(len(lens), 8, 2, 128, 64, lens, dtype=dtype)


@pytest.mark.parametrize("hd,nh,nkv,n", [(128, 8, 1, 100001), (64, 32, 1, 65536), (128, 64, 8, 33000)])
def test_attention_one_long_sequence(hd, nh, nkv, n):
    attend(1, nh, nkv, hd, 64, [n])


def test_attention_many_sequences():
    lens = [(i * 37) % 211 for i in range(1500)]
    attend(1500, 4, 2, 64, 16, lens, n_pages=500)


def test_attention_nothing_beyond_the_length_counts():
    """NaN bytes behind the last token, NaN and infinite scales of pages past it, tables that hold rubbish there."""
    import torch
    lens = [1, 17, 40, 64, 65, 100]

    def edit(q, cache, table):
        kc, vc, ks, vs = cache
        used = set()
        for b, n in enumerate(lens):
            full = -(-n // 32)
            for c in range(full):
                page = int(table[b, c])
                used.add(page)
                if c == full - 1 and n % 32:
                    for t in (kc, vc):
                        t.view(torch.uint8)[page, :, n % 32:] = 0x7F
            table[b, full:] = -7 if b % 2 else 1 << 29
        for page in set(range(kc.shape[0])) - used:
            for t in (kc, vc):
                t.view(torch.uint8)[page] = 0xFF
            ks[page] = float("nan")
            vs[page] = float("inf")
    attend(6, 8, 2, 128, 32, lens, edit=edit, extra_cols=2)
    lens = [1, 16, 17, 33, 47]

    def edit16(q, cache, table):
        for b, n in enumerate(lens):
            last = -(-n // 16)
            spare = cache[0].shape[0] - 1
            table[table == spare] = 0
            cache[2][spare], cache[3][spare] = float("nan"), float("nan")
            cache[1].view(torch.uint8)[spare] = 0x7F
            table[b, last:] = spare
    attend(5, 4, 4, 64, 16, lens, edit=edit16, extra_cols=1, seed=3)


def test_attention_hides_pages_outside_the_cache():
    def edit(q, cache, table):
        table[0, 0] = -1
        table[1, 1] = cache[0].shape[0]
        table[2, :] = -1                      # nothing left: an empty row
        table[3, 2] = 2 ** 31 - 1
    got = attend(4, 8, 2, 64, 16, [40, 40, 40, 48], edit=edit)
    import torch
    assert torch.all(got["out"][2] == 0)
    attend(4, 8, 2, 128, 64, [200, 130, 64, 180], edit=edit)


def test_attention_lengths_past_the_table_and_negative():
    import torch
    from paper_2607_18631_b200 import ops
    cache = make_cache(8, 2, 16, 64)
    table = torch.arange(4, dtype=torch.int32, device="cuda").reshape(2, 2)
    q = torch.randn(2, 4, 64, device="cuda").to(torch.bfloat16)
    far = ops.pf_decode_attention(q, *cache, torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32, device="cuda"), table, lse=True)
    want = ops.pf_decode_attention(q, *cache, torch.tensor([32, 0], dtype=torch.int32, device="cuda"), table, lse=True)
    assert torch.equal(far["out"], want["out"]) and torch.equal(far["lse"], want["lse"]) and torch.all(far["out"][1] == 0)


def test_attention_extreme_queries_and_scales():
    import torch
    attend(3, 8, 2, 128, 64, [70, 300, 9], q_mul=0.0)
    attend(3, 8, 2, 128, 64, [70, 300, 9], q_mul=1e-30, sm=1e29)
    attend(3, 8, 2, 128, 64, [70, 300, 9], q_mul=1e30, sm=3e-31)
    attend(3, 8, 2, 64, 16, [70, 300, 9], q_mul=30.0)                 # a few tokens take all the weight
    attend(2, 8, 2, 64, 16, [70, 300], sm=0.0)                        # all alike
    attend(2, 8, 2, 64, 16, [70, 300], sm=-0.1)

    def edit(q, cache, table):
        cache[3][::2] *= 2.0 ** -30                                   # pages whose values hardly count
        cache[3][::3] *= 2.0 ** 20
    attend(4, 8, 2, 128, 16, [70, 300, 9, 1000], edit=edit)

    def zeros(q, cache, table):
        cache[1].view(torch.uint8)[:] = 0
        cache[3][:] = 0.0
    attend(2, 8, 2, 128, 16, [70, 300], edit=zeros)


def test_attention_strides_outputs_and_refusals():
    import torch
    from paper_2607_18631_b200 import PlanfrontError, ops
    cache = make_cache(20, 2, 32, 64)
    table = torch.randperm(20, device="cuda")[:12].reshape(3, 4).to(torch.int32)
    ln = torch.tensor([100, 1, 77], dtype=torch.int32, device="cuda")
    qkv = torch.randn(3, 12 * 64, device="cuda").to(torch.bfloat16)
    q = qkv[:, :8 * 64].unflatten(1, (8, 64))
    want = ops.pf_decode_attention(q.contiguous(), *cache, ln, table)["out"]
    hold = torch.zeros(3, 10 * 64, device="cuda", dtype=torch.bfloat16)
    out = hold[:, 64:9 * 64].unflatten(1, (8, 64))
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda").fill_(0xFF)
    got = ops.pf_decode_attention(q, *cache, ln, table, out=out, workspace=ws)["out"]
    assert got.data_ptr() == out.data_ptr() and torch.equal(got, want)
    assert torch.all(hold[:, :64] == 0) and torch.all(hold[:, 9 * 64:] == 0)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = ops.pf_decode_attention(q, *cache, ln, table, stream=s)["out"]
    s.synchronize()
    assert torch.equal(got, want)
    assert ops.pf_decode_attention(q[:0], *cache, ln[:0], table[:0])["out"].shape == (0, 8, 64)
    for bad in (lambda: ops.pf_decode_attention(q.float(), *cache, ln, table), lambda: ops.pf_decode_attention(q[:, :7], *cache, ln, table),
                lambda: ops.pf_decode_attention(q, *cache, ln[:2], table), lambda: ops.pf_decode_attention(q, *cache, ln.long(), table),
                lambda: ops.pf_decode_attention(q, *cache, ln, table[:, ::2]), lambda: ops.pf_decode_attention(q, *cache, ln, table, workspace=ws[:256]),
                lambda: ops.pf_decode_attention(q, *cache, ln, table, workspace=ws[1:]), lambda: ops.pf_decode_attention(q, *cache, ln, table, sm_scale=float("nan")),
                lambda: ops.pf_decode_attention(q.cpu(), *cache, ln, table), lambda: ops.pf_decode_attention(q, cache[0].view(torch.uint8), *cache[1:], ln, table)):
        with pytest.raises(PlanfrontError):
            bad()


def test_attention_in_a_graph():
    import torch
    from paper_2607_18631_b200 import ops
    cache = make_cache(64, 2, 64, 128)
    table = torch.arange(64, dtype=torch.int32, device="cuda").reshape(2, 32)
    ln = torch.tensor([1900, 60], dtype=torch.int32, device="cuda")
    q = torch.randn(2, 16, 128, device="cuda").to(torch.bfloat16)
    out, ws = torch.empty_like(q), torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
    ops.pf_decode_attention(q, *cache, ln, table, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.pf_decode_attention(q, *cache, ln, table, out=out, workspace=ws)
    ln.copy_(torch.tensor([33, 2048], dtype=torch.int32, device="cuda"))       # the lengths of another step
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ops.pf_decode_attention(q, *cache, ln, table)["out"])


def test_overlapping_rows_are_refused():
    import torch
    from paper_2607_18631_b200 import PlanfrontError, ops
    cache = make_cache(8, 2, 16, 64)
    d = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(6, dtype=torch.int32, device="cuda").reshape(3, 2)
    q, k = torch.randn(1, 4, 64, device="cuda").to(torch.bfloat16), torch.randn(1, 2, 64, device="cuda").to(torch.bfloat16)
    with pytest.raises(PlanfrontError):
        ops.pf_decode_attention(q.expand(3, 4, 64), *cache, d(3, 4, 5), table)
    with pytest.raises(PlanfrontError):
        ops.pf_kv_append(*cache, k.expand(3, 2, 64), k.expand(3, 2, 64), d(0, 1, 2, 3), d(3, 4, 5), table, max_new=1)
