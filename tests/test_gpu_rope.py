"""pf_rope and pf_kv_append_rope against plain implementations in 64 bits.

Tolerances.  An angle is exact to 2^-32 turns; its upper 32 bits become a 32-bit float (2^-25 turns, 2 pi 2^-25 radians, at most).  Sine and cosine carry
2^-21.41 where the result has 16 or 8 bits (the special-function unit's bound between -pi and pi), less otherwise; so with pair length r = |(a, b)| and
amplitude m an element is off by at most m r (sqrt(2) 2^-21.41 + 2 pi 2^-25) < m r 2^-20, plus half a step of the output type.
The cache's bytes are compared with what the rounding of any value within that distance gives."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

PART = dict(bfloat16=2.0 ** -8, float16=2.0 ** -11, float32=2.0 ** -24)
TINY = dict(bfloat16=2.0 ** -134, float16=2.0 ** -25, float32=2.0 ** -150)      # half a step below the normals


def turned(x, positions, rotary, transposed=False):
    """64 bits, as a matrix of each pair; and the pairs' lengths."""
    import torch
    x, R = x.double().cpu(), rotary.rot
    f = torch.tensor(rotary.frequencies, dtype=torch.float64)
    t = positions.cpu().double()[:, None] * f
    c, s = (rotary.amplitude * g(t)[:, None, :] for g in (torch.cos, torch.sin))
    if transposed:
        s = -s
    i = torch.arange(R // 2)
    a, b = (i, i + R // 2) if rotary.layout == "half" else (2 * i, 2 * i + 1)
    y, r = x.clone(), torch.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    r[..., a] = r[..., b] = abs(rotary.amplitude) * torch.hypot(x[..., a], x[..., b])
    return y, r


def check(got, x, positions, rotary, transposed=False):
    import torch
    want, r = turned(x, positions, rotary, transposed)
    name = str(x.dtype).split(".")[1]
    err = (got.cpu().double() - want).abs()
    assert torch.all(err <= r * 2.0 ** -20 + want.abs() * PART[name] + TINY[name] + r * 2.0 ** -20 * PART[name]), float(err.max())
    rest = slice(rotary.rot, None)
    assert torch.equal(got[..., rest].cpu(), x[..., rest].cpu())


def case(tokens, heads, hd, dtype, seed=0, far=200000):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(tokens, heads, hd, generator=g, device="cuda").mul(3).to(getattr(torch, dtype))
    return x, torch.randint(0, far, (tokens,), generator=g, device="cuda").to(torch.int32)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,hd,rot", [(1, 1, 64, 64), (1, 32, 128, 128), (5, 25, 64, 16), (300, 3, 128, 64), (7, 2, 80, 32), (9, 5, 96, 96), (3, 7, 50, 34), (4, 3, 20, 20),
                                                 (2, 9, 256, 0), (1, 1, 2, 2), (2, 65, 1, 0), (700, 40, 128, 128)])
def test_rope(tokens, heads, hd, rot, layout, dtype):
    from paper_2607_18631_b200 import ops
    x, pos = case(tokens, heads, hd, dtype)
    rotary = ops.Rotary(rot, layout=layout)
    for transposed in (False, True):
        check(ops.pf_rope(x, pos, rotary, transposed=transposed), x, pos, rotary, transposed)


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), dict(scaling="parts", factor=32.0, amplitude=1.3466),
                                dict(scaling="parts", factor=8.0, original=4096, low=2.0, high=16.0, base=500000.0), dict(amplitude=-0.5), dict(frequencies=[0.0, 1.0, -0.25, 7.5] * 16)])
def test_rope_scalings(kw):
    from paper_2607_18631_b200 import ops
    x, pos = case(33, 4, 128, "float32", far=1 << 20)
    rotary = ops.Rotary(128, **kw)
    check(ops.pf_rope(x, pos, rotary), x, pos, rotary)


def test_rope_at_every_32_bit_position():
    """Frequencies that are binary fractions of a turn have exact angles anywhere."""
    import torch
    from paper_2607_18631_b200 import ops
    x, _ = case(8, 2, 16, "float32")
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, -77, 12345678], dtype=torch.int32, device="cuda")
    k = [2.0 ** -i for i in (1, 2, 3, 5, 8, 13, 21, 30)]
    rotary = ops.Rotary(16, frequencies=[2 * math.pi * f for f in k])
    got = ops.pf_rope(x, pos, rotary)
    rotary.frequencies = [2 * math.pi * f for f in k]
    # the oracle's angle: the position modulo a turn's positions, exactly
    want = []
    for t, p in enumerate(pos.tolist()):
        angle = torch.tensor([2 * math.pi * ((p % round(1 / f)) * f) for f in k], dtype=torch.float64)
        a, b = x[t].cpu().double().split(8, 1)
        want.append(torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], 1))
    assert torch.allclose(got.cpu().double(), torch.stack(want), rtol=0, atol=float(x.abs().max()) * 1.5 * 2.0 ** -20)


def test_rope_strides_and_in_place():
    import torch
    from paper_2607_18631_b200 import ops
    x, pos = case(37, 6, 64, "bfloat16")
    rotary = ops.Rotary(64)
    want = ops.pf_rope(x, pos, rotary)
    wide = torch.zeros(37, 11, 64, device="cuda", dtype=x.dtype)
    wide[:, 2:8] = x
    before = wide.clone()
    assert torch.equal(ops.pf_rope(wide[:, 2:8], pos, rotary), want)                     # a slice of a fused projection
    assert ops.pf_rope(wide[:, 2:8], pos, rotary, out=wide[:, 2:8]) is not None
    assert torch.equal(wide[:, 2:8], want) and torch.equal(wide[:, :2], before[:, :2]) and torch.equal(wide[:, 8:], before[:, 8:])
    swapped = x.transpose(0, 1).contiguous().transpose(0, 1)                             # tokens inside heads
    assert not swapped.is_contiguous() and torch.equal(ops.pf_rope(swapped, pos, rotary), want)
    assert torch.equal(ops.pf_rope(x, pos, rotary, out=swapped), want)
    odd = torch.zeros(37 * 6 * 64 + 1, device="cuda", dtype=x.dtype)[1:].view(37, 6, 64)      # 2 bytes past a boundary
    odd.copy_(x)
    assert torch.equal(ops.pf_rope(odd, pos, rotary), want)
    assert ops.pf_rope(x[:0], pos[:0], rotary).shape == (0, 6, 64) and ops.pf_rope(x[:, :0], pos, rotary).shape == (37, 0, 64)


def test_rope_gradient_against_differences():
    """<dy, R x> and <R^T dy, x> are the same number; and the transposed rotation undoes the rotation but for the amplitude squared."""
    import torch
    from paper_2607_18631_b200 import ops
    x, pos = case(50, 4, 64, "float32")
    dy, _ = case(50, 4, 64, "float32", seed=1)
    for layout in ("half", "interleaved"):
        rotary = ops.Rotary(48, layout=layout, amplitude=1.25)
        y, dx = ops.pf_rope(x, pos, rotary), ops.pf_rope(dy, pos, rotary, transposed=True)
        # per head, 64 products of up to |x||dy|: both sides are off by m |x||dy| 2^-20
        bound = 2 * 1.25 * x.double().norm(dim=-1) * dy.double().norm(dim=-1) * 2.0 ** -20
        assert torch.all(((dy.double() * y.double()).sum(-1) - (dx.double() * x.double()).sum(-1)).abs() <= bound)
        back = ops.pf_rope(y, pos, rotary, transposed=True)[..., :48] / 1.25 ** 2
        assert torch.all((back - x[..., :48]).abs() <= x.norm(dim=-1, keepdim=True) * 2.0 ** -18)
        # differences: the map is linear, so a difference quotient of any step is the derivative
        step = torch.zeros_like(x)
        step[:, :, 5] = 0.5
        slope = ((ops.pf_rope(x + step, pos, rotary).double() - y.double()) * dy.double()).sum(-1) / 0.5
        assert torch.allclose(slope, dx[..., 5].double(), rtol=0, atol=float((1.25 * (x.norm(dim=-1) + 1) * dy.norm(dim=-1)).max()) * 2.0 ** -18)


def test_rope_spoils_only_the_pair():
    import torch
    from paper_2607_18631_b200 import ops
    x, pos = case(4, 3, 64, "bfloat16")
    bad = x.clone()
    bad[1, 2, 3], bad[2, 0, 40] = float("nan"), float("inf")
    rotary = ops.Rotary(64)
    good, got = ops.pf_rope(x, pos, rotary), ops.pf_rope(bad, pos, rotary)
    same = torch.ones_like(x, dtype=torch.bool)
    same[1, 2, [3, 35]] = same[2, 0, [8, 40]] = False
    assert torch.equal(good[same], got[same]) and not torch.isfinite(got[~same].float()).any()


# ------------------------------------------------------------------ into the cache
def rope_append_case(n_kv, hd, page, new, past, rot=None, layout="half", heads=0, dtype="bfloat16", positions=False, seed=0, edit=None, max_new=None, amplitude=1.0):
    """The keys that go into the cache are bracketed: what 64 bits give, rounded to e4m3 a little up and a little down."""
    import torch
    from paper_2607_18631_b200 import ops
    from test_gpu_kv_attention import make_cache, reference_append
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    B, dt = len(new), getattr(torch, dtype)
    cols = max(-(-(max(p, 0) + n) // page) for p, n in zip(past, new)) + 1
    n_pages = B * cols + 2
    cache = make_cache(n_pages, n_kv, page, hd, seed)
    table = torch.randperm(n_pages, generator=g, device="cuda")[:B * cols].reshape(B, cols).to(torch.int32)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    total = cu[-1] + 3                                    # rows behind the last sequence
    k, v = (torch.randn(total, n_kv, hd, generator=g, device="cuda").mul(s).to(dt) for s in (3.0, 0.01))
    q = torch.randn(total, heads, hd, generator=g, device="cuda").to(dt) if heads else None
    if edit:
        edit(k, v, table)
    d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rotary = ops.Rotary(hd if rot is None else rot, layout=layout, amplitude=amplitude)
    at = torch.zeros(total, dtype=torch.int64)
    for b in range(B):
        at[cu[b]:cu[b + 1]] = torch.arange(new[b]) + max(0, past[b])
    if positions:
        at += torch.randint(0, 100000, (total,))
    most = max(new) if max_new is None else max_new
    mark = torch.full_like(q, 7.0) if heads else None
    before = [t.cpu().clone() for t in cache]
    got_q = ops.pf_kv_append_rope(*cache, q, k, v, d(cu), d(past), table, rotary, max_new=most, positions=at.to(torch.int32).cuda() if positions else None, q_out=mark)
    exact, r = turned(k, at, rotary)
    exact, r = exact.float().double(), r
    want = [t.clone() for t in before]
    reference_append(*want, exact, v.cpu(), cu, past, table.cpu(), most)
    got = [t.cpu() for t in cache]
    assert torch.equal(got[3], want[3]) and torch.equal(got[1].view(torch.uint8), want[1].view(torch.uint8))      # values: as without rotation
    assert torch.equal(got[2], want[2])                                                 # the keys' scales (no maximum of these seeds lies on a border)
    low, high = ([t.clone() for t in before] for _ in range(2))
    margin = r * 2.0 ** -20 + 1e-30
    for part, x in ((low, exact - margin), (high, exact + margin)):
        part[2] = want[2].clone()                         # old tokens and scales as they have to be
        reference_append(part[0], part[1], want[2].clone(), part[3], exact, v.cpu(), cu, past, table.cpu(), most)
        for b in range(B):
            for j in range(min(new[b], most)):
                p = max(0, past[b]) + j
                pg = int(table[b, p // page]) if p // page < cols else -1
                if 0 <= pg < n_pages:
                    part[0][pg, :, p % page] = (x[cu[b] + j] / want[2][pg].double()[:, None]).clamp(-448, 448).float().to(torch.float8_e4m3fn)
    old = want[0].clone()
    for part in (low, high):                              # what was there before: exactly the reference's
        for b in range(B):
            s0 = max(0, past[b])
            if new[b] and s0 % page and s0 // page < cols:
                pg = int(table[b, s0 // page])
                if 0 <= pg < n_pages:
                    part[0][pg, :, :s0 % page] = old[pg, :, :s0 % page]
    a, lo, hi = got[0].float(), low[0].float(), high[0].float()
    ok = (a >= torch.minimum(lo, hi)) & (a <= torch.maximum(lo, hi)) | (torch.isnan(a) & torch.isnan(want[0].float()))
    assert torch.all(ok), int((~ok).sum())
    if heads:
        assert got_q is mark
        used = torch.zeros(total, dtype=torch.bool)
        for b in range(B):
            used[cu[b]:cu[b] + min(new[b], most)] = True
        assert torch.all(mark[~used.cuda()] == 7.0)
        check(mark[used.cuda()], q[used.cuda()], at[used], rotary)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_append_rope_single_tokens(page, hd, layout):
    rope_append_case(3, hd, page, [1] * 9, [0, 1, page - 1, page, page + 1, 2 * page - 1, 5, 15, 3 * page + 7], layout=layout, heads=6)


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("hd,rot", [(64, 64), (64, 16), (128, 128), (128, 48), (128, 0)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_append_rope_ragged_prompts(page, hd, rot, dtype):
    rope_append_case(2, hd, page, [1, 0, page, page + 1, 3 * page - 1, 4, 77], [0, 5, 0, page - 1, 3, 2 * page, 9], rot=rot, dtype=dtype, heads=10, positions=True,
                     layout="interleaved" if rot == 48 else "half")


def test_append_rope_few_tokens_and_max_new():
    rope_append_case(4, 128, 16, [4, 3, 2, 4], [14, 15, 13, 12], heads=4, amplitude=1.5)
    rope_append_case(1, 64, 16, [40, 3, 25], [7, 0, 16], heads=2, max_new=20)
    rope_append_case(1, 64, 16, [40, 3, 25], [7, 0, 16], heads=2, max_new=2)
    rope_append_case(2, 64, 32, [6, 9], [3, 0])


def test_append_rope_drops_what_has_no_place():
    def edit(k, v, table):
        table[0, 0] = -1
        table[1, 1] = 1 << 30
    rope_append_case(2, 64, 16, [5, 40, 1], [3, 1, 0], heads=2, edit=edit)


def test_append_rope_without_rotation_is_the_append():
    """Nothing turns: the bytes of pf_kv_append.  A rotation of pf_rope followed by pf_kv_append differs by the rounding in between only."""
    import torch
    from paper_2607_18631_b200 import ops
    from test_gpu_kv_attention import make_cache
    d = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.randperm(12, device="cuda").to(torch.int32).reshape(3, 4)
    k, v = (torch.randn(70, 2, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
    one, two = make_cache(12, 2, 32, 128), make_cache(12, 2, 32, 128)
    args = d(0, 30, 31, 70), d(3, 0, 40), table
    ops.pf_kv_append(*one, k, v, *args, max_new=39)
    assert ops.pf_kv_append_rope(*two, None, k, v, *args, ops.Rotary(0), max_new=39) is None
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(one, two))


def test_append_rope_captured_and_replayed():
    import torch
    from paper_2607_18631_b200 import ops
    from test_gpu_kv_attention import make_cache
    d = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rotary, table = ops.Rotary(64), torch.arange(6, dtype=torch.int32, device="cuda").reshape(2, 3)
    q, k, v = (torch.randn(2, h, 64, device="cuda").to(torch.bfloat16) for h in (4, 2, 2))
    lengths, cu = d(0, 20), d(0, 1, 2)
    eager, replayed = make_cache(6, 2, 16, 64), make_cache(6, 2, 16, 64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.pf_kv_append_rope(*replayed, q, k, v, cu, lengths, table, rotary, max_new=1)
    for step in range(3):
        graph.replay()
        want = ops.pf_kv_append_rope(*eager, q, k, v, cu, lengths, table, rotary, max_new=1)
        assert torch.equal(out, want)
        lengths += 1
        k.mul_(2)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(eager, replayed))
