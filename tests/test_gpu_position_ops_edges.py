"""Rotary positions, the rotated append and shared prefixes where calls meet: refusals, large offsets, several streams, captured gradients."""
from __future__ import annotations

import pytest

from test_gpu_ops_refusals import refused, workspaces
from test_gpu_prefix_attention import build, d32, run

pytestmark = pytest.mark.gpu


def small():
    import torch
    cache = [torch.zeros(4, 2, 16, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)] + [torch.ones(4, 2, device="cuda") for _ in range(2)]
    q, k = (torch.randn(2, h, 64, device="cuda").to(torch.bfloat16) for h in (4, 2))
    return cache, q, k, d32([5, 3]), d32([[0], [1]]), d32([20]), d32([[2, 3]]), d32([0, 2])


def test_calls_that_are_refused():
    """Nothing is launched."""
    import torch
    from paper_2607_18631_b200 import PlanfrontError, ops
    cache, q, k, lengths, table, plen, ptable, cu = small()
    rotary, pos, one_each = ops.Rotary(64), d32([0, 1]), d32([0, 1, 2])
    big = 1 << 32

    class Elsewhere:
        device_index, cuda_stream = torch.cuda.current_device() + 1, 0

    def rope(x=q, pos=pos, **kw):
        return lambda: ops.pf_rope(x, pos, rotary, **kw)

    def append(q=q, k=k, v=k, rotary=rotary, max_new=1, cu_new=one_each, lengths=lengths, table=table, **kw):
        return lambda: ops.pf_kv_append_rope(*cache, q, k, v, cu_new, lengths, table, rotary, max_new=max_new, **kw)

    def prefix(q=q, cu=cu, plen=plen, ptable=ptable, lengths=lengths, table=table, **kw):
        return lambda: ops.pf_prefix_attention(q, *cache, lengths, table, plen, ptable, cu, **kw)
    for call in (rope(x=q[0]), rope(x=q.double()), rope(x=q.cpu()), rope(pos=pos.long()), rope(pos=pos[:1]), rope(x=q.transpose(1, 2)), rope(x=q[:, :1].expand(2, 4, 64)),
                 rope(out=q[:1]), rope(out=q.float()), rope(stream=Elsewhere()), rope(x=torch.zeros(2, 4, 32, device="cuda")),      # fewer elements than are rotated
                 append(v=k.float()), append(q=q.half()), append(q=q[:1]), append(q=q[:, :, :32]), append(q=None, q_out=q), append(q_out=q[:, :2]), append(cu_new=one_each[:2]),
                 append(positions=d32([0])), append(positions=pos.long()), append(max_new=big + 1), append(rotary=ops.Rotary(24)), append(stream=Elsewhere()), append(k=k.float(), v=k.float(), q=None),
                 append(table=table[:1]), prefix(q=q.float()), prefix(q=q[:, :3]), prefix(cu=cu[:1]), prefix(cu=None, plen=d32([1, 1]), ptable=ptable.expand(2, 2).contiguous()),
                 prefix(plen=plen.long()), prefix(ptable=ptable[0]), prefix(ptable=ptable.expand(2, 2)), prefix(lengths=lengths[:1]), prefix(out=q[:1]), prefix(stream=Elsewhere()),
                 prefix(sm_scale=float("nan")), *(prefix(workspace=ws) for ws in workspaces()), prefix(workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))):
        refused(call)
    for kw in (dict(rot=63), dict(rot=-2), dict(rot=64, layout="other"), dict(rot=64, scaling="other"), dict(rot=64, frequencies=[1.0]), dict(rot=64, amplitude=float("nan")),
               dict(rot=2, frequencies=[float("inf")]), dict(rot=64, base=-1.0)):
        with pytest.raises(PlanfrontError):
            ops.Rotary(**kw)


def test_places_behind_4_gigabytes():
    """A cache of 5 GB a tensor, of which the last pages are used."""
    import torch
    from paper_2607_18631_b200 import ops
    pages, n_kv, page, hd = 39000, 8, 128, 128
    cache = [torch.empty(pages, n_kv, page, hd, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)] + [torch.empty(pages, n_kv, device="cuda") for _ in range(2)]
    used = [pages - 1, 3, pages - 2, pages - 3]
    near = [torch.empty(4, n_kv, page, hd, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)] + [torch.empty(4, n_kv, device="cuda") for _ in range(2)]
    rotary = ops.Rotary(hd)
    k, v, q = (torch.randn(400, h, hd, device="cuda").to(torch.bfloat16) for h in (n_kv, n_kv, 16))
    for c, where in ((cache, used), (near, [0, 1, 2, 3])):
        ops.pf_kv_append_rope(*c, None, k, v, d32([0, 300, 400]), d32([0, 0]), d32([where[:3], [where[3]] * 3]), rotary, max_new=300)
    at = torch.tensor(used, device="cuda")
    assert all(torch.equal(c[at], n) for c, n in zip(cache[2:], near[2:]))
    for c, n in zip(cache[:2], near[:2]):
        got, want = c.view(torch.uint8)[at], n.view(torch.uint8)
        assert torch.equal(got[:2], want[:2]) and torch.equal(got[2][:, :44], want[2][:, :44]) and torch.equal(got[3][:, :100], want[3][:, :100])
    rest = d32([0] * 5)
    for own in (rest, d32([100] * 5)):
        a, b = (ops.pf_prefix_attention(q[:5], *c, own, d32([[w[3]]] * 5), d32([300]), d32([w[:3]]), lse=True) for c, w in ((cache, used), (near, [0, 1, 2, 3])))
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def test_calls_on_several_streams_at_once():
    import torch
    from paper_2607_18631_b200 import ops
    cases = [build(2, 128, 64, [40], [9000], [17 * i % 300 for i in range(40)], 16, seed=1), build(4, 64, 16, [3, 90], [700, 3000], [5] * 93, 16, seed=2),
             build(1, 128, 32, [200], [1500], [100] * 200, 8, seed=3)]
    want = [run(*c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    dev = [(c[0], *c[1], d32(c[2]), c[3], d32(c[4]), c[5], d32(c[6])) for c in cases]
    torch.cuda.synchronize()
    got = [[ops.pf_prefix_attention(*d, lse=True, stream=s) for d, s in zip(dev, streams)] for _ in range(6)]
    torch.cuda.synchronize()
    for round_ in got:
        for g, w in zip(round_, want):
            assert torch.equal(g["out"], w["out"]) and torch.equal(g["lse"], w["lse"])


def test_a_rotation_and_its_gradient_captured_together():
    import torch
    from paper_2607_18631_b200 import ops
    rotary, pos = ops.Rotary(48, layout="interleaved"), torch.arange(100, dtype=torch.int32, device="cuda")
    x, dy = (torch.randn(100, 3, 64, device="cuda").to(torch.float16) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    ops.pf_rope(x, pos, rotary)
    with torch.cuda.graph(graph):
        y = ops.pf_rope(x, pos, rotary)
        dx = ops.pf_rope(dy, pos, rotary, transposed=True)
    for shift in (0, 70000):
        pos += shift
        graph.replay()
        assert torch.equal(y, ops.pf_rope(x, pos, rotary)) and torch.equal(dx, ops.pf_rope(dy, pos, rotary, transposed=True))


def test_a_padded_batch_leaves_other_rows_as_they_were():
    """Queries of a padded batch rotated in place: rows that no sequence has, and rows past max_new, stay."""
    import torch
    from paper_2607_18631_b200 import ops
    cache, *_ = small()
    rotary = ops.Rotary(64)
    q = torch.randn(12, 4, 64, device="cuda").to(torch.bfloat16)
    k = torch.randn(12, 2, 64, device="cuda").to(torch.bfloat16)
    for max_new in (3, 5):                                # by sequence, and by row
        before = q.clone()
        ops.pf_kv_append_rope(*cache, q, k, k, d32([2, 8, 8, 9]), d32([0, 4, 1]), d32([[0], [1], [2]]), rotary, max_new=max_new, q_out=q)
        rows = torch.zeros(12, dtype=torch.bool, device="cuda")
        rows[2:2 + max_new] = rows[8] = True
        assert torch.equal(q[~rows], before[~rows])
        at = torch.zeros(12, dtype=torch.int32, device="cuda")
        at[2:8] = torch.arange(6, device="cuda")
        at[8] = 1
        assert torch.equal(q[rows], ops.pf_rope(before, at, rotary)[rows])
