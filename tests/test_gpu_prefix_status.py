"""The status word of pf_prefix_attention: 0 after a complete call, 1 after one of which a wait ran out; the decode layer reads it."""
from __future__ import annotations

import pytest

from test_gpu_ops_refusals import refused
from test_gpu_prefix_attention import build, d32, run

pytestmark = pytest.mark.gpu


@pytest.fixture
def lost_wait():
    """While it lasts a block of the kernel waits in vain, 500 polls (a millisecond) long."""
    from paper_2607_18631_b200.binding import load_library
    L = load_library()
    yield lambda on: L.pf_prefix_waits(500 if on else 0, int(on))
    assert L.pf_prefix_waits(0, 0) == 0


@pytest.mark.parametrize("B,heads,n_kv,length,hd", [(1, 1, 1, 1, 64), (3, 8, 2, 600, 128), (200, 8, 2, 4000, 64), (40, 16, 4, 30000, 128)])
def test_a_wait_that_runs_out_is_reported(B, heads, n_kv, length, hd, lost_wait):
    import torch
    args = build(n_kv, hd, 64, [B], [length], [i % 50 for i in range(B)], heads)
    words = d32([7, 7, 7])
    want = run(*args, status=words[1:2])
    assert words.tolist() == [7, 0, 7] and torch.isfinite(want["out"].float()).all()
    assert lost_wait(True) == 0
    got = run(*args, status=words[1:2])
    assert words.tolist() == [7, 1, 7] and torch.isnan(got["out"].float()).any()
    assert lost_wait(False) == 0
    again = run(*args, status=words[1:2])
    assert words.tolist() == [7, 0, 7] and torch.equal(again["out"], want["out"])


def test_calls_without_a_wait_are_complete():
    """No group, no column, no prefix token, no sequence."""
    from paper_2607_18631_b200 import ops
    q, cache, own, table, plen, ptable, cu = build(2, 64, 16, [4], [50], [9] * 4, 8)
    calls = [(q, own, table, [], ptable[:0], [0]), (q, own, table, plen, ptable[:, :0].contiguous(), cu), (q, own, table, [0], ptable, cu), (q[:0], [], table[:0], plen, ptable, [0, 0]),
             (q, [0] * 4, table, [0], ptable, cu)]
    for q_, own_, table_, plen_, ptable_, cu_ in calls:
        word = d32([7])
        ops.pf_prefix_attention(q_, *cache, d32(own_), table_, d32(plen_), ptable_, d32(cu_), status=word)
        assert int(word) == 0


def test_a_status_that_is_not_one_word_is_refused():
    import torch
    args = build(2, 64, 16, [4], [50], [9] * 4, 8)
    for bad in (torch.zeros(1, dtype=torch.uint8, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"),
                torch.zeros(1, dtype=torch.float32, device="cuda"), torch.zeros(1, dtype=torch.int32)):
        refused(lambda: run(*args, status=bad))


def test_a_captured_call_reports_each_time(lost_wait):
    import torch
    from paper_2607_18631_b200 import ops
    q, cache, own, table, plen, ptable, cu = build(2, 64, 16, [4], [500], [9] * 4, 8)
    dev, word, graph = (d32(own), table, d32(plen), ptable, d32(cu)), d32([7]), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.pf_prefix_attention(q, *cache, *dev, status=word)
    for _ in range(2):
        word.fill_(7)
        graph.replay()
        assert int(word) == 0


def test_the_decode_layer_says_so(lost_wait):
    import torch
    from paper_2607_18631_b200 import PlanfrontError
    from paper_2607_18631_b200 import decode_layer as D
    shape = dict(tokens=6, hidden=256, heads=8, kv_heads=2, head_dim=64, experts=8, local=8, top_k=2, ffn=96, shared=1, weights="bf16")
    layer = D.DecodeLayer(shape, context=37, page=16, seed=3, prefix=200)
    x, residual = (torch.randn(6, 256, device="cuda").to(torch.bfloat16) for _ in range(2))
    layer.step(x, residual)
    layer.check()
    assert lost_wait(True) == 0
    layer.step(x, residual)
    with pytest.raises(PlanfrontError, match="prefixes"):
        layer.check()
    assert lost_wait(False) == 0
    layer.step(x, torch.zeros_like(residual))
    layer.check()
