"""Arguments that would have the kernels write outside their tensors are refused on the host: nothing is launched."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu


def refused(call):
    from paper_2607_18631_b200 import PlanfrontError
    from paper_2607_18631_b200.binding import pf_launch_count
    before = pf_launch_count()
    with pytest.raises(PlanfrontError):
        call()
    assert pf_launch_count() == before


def moe_layer():
    import torch
    from paper_2607_18631_b200 import ops
    w = [torch.randn(*s, device="cuda").to(torch.bfloat16) for s in ((8, 128), (8, 32, 128), (8, 32, 128), (8, 128, 32))]
    return ops.MoeLayer(*w, top_k=2), torch.randn(3, 128, device="cuda").to(torch.bfloat16)


def workspaces():
    """Tensors whose elements are more than the bytes behind them, or do not lie side by side."""
    import torch
    small = torch.zeros(1, dtype=torch.uint8, device="cuda")
    return small.expand(1 << 25), torch.zeros(1 << 25, dtype=torch.uint8, device="cuda")[::2], torch.zeros(64, 64, device="cuda").unfold(0, 32, 1)


def test_workspaces_that_overlap_are_refused():
    import torch
    from paper_2607_18631_b200 import ops
    layer, x = moe_layer()
    cache = [torch.zeros(4, 2, 16, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)] + [torch.ones(4, 2, device="cuda") for _ in range(2)]
    q, table = torch.randn(2, 4, 64, device="cuda").to(torch.bfloat16), torch.arange(4, dtype=torch.int32, device="cuda").reshape(2, 2)
    lengths = torch.tensor([5, 20], dtype=torch.int32, device="cuda")
    for ws in workspaces():
        refused(lambda: layer.forward(x, workspace=ws))
        refused(lambda: ops.pf_decode_attention(q, *cache, lengths, table, workspace=ws))


def test_a_status_that_is_not_one_word_is_refused():
    import torch
    layer, x = moe_layer()
    for bad in (torch.zeros(1, dtype=torch.uint8, device="cuda"), torch.zeros(2, dtype=torch.int16, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.float32, device="cuda")):
        refused(lambda: layer.forward(x, status=bad))
    ok = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    layer.forward(x, status=ok)
    assert int(ok) == 0


def test_counts_that_do_not_fit_32_bits_are_refused():
    """2^32 + 3 is not 3."""
    import torch
    from paper_2607_18631_b200 import ops
    big = 1 << 32
    d = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = [torch.zeros(4, 2, 16, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)] + [torch.ones(4, 2, device="cuda") for _ in range(2)]
    k, table, x = torch.randn(3, 2, 64, device="cuda").to(torch.bfloat16), d(0, 1).reshape(1, 2), torch.randn(2, 256, device="cuda")
    refused(lambda: ops.pf_kv_append(*cache, k, k, d(0, 3), d(0), table, max_new=big + 3))
    refused(lambda: ops.pf_add_rms_norm(x, group=big + 128))
    w = [torch.randn(*s, device="cuda").to(torch.bfloat16) for s in ((8, 128), (8, 32, 128), (8, 32, 128), (8, 128, 32))]
    for kw in (dict(top_k=big + 2), dict(top_k=2, first_expert=big), dict(top_k=2, n_shared=-big)):
        refused(lambda: ops.MoeLayer(*w, **kw))


def test_a_stream_of_another_device_is_refused():
    import torch
    from paper_2607_18631_b200 import ops

    class Elsewhere:
        device_index, cuda_stream = torch.cuda.current_device() + 1, 0
    layer, x = moe_layer()
    d = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = [torch.zeros(4, 2, 16, 64, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)] + [torch.ones(4, 2, device="cuda") for _ in range(2)]
    k, table = torch.randn(3, 2, 64, device="cuda").to(torch.bfloat16), d(0, 1).reshape(1, 2)
    w = [torch.randn(*s, device="cuda").to(torch.bfloat16) for s in ((8, 128), (8, 32, 128), (8, 32, 128), (8, 128, 32))]
    for call in (lambda: ops.pf_add_rms_norm(x, stream=Elsewhere()), lambda: ops.pf_kv_append(*cache, k, k, d(0, 3), d(0), table, max_new=3, stream=Elsewhere()),
                 lambda: ops.pf_decode_attention(k[:1], *cache, d(3), table, stream=Elsewhere()), lambda: layer.forward(x, stream=Elsewhere()),
                 lambda: ops.MoeLayer(*w, top_k=2, stream=Elsewhere())):
        refused(call)
