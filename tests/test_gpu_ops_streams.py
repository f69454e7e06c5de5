"""The operators on another stream than their tensors': what a caller may drop at once, and what waits for what."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

DELAY = 20_000_000        # cycles that a stream is kept busy: some 10 ms


def weights(seed=0, E=16, H=512, F=256):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    mats = [rn(*s).mul(100).clamp(-448, 448).to(torch.float8_e4m3fn) for s in ((E, F, H), (E, F, H), (E, H, F))]
    scales = [torch.full((E, -(-m.shape[1] // 128), -(-m.shape[2] // 128)), 0.01 * m.shape[2] ** -0.5, device="cuda") for m in mats]
    return rn(E, H).mul(H ** -0.5).to(torch.bfloat16), mats, scales


def make(router, mats, scales, stream=None):
    from paper_2607_18631_b200 import ops
    return ops.MoeLayer(router, *mats, top_k=4, gate_scale=scales[0], up_scale=scales[1], down_scale=scales[2], stream=stream)


def test_weights_packed_on_a_side_stream_may_be_dropped_at_once():
    """The packing waits behind queued work; meanwhile the weights are dropped, their memory is asked for again and overwritten, and the
    layer is used on the default stream."""
    import torch
    x = torch.randn(5, 512, device="cuda").to(torch.bfloat16)
    want = make(*weights()).forward(x)
    side = torch.cuda.Stream()
    router, mats, scales = weights()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY)
    layer = make(router, mats, scales, stream=side)
    sizes = [(t.shape, t.dtype) for t in mats + scales]
    del mats, scales
    rubbish = [torch.full(shape, float("nan"), device="cuda").to(dtype) for shape, dtype in sizes for _ in range(2)]
    got = layer.forward(x)
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want), len(rubbish)


def test_a_packing_waits_for_weights_that_are_still_being_made():
    import torch
    x = torch.randn(3, 512, device="cuda").to(torch.bfloat16)
    router, mats, scales = weights(1)
    want = make(router, mats, scales).forward(x)
    late = [torch.zeros_like(m) for m in mats]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(DELAY)
    for dst, src in zip(late, mats):
        dst.copy_(src)
    layer = make(router, late, scales, stream=side)
    got = layer.forward(x, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_a_layer_dropped_while_another_stream_reads_it():
    import torch
    x = torch.randn(5, 512, device="cuda").to(torch.bfloat16)
    args = weights(2)
    want = make(*args).forward(x)
    layer, side = make(*args), torch.cuda.Stream()
    size = layer.packed.numel()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY)
        got = layer.forward(x)
    del layer
    rubbish = [torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want), len(rubbish)


def test_inputs_of_a_call_on_another_stream_may_be_dropped_at_once():
    import torch
    from paper_2607_18631_b200 import ops
    side = torch.cuda.Stream()
    x = torch.randn(64, 4096, device="cuda").to(torch.bfloat16)
    want = ops.pf_add_rms_norm(x, x, y=True)
    mine, res = x.clone(), x.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY)
    got = ops.pf_add_rms_norm(mine, res, y=True, stream=side)
    del mine, res
    rubbish = [torch.full_like(x, float("nan")) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(got[n].view(torch.uint8), want[n].view(torch.uint8)) for n in want), len(rubbish)
