"""The decode layer against the plan it stands for (CPU) and its parts against the formulas in 64 bits, each against its own size (GPU)."""
from __future__ import annotations

import pytest

from paper_2607_18631_b200 import PlanfrontError
from paper_2607_18631_b200 import decode_layer as D

BASE = dict(kv=0, batch=64, dpa=0, ep=1, tp=1)


def space(**model):
    cfg = D.example_space(64, 1024)
    cfg["model"].update(model)
    return cfg


def test_experts_see_the_tokens_of_all_attention_groups():
    """The serving model routes the whole batch to the experts, whoever runs its attention."""
    s = D.layer_shape(space(), dict(BASE, dpa=1, tp=2, ep=4))
    assert s["tokens"] == 16 and s["expert_tokens"] == 64
    s = D.layer_shape(space(), dict(BASE, tp=8, ep=4))
    assert s["tokens"] == s["expert_tokens"] == 64


def test_shared_experts_of_any_width_are_held():
    s = D.layer_shape(space(), dict(BASE, tp=2))
    assert (s["shared"], s["shared_ffn"], s["ffn"]) == (2, 704, 704)
    s = D.layer_shape(space(Fs=2816), dict(BASE, tp=2))
    assert (s["shared"], s["shared_ffn"], s["ffn"]) == (2, 1408, 704)
    s = D.layer_shape(space(), dict(BASE, tp=8, ep=4))     # routed experts are split over 2, dense weights over 8
    assert (s["shared"], s["shared_ffn"], s["ffn"]) == (2, 176, 704)
    assert D.layer_shape(space(S=0), BASE)["shared"] == 0


def test_heads_that_do_not_split_are_refused():
    assert D.layer_shape(space(nh=24, nkv=6), dict(BASE, tp=3))["kv_heads"] == 2
    assert D.layer_shape(space(nh=24, nkv=4), dict(BASE, tp=8))["kv_heads"] == 1      # two GPUs hold the same head
    for nkv, tp in ((6, 4), (3, 2), (12, 8), (5, 4)):
        with pytest.raises(PlanfrontError):
            D.layer_shape(space(nh=24, nkv=nkv), dict(BASE, tp=tp))
    with pytest.raises(PlanfrontError):
        D.layer_shape(space(), dict(BASE, batch=2, dpa=1, ep=4))


def test_parts_too_small_for_a_rate_do_not_enter_the_cluster():
    cfg = D.example_space(8, 512)
    big, tiny = (20.0, 100_000_000), (9.0, 2_500_000)
    assert D.with_measured_hbm(cfg, {"attention": tiny, "experts": big})["cluster"]["hbm_bw"] == pytest.approx(5e12)
    assert D.with_measured_hbm(cfg, {"attention": tiny, "experts": tiny})["cluster"]["hbm_bw"] == cfg["cluster"]["hbm_bw"]


@pytest.mark.gpu
def test_measured_parts_come_from_hbm():
    """A cache of 34 MB, which the L2 would hold: measured as a call is after other work has gone through the L2."""
    import torch
    shape = dict(tokens=64, hidden=512, heads=16, kv_heads=4, head_dim=128, experts=4, local=4, top_k=1, ffn=64, shared=0, weights="bf16")
    layer = D.DecodeLayer(shape, context=500, page=64)
    parts = layer.measure()
    assert set(parts) == {"attention", "experts"} and parts["attention"][1] == 64 * 500 * 4 * 128 * 2
    q = torch.randn(64, 16, 128, device="cuda").to(torch.bfloat16)
    filler = torch.zeros(1 << 29, dtype=torch.uint8, device="cuda")
    cold = []
    for _ in range(10):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        filler.view(torch.int32).amax()
        a.record()
        layer.attend(q)
        b.record()
        torch.cuda.synchronize()
        cold.append(a.elapsed_time(b) * 1e3)
    assert parts["attention"][0] > 0.75 * sorted(cold)[5]


@pytest.mark.gpu
def test_a_wait_that_ran_out_is_raised():
    import torch
    from paper_2607_18631_b200.binding import load_library
    L = load_library()
    shape = dict(tokens=3, hidden=256, heads=4, kv_heads=2, head_dim=64, experts=4, local=4, top_k=2, ffn=64, shared=0, weights="bf16")
    layer = D.DecodeLayer(shape, context=5, page=16)
    x, residual = (torch.randn(3, 256, device="cuda").to(torch.bfloat16) for _ in range(2))
    assert L.pf_moe_meeting(2000, 1) == 0
    try:
        assert torch.isnan(layer.step(x, residual.clone()).float()).all()
        with pytest.raises(PlanfrontError):
            layer.check()
    finally:
        assert L.pf_moe_meeting(0, 0) == 0
    layer.step(x, residual)
    layer.check()
