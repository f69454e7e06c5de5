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
