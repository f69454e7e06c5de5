"""The decode layer that runs the operators together: shapes from a plan (CPU), a step against the formulas (GPU)."""
from __future__ import annotations

import math

import pytest

from paper_2607_18631_b200 import PlanfrontError
from paper_2607_18631_b200 import decode_layer as D


def test_shapes_follow_the_plan():
    cfg = D.example_space(64, 1024)
    base = dict(kv=0, batch=64, dpa=0, ep=1, tp=1)
    s = D.layer_shape(cfg, base)
    assert (s["heads"], s["kv_heads"], s["local"], s["ffn"], s["tokens"], s["weights"], s["shared"]) == (32, 8, 64, 1408, 64, "bf16", 2)
    s = D.layer_shape(cfg, dict(base, kv=1, tp=8, ep=4))
    assert (s["heads"], s["kv_heads"], s["local"], s["ffn"], s["weights"]) == (4, 1, 16, 704, "e4m3")
    s = D.layer_shape(cfg, dict(base, dpa=1, tp=2, ep=4))
    assert (s["tokens"], s["local"], s["ffn"]) == (16, 16, 704)
    cfg["model"]["attn_kind"] = 1
    with pytest.raises(PlanfrontError):
        D.layer_shape(cfg, base)
    cfg = D.example_space(64, 1024)
    with pytest.raises(PlanfrontError):
        D.layer_shape(cfg, dict(base, tp=5))


def test_measured_rate_enters_the_cluster():
    cfg = D.example_space(8, 512)
    new = D.with_measured_hbm(cfg, {"attention": (10.0, 40_000_000), "experts": (30.0, 160_000_000)})
    assert new["cluster"]["hbm_bw"] == pytest.approx(5e12) and cfg["cluster"]["hbm_bw"] == 7.7e12


@pytest.mark.gpu
@pytest.mark.parametrize("weights", ["bf16", "e4m3"])
def test_step_is_the_layers_formula(weights):
    """Three steps against the layer in 64 bits.  Each stage rounds its output to bf16 (2^-8) or, in front of e4m3 experts, to e4m3 (2^-4); stages
    after a rounding carry it on with gains of order one, so the parts added to the stream are held to a relative 2-norm error of 2^-4 (bf16: five
    stages of 2^-8 and the cache's e4m3, averaged over the context, stay below it) and 2^-2 for e4m3 activations."""
    import torch
    shape = dict(tokens=5, hidden=256, heads=8, kv_heads=2, head_dim=64, experts=8, local=8, top_k=2, ffn=96, shared=1, weights=weights)
    layer = D.DecodeLayer(shape, context=100, page=16, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(5, 256, generator=g, device="cuda").to(torch.bfloat16)
    residual = torch.randn(5, 256, generator=g, device="cuda").to(torch.bfloat16)
    for step in range(3):
        n0 = layer.cached
        before = residual.double() + x.double()
        out = layer.step(x, residual)
        assert layer.cached == n0 + 1 and torch.all(layer.lengths == n0 + 1)
        norm = lambda t: t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-6)  # noqa: E731
        q = (norm(before) @ layer.w_qkv.double().T)[:, :8 * 64].reshape(5, 8, 64)
        attn = torch.zeros(5, 8, 64, dtype=torch.float64, device="cuda")
        for b in range(5):
            pages = layer.table[b, :-(-(n0 + 1) // 16)].long()
            k, v = ((c[pages].double() * s[pages].double()[:, :, None, None]).transpose(1, 2).reshape(-1, 2, 64)[:n0 + 1] for c, s in zip(layer.cache, layer.scales))
            for h in range(8):
                w = torch.softmax(k[:, h // 4] @ q[b, h] / math.sqrt(64), 0)
                attn[b, h] = w @ v[:, h // 4]
        stream = before + attn.flatten(1) @ layer.w_out.double().T
        assert float((residual.double() - stream).norm() / stream.norm()) < 2.0 ** -4
        y = norm(residual.double()).to(torch.bfloat16)
        got = layer.moe.forward(y)["out"].double()         # the experts on the same stream, without 8-bit tokens
        assert float((out.double() - got).norm() / got.norm()) < (2.0 ** -4 if weights == "bf16" else 2.0 ** -2)
        x = out
    layer.cached = layer.room
    with pytest.raises(PlanfrontError):
        layer.step(x, residual)


@pytest.mark.gpu
def test_the_command_runs(capsys):
    D.main(["--batch", "4", "--context", "300", "--steps", "2"])
    out = capsys.readouterr().out
    assert "attention" in out and "experts" in out and "tokens/s/GPU" in out
