"""The decode layer against the plan it stands for (CPU) and its parts against the formulas in 64 bits, each against its own size (GPU)."""
from __future__ import annotations

import math

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


# ------------------------------------------------------------------ on a GPU
def build(monkeypatch, **shape):
    """A layer and the weights its expert layers were made of: [(router, matrices in 64 bits, n_shared)]."""
    from paper_2607_18631_b200 import ops
    made, real = [], ops.MoeLayer

    def block(w, scale):
        if scale is None:
            return w.double()
        return w.double() * scale.repeat_interleave(128, 1)[:, :w.shape[1]].repeat_interleave(128, 2)[:, :, :w.shape[2]].double()

    def record(router, gate, up, down, *, gate_scale=None, up_scale=None, down_scale=None, n_shared=0, **kw):
        made.append((router.double(), [block(w, s) for w, s in ((gate, gate_scale), (up, up_scale), (down, down_scale))], n_shared))
        return real(router, gate, up, down, gate_scale=gate_scale, up_scale=up_scale, down_scale=down_scale, n_shared=n_shared, **kw)
    monkeypatch.setattr(ops, "MoeLayer", record)
    return D.DecodeLayer(shape, context=7, page=16, seed=4), made


def norm(t):
    import torch
    return t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-6)


def experts(y, made, top_k):
    """The layers' formula for tokens y in 64 bits."""
    import torch
    out = torch.zeros_like(y)
    for router, (gate, up, down), n_shared in made:
        local = gate.shape[0] - n_shared
        chosen, ids = torch.sort(y @ router.T, dim=1, descending=True, stable=True)
        w = torch.softmax(chosen[:, :top_k], 1)
        for e in range(gate.shape[0]):
            part = (w * (ids[:, :top_k] == e)).sum(1) if e < local else torch.ones(y.shape[0], dtype=y.dtype, device=y.device)
            g = y @ gate[e].T
            out += part[:, None] * ((g * torch.sigmoid(g) * (y @ up[e].T)) @ down[e].T)
    return out


def far(a, b):
    return float((a - b).norm() / b.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("weights", ["bf16", "e4m3"])
@pytest.mark.parametrize("more", [dict(shared=1), dict(shared=1, expert_tokens=21, shared_ffn=160)])
def test_each_part_of_a_step_against_its_own_size(weights, more, monkeypatch):
    """Relative 2-norm errors, roundings taken as independent (a rounding to bf16 is 2^-8 / sqrt(3) of the value, to e4m3 2^-4 / sqrt(3)).

    What attention adds: scores of size sm |q| |k| = 8 carry the roundings of y and q, 0.0032 of it, so the weights are off by 0.026; the stream's own
    rounding is 0.0023 of it and the stream some 4 times what attention adds with 8 cached tokens: 0.03 together, held to 2^-3.  The newest token's key
    and value, from y and k in bf16 and one rounding to e4m3: 0.04, held to 2^-3.  What the experts add: bf16 tokens, hidden activations and sums, 0.01, held to
    2^-4; e4m3 tokens 0.036 through two factors, 0.06, held to 2^-3.  An oracle with a mistake has to lie beyond the bound."""
    import torch
    T, hd = 5, 64
    shape = dict(tokens=T, hidden=256, heads=8, kv_heads=2, head_dim=hd, experts=8, local=8, top_k=2, ffn=96, weights=weights, **more)
    layer, made = build(monkeypatch, **shape)
    assert len(made) == (2 if "shared_ffn" in more else 1)
    g = torch.Generator(device="cuda").manual_seed(9)
    x, residual = (torch.randn(T, 256, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    for _ in range(3):
        n = layer.cached + 1
        before = residual.double() + x.double()
        out = layer.step(x, residual)
        qkv = (norm(before) @ layer.w_qkv.double().T).reshape(T, 12, hd)
        q, newest = qkv[:, :8], qkv[:, 8:]

        def attention(tokens=n, scale=1 / math.sqrt(hd), part=1.0):
            a = torch.zeros(T, 8, hd, dtype=torch.float64, device="cuda")
            for b in range(T):
                pages = layer.table[b, :-(-n // 16)].long()
                k, v = ((c[pages].double() * s[pages].double()[:, :, None, None]).transpose(1, 2).reshape(-1, 2, hd)[:n] for c, s in zip(layer.cache, layer.scales))
                assert far(torch.cat([k[n - 1], v[n - 1]]), newest[b]) < 2.0 ** -3
                for h in range(8):
                    a[b, h] = torch.softmax(k[:tokens, h // 4] @ q[b, h] * scale, 0) @ v[:tokens, h // 4]
            return part * a.flatten(1) @ layer.w_out.double().T
        added = residual.double() - before
        assert far(added, attention()) < 2.0 ** -3
        for mistake in (dict(part=0.5), dict(scale=1 / 16), dict(tokens=n - 1)):
            assert far(added, attention(**mistake)) > 2.0 ** -3, mistake
        y = norm(residual.double())
        bound = 2.0 ** -4 if weights == "bf16" else 2.0 ** -3
        assert far(out.double(), experts(y, made, 2)) < bound
        assert far(out.double(), experts(y, [(r, [m[:8] for m in ws], 0) for r, ws, _ in made], 2)) > bound      # no shared expert
        x = out
    layer.check()


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
