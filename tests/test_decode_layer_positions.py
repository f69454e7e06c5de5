"""The decode layer with rotary positions and a shared prefix: its parts together, step by step, against the formulas in 64 bits."""
from __future__ import annotations

import math

import pytest

from paper_2607_18631_b200 import decode_layer as D

pytestmark = pytest.mark.gpu


def shape(weights="bf16", **kw):
    return dict(dict(tokens=6, hidden=256, heads=8, kv_heads=2, head_dim=64, experts=8, local=8, top_k=2, ffn=96, shared=1, weights=weights), **kw)


def rotated(x, positions, rotary):
    """[tokens, heads, hd] in 64 bits, halves of the first `rot` elements."""
    import torch
    f = torch.tensor(rotary.frequencies, dtype=torch.float64, device=x.device)
    t = positions.double()[:, None, None] * f
    n = len(f)
    a, b = x[..., :n], x[..., n:2 * n]
    return torch.cat([a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin(), x[..., 2 * n:]], -1)


@pytest.mark.parametrize("prefix,rotary", [(0, dict(rot=64)), (200, None), (200, dict(rot=64, base=500000.0)), (77, dict(rot=32)), (16, dict(rot=64, scaling="linear", factor=4.0))])
def test_steps_are_the_layers_formula(prefix, rotary):
    """Tolerances as for the layer without positions: five stages of 2^-8 and the cache's e4m3 averaged over the context stay below 2^-4 of the stream."""
    import torch
    layer = D.DecodeLayer(shape(), context=37, page=16, seed=3, prefix=prefix, rotary=rotary)
    g = torch.Generator(device="cuda").manual_seed(5)
    x, residual = (torch.randn(6, 256, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))

    def tokens(row, n):
        pages = row[:-(-n // 16)].long()
        return [(c[pages].double() * s[pages].double()[:, :, None, None]).transpose(1, 2).reshape(-1, 2, 64)[:n] for c, s in zip(layer.cache, layer.scales)]
    for step in range(3):
        n0 = layer.cached
        before = residual.double() + x.double()
        out = layer.step(x, residual)
        assert layer.cached == n0 + 1 and torch.all(layer.lengths == n0 + 1)
        norm = lambda t: t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-6)  # noqa: E731
        y = norm(before)
        qkv = (y @ layer.w_qkv.double().T).unflatten(1, (12, 64))
        q, k_new = qkv[:, :8], qkv[:, 8:10]
        at = torch.full((6,), prefix + n0, device="cuda")
        if rotary:
            q, k_new = rotated(q, at, layer.rotary), rotated(k_new, at, layer.rotary)
        attn = torch.zeros(6, 8, 64, dtype=torch.float64, device="cuda")
        for b in range(6):
            k, v = tokens(layer.table[b], n0 + 1)
            # the newest key: bf16 roundings of the norm and the projection (2^-8 of the head's largest products), and e4m3's 2^-4 of the element or half its least step
            big = k_new[b].abs().amax()
            assert torch.all((k[-1] - k_new[b]).abs() <= k_new[b].abs() * 2.0 ** -4 + big * (2.0 ** -6 + 2.0 ** -10 * 448 / 224))
            if prefix:
                k, v = (torch.cat([p, own]) for p, own in zip(tokens(layer.prefix_table[0], prefix), (k, v)))
            for h in range(8):
                w = torch.softmax(k[:, h // 4] @ q[b, h] / math.sqrt(64), 0)
                attn[b, h] = w @ v[:, h // 4]
        stream = before + attn.flatten(1) @ layer.w_out.double().T
        assert float((residual.double() - stream).norm() / stream.norm()) < 2.0 ** -4
        x = out
    layer.check()


def test_a_shared_prefix_is_every_sequences_own():
    """The same tokens as a prefix and as each sequence's first ones: scores depend on differences of positions only, and where they lie does not matter."""
    import torch
    shared = D.DecodeLayer(shape(), context=32, page=16, seed=7, prefix=64, rotary=dict(rot=64))
    alone = D.DecodeLayer(shape(), context=96, page=16, seed=7, rotary=dict(rot=64))
    for c, s in ((0, 0), (1, 1)):                         # the other layer's pages become copies: the prefix's four, then the own ones
        for b in range(6):
            for i in range(4):
                alone.cache[c].view(torch.uint8)[alone.table[b, i].long()] = shared.cache[c].view(torch.uint8)[shared.prefix_table[0, i].long()]
                alone.scales[s][alone.table[b, i].long()] = shared.scales[s][shared.prefix_table[0, i].long()]
            for i in range(2):
                alone.cache[c].view(torch.uint8)[alone.table[b, 4 + i].long()] = shared.cache[c].view(torch.uint8)[shared.table[b, i].long()]
                alone.scales[s][alone.table[b, 4 + i].long()] = shared.scales[s][shared.table[b, i].long()]
    x = torch.randn(6, 256, device="cuda").to(torch.bfloat16)
    r1, r2 = torch.zeros_like(x), torch.zeros_like(x)
    shared.step(x, r1)
    alone.step(x, r2)
    # both attentions within 2^-11 weights of the exact one and rounded to bf16; the projection carries that on
    assert float((r1.double() - r2.double()).norm() / r2.double().norm()) < 2.0 ** -7


def test_the_command_runs_with_a_prefix_and_positions(capsys):
    D.main(["--batch", "4", "--context", "100", "--steps", "2", "--prefix", "500", "--rope", "10000"])
    out = capsys.readouterr().out
    assert "attention" in out and "experts" in out and "tokens/s/GPU" in out
