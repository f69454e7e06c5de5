"""Rotary positions: 32-bit arithmetic throughout, so that an element much smaller than its pair is rounded as exactly as the others.

Tolerance.  A pair's angle is exact to 2^-32 turns, 2 pi 2^-32 radians times the pair's length r and the amplitude.  With one element of the pair 0 the result is the other times
amplitude times cosine or sine: sine and cosine in 32 bits with 2^-23 of their own size, amplitude and product with 2^-24 each, so 2^-22 relative, and half a step of the type."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

PART = dict(bfloat16=2.0 ** -8, float16=2.0 ** -11, float32=2.0 ** -24)
STEP = dict(bfloat16=2.0 ** -134, float16=2.0 ** -25, float32=2.0 ** -150)      # half a step below the normals


def near_quarter_turns(n):
    """Angles at 2^-2 to 2^-16 radians, either side, from each quarter of a turn, and some anywhere."""
    out = []
    for i in range(n):
        off = 2.0 ** (-2 - 14 * ((i * 0.6180339887) % 1)) * (-1) ** i
        out.append(i % 4 * math.pi / 2 + off if i % 5 else 7.0 * ((i * 0.7548776662) % 1))
    return out


def check(got, x, angles, layout, amplitude):
    import torch
    n = len(angles)
    t = torch.tensor(angles, dtype=torch.float64)
    x = x.double().cpu()
    i = torch.arange(n)
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    c, s = amplitude * torch.cos(t), amplitude * torch.sin(t)
    want, r = x.clone(), torch.zeros_like(x)
    want[..., a], want[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    r[..., a] = r[..., b] = abs(amplitude) * torch.hypot(x[..., a], x[..., b])
    name = str(got.dtype).split(".")[1]
    err = (got.double().cpu() - want).abs()
    bound = want.abs() * (PART[name] + 2.0 ** -22) + r * 2 * math.pi * 2.0 ** -32 + STEP[name]
    assert torch.all(err <= bound), float((err / bound).max())


def heads(tokens, n, hd, rot, dtype, layout):
    """Of each pair one element or the other is 0."""
    import torch
    x = torch.randn(tokens, n, hd, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").abs().add(0.5).to(getattr(torch, dtype))
    for t in range(tokens):
        if layout == "half":
            x[t, :, rot // 2:rot] *= t % 2
            x[t, :, :rot // 2] *= 1 - t % 2
        else:
            x[t, :, t % 2:rot:2] = 0
    return x


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,rot,amplitude", [(128, 128, 1.0), (256, 192, 0.75), (50, 50, 1.0), (80, 40, -1.25)])
def test_rope_next_to_quarter_turns(hd, rot, amplitude, layout, dtype):
    import torch
    from paper_2607_18631_b200 import ops
    angles = near_quarter_turns(rot // 2)
    rotary = ops.Rotary(rot, layout=layout, frequencies=angles, amplitude=amplitude)
    x = heads(6, 9, hd, rot, dtype, layout)
    one = torch.ones(6, dtype=torch.int32, device="cuda")
    check(ops.pf_rope(x, one, rotary)[..., :rot], x[..., :rot], angles, layout, amplitude)
    check(ops.pf_rope(x, one, rotary, transposed=True)[..., :rot], x[..., :rot], [-a for a in angles], layout, amplitude)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("new", [[1] * 6, [6]])
def test_the_appends_queries_next_to_quarter_turns(layout, dtype, new):
    import torch
    from paper_2607_18631_b200 import ops
    angles = near_quarter_turns(64)
    rotary = ops.Rotary(128, layout=layout, frequencies=angles)
    cache = [torch.zeros(6, 1, 16, 128, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)] + [torch.ones(6, 1, device="cuda") for _ in range(2)]
    d = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, k = heads(6, 9, 128, 128, dtype, layout), heads(6, 1, 128, 128, dtype, layout)
    cu = [sum(new[:i]) for i in range(len(new) + 1)]
    got = ops.pf_kv_append_rope(*cache, q, k, k, d(cu), d([0] * len(new)), d([[i] for i in range(len(new))]), rotary, max_new=max(new), positions=d([1] * 6))
    check(got, q, angles, layout, 1.0)
