"""pf_rope in a backward pass: the gradient is the transposed rotation of the result's gradient.

Tolerance, with r the length of a pair of what is rotated: sines and cosines 2^-23, amplitude, two products and a sum 2^-24 each, so amplitude r 2^-21, and half a step of the type."""
from __future__ import annotations

import pytest

from test_gpu_ops_refusals import refused

pytestmark = pytest.mark.gpu

PART = dict(bfloat16=2.0 ** -8, float16=2.0 ** -11, float32=2.0 ** -24)


def case(dtype="float32", tokens=50, heads=4, hd=64, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, dy = (torch.randn(tokens, heads, hd, generator=g, device="cuda").to(getattr(torch, dtype)) for _ in range(2))
    return x, dy, torch.randint(0, 1 << 20, (tokens,), generator=g, device="cuda").to(torch.int32)


def formula(x, positions, rotary):
    """64 bits, by operations that torch differentiates itself."""
    import torch
    n = rotary.rot // 2
    t = positions.double()[:, None, None] * torch.tensor(rotary.frequencies, dtype=torch.float64, device=x.device)
    c, s = rotary.amplitude * t.cos(), rotary.amplitude * t.sin()
    a, b = (x[..., :n], x[..., n:2 * n]) if rotary.layout == "half" else (x[..., 0:2 * n:2], x[..., 1:2 * n:2])
    u, v = a * c - b * s, b * c + a * s
    turned = torch.cat([u, v], -1) if rotary.layout == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * n:]], -1)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,rot", [(64, 64), (64, 48), (50, 34)])
@pytest.mark.parametrize("transposed", [False, True])
def test_the_gradient_is_the_formulas(dtype, layout, hd, rot, transposed):
    import torch
    from paper_2607_18631_b200 import ops
    x, dy, pos = case(dtype, hd=hd)
    rotary = ops.Rotary(rot, layout=layout, amplitude=1.25)
    exact = x.double().requires_grad_()
    turned = formula(exact, -pos if transposed else pos, rotary)
    want, = torch.autograd.grad(turned, exact, dy.double())
    x.requires_grad_()
    y = ops.pf_rope(x, pos, rotary, transposed=transposed)
    assert y.requires_grad and torch.equal(y.detach(), ops.pf_rope(x.detach(), pos, rotary, transposed=transposed))
    y.backward(dy)
    r = dy.double().norm(dim=-1, keepdim=True)          # no pair is longer than its head
    assert x.grad.dtype == x.dtype and torch.all((x.grad.double() - want).abs() <= 1.25 * r * 2.0 ** -21 + want.abs() * PART[dtype] * 1.001 + 2.0 ** -25)


def test_gradients_that_are_no_plain_tensors():
    """Of a sum (one number, expanded), of transposed heads, of a slice; and of x that is a slice."""
    import torch
    from paper_2607_18631_b200 import ops
    x, dy, pos = case()
    rotary = ops.Rotary(64)
    leaf = x.clone().requires_grad_()
    ops.pf_rope(leaf, pos, rotary).sum().backward()
    assert torch.equal(leaf.grad, ops.pf_rope(torch.ones_like(x), pos, rotary, transposed=True))
    want = ops.pf_rope(dy, pos, rotary, transposed=True)
    for given in (dy.transpose(0, 1).contiguous().transpose(0, 1), dy.transpose(1, 2).contiguous().transpose(1, 2), torch.cat([dy, dy], 1)[:, 2:6].clone(memory_format=torch.preserve_format)):
        leaf = x.clone().requires_grad_()
        ops.pf_rope(leaf, pos, rotary).backward(given)
        assert torch.equal(leaf.grad, ops.pf_rope(given.contiguous(), pos, rotary, transposed=True))
    wide = torch.zeros(50, 9, 64, device="cuda")
    wide[:, 3:7] = x
    wide.requires_grad_()
    ops.pf_rope(wide[:, 3:7], pos, rotary).backward(dy)
    assert torch.equal(wide.grad[:, 3:7], want) and not wide.grad[:, :3].any() and not wide.grad[:, 7:].any()
    empty = x[:0].clone().requires_grad_()
    ops.pf_rope(empty, pos[:0], rotary).sum().backward()
    assert empty.grad.shape == (0, 4, 64)


def test_against_differences_and_twice():
    """The map is linear, so a difference quotient of any step is the derivative; the gradient's gradient is the rotation again."""
    import torch
    from paper_2607_18631_b200 import ops
    x, dy, pos = case()
    rotary = ops.Rotary(48, layout="interleaved")
    leaf, given = x.clone().requires_grad_(), dy.clone().requires_grad_()
    y = ops.pf_rope(leaf, pos, rotary)
    grad, = torch.autograd.grad(y, leaf, given, create_graph=True)
    step = torch.zeros_like(x)
    step[:, :, 5] = 0.5
    slope = ((ops.pf_rope(x + step, pos, rotary).double() - y.detach().double()) * dy.double()).sum(-1) / 0.5
    # two rotations of heads up to |x| + 1 long, each off by 2^-21 of it, times |dy|, over the step
    assert torch.all((slope - grad[..., 5].double()).abs() <= (x.double().norm(dim=-1) + 1) * dy.double().norm(dim=-1) * 2.0 ** -18)
    twice, = torch.autograd.grad(grad, given, x)
    assert torch.equal(twice, ops.pf_rope(x, pos, rotary))


def test_where_no_graph_is_asked_for():
    import torch
    from paper_2607_18631_b200 import ops
    x, dy, pos = case()
    rotary = ops.Rotary(64)
    leaf = x.clone().requires_grad_()
    with torch.no_grad():
        assert not ops.pf_rope(leaf, pos, rotary).requires_grad
        out = torch.empty_like(x)
        assert ops.pf_rope(leaf, pos, rotary, out=out) is out
    for call in (lambda: ops.pf_rope(leaf, pos, rotary, out=out), lambda: ops.pf_rope(x, pos, rotary, out=leaf), lambda: ops.pf_rope(leaf, pos[:3], rotary),
                 lambda: ops.pf_rope(leaf[0], pos, rotary)):
        refused(call)
    y = ops.pf_rope(leaf, pos, rotary)
    pos += 1                                              # the backward pass needs what they were
    with pytest.raises(RuntimeError):
        y.backward(dy)


def test_on_another_stream_and_captured():
    import torch
    from paper_2607_18631_b200 import ops
    x, dy, pos = case("bfloat16")
    rotary = ops.Rotary(64)
    want = ops.pf_rope(dy, pos, rotary, transposed=True)
    side, leaf = torch.cuda.Stream(), x.clone().requires_grad_()
    torch.cuda.synchronize()
    y = ops.pf_rope(leaf, pos, rotary, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    grad, = torch.autograd.grad(y, leaf, dy)
    torch.cuda.synchronize()
    assert torch.equal(grad, want)
    del y, grad
    leaf, given, graph = x.clone().requires_grad_(), dy.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ops.pf_rope(leaf, pos, rotary)
        grad, = torch.autograd.grad(y, leaf, given)
    for shift in (0, 5):
        given.add_(shift)
        graph.replay()
        assert torch.equal(grad, ops.pf_rope(given, pos, rotary, transposed=True)) and torch.equal(y.detach(), ops.pf_rope(x, pos, rotary))
