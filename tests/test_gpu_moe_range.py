"""pf_moe_forward with e4m3 weights whose hidden units differ much in size.

Hidden activations enter the second product as fp16 numbers times a power of two that is known before they are: |h_f| <= |x|^2 p, p the product of the
largest gate and up row norms of the 128 units that f belongs to.  It is at most 2^-13 1.02 |x|^2 p, so fp16's least half
step, 2^-25, costs a unit less than 2^-37 |x|^2 p of its own block, whatever other blocks hold; other terms as in test_gpu_moe."""
from __future__ import annotations

import pytest

from test_gpu_moe import blocks, layer_inputs

pytestmark = pytest.mark.gpu


def check(x, router, ws, sc, ids, got):
    import torch
    T, H = x.shape
    F = ws[0].shape[1]
    xv = x.double()
    wts = torch.softmax((xv @ router.double().T).gather(1, ids.long()), 1)
    out, tol = (torch.zeros(T, H, dtype=torch.float64, device=x.device) for _ in range(2))
    e1, e2 = H * 2.0 ** -23 + 2.0 ** -11, 2.0 ** -11 + 2.0 ** -20
    for e in range(ws[0].shape[0]):
        w = (wts * (ids == e)).sum(1)
        rows = w.nonzero()[:, 0]
        if not rows.numel():
            continue
        gate, up, down = (m[e:e + 1].double() * blocks(m[e:e + 1], s[e:e + 1]) for m, s in zip(ws, sc))
        v = xv[rows]
        g, u = v @ gate[0].T, v @ up[0].T
        ag, au = v.abs() @ gate[0].abs().T, v.abs() @ up[0].abs().T
        silu = g * torch.sigmoid(g)
        h = silu * u
        p = torch.cat([torch.full((min(128, F - f),), float(gate[0, f:f + 128].norm(dim=1).amax() * up[0, f:f + 128].norm(dim=1).amax()), dtype=torch.float64, device=x.device)
                       for f in range(0, F, 128)])
        dh = e1 * (1.1 * ag * u.abs() + (silu.abs() + 1.1 * e1 * ag) * au) + e2 * h.abs() + 2.0 ** -37 * (v * v).sum(1, keepdim=True) * p
        y = h @ down[0].T
        out[rows] += w[rows, None] * y
        tol[rows] += w[rows, None] * ((dh + F * 2.0 ** -23 * h.abs()) @ down[0].abs().T + 2.0 ** -18 * y.abs())
    tol = tol + 2.0 ** -8 * (out.abs() + tol)
    err = (got.double() - out).abs()
    assert torch.all(err <= tol), float((err / tol).max())


@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("H,F", [(512, 512), (256, 300)])
@pytest.mark.parametrize("up_by,down_by", [(2.0 ** 14, 2.0 ** -28), (2.0 ** 14, 1e-12), (2.0 ** -14, 2.0 ** 20), (2.0 ** 10, 2.0 ** -10)])
def test_blocks_of_outlier_units(T, H, F, up_by, down_by):
    """One block's gate and up rows times `up_by` each, its down columns times `down_by`."""
    import torch
    from paper_2607_18631_b200 import ops
    x, router, ws, sc = layer_inputs(T, H, F, 4, 4, 0, "e4m3", seed=T + F)
    sc[0][:, 1] *= up_by
    sc[1][:, 1] *= up_by
    sc[2][:, :, 1] *= down_by
    layer = ops.MoeLayer(router, *ws, top_k=2, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2])
    got = layer.forward(x)
    check(x, router, ws, sc, got["ids"], got["out"])


@pytest.mark.parametrize("which", [0, 1])
def test_outliers_of_gate_and_up_in_different_blocks(which):
    import torch
    from paper_2607_18631_b200 import ops
    x, router, ws, sc = layer_inputs(9, 512, 640, 4, 4, 0, "e4m3", seed=which)
    sc[which][:, 1] *= 2.0 ** 20
    sc[1 - which][:, 3] *= 2.0 ** -20
    sc[2][:, :, 1] *= 2.0 ** -20
    sc[2][:, :, 3] *= 2.0 ** 20
    layer = ops.MoeLayer(router, *ws, top_k=2, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2])
    got = layer.forward(x)
    check(x, router, ws, sc, got["ids"], got["out"])


def test_an_outlier_unit_among_its_neighbours_and_an_outlier_channel():
    import torch
    from paper_2607_18631_b200 import ops
    x, router, ws, sc = layer_inputs(9, 512, 256, 4, 4, 0, "e4m3", seed=8)
    small = (ws[0].float() * 2.0 ** -5).to(torch.float8_e4m3fn), (ws[1].float() * 2.0 ** -5).to(torch.float8_e4m3fn)
    for s, w in zip(small, ws):
        s.view(torch.uint8)[:, 7] = w.view(torch.uint8)[:, 7]              # unit 7 is 2^5 above the others in both
    x[:, 100] *= 2.0 ** 6                                                  # and one channel 2^6 above the rest in every token
    ws = [*small, ws[2]]
    layer = ops.MoeLayer(router, *ws, top_k=2, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2])
    got = layer.forward(x)
    check(x, router, ws, sc, got["ids"], got["out"])


def test_weights_without_size_and_weights_that_are_not_numbers():
    """Empty experts give zeros; a NaN weight spoils what it enters and no other expert's tokens."""
    import torch
    from paper_2607_18631_b200 import ops
    x, router, ws, sc = layer_inputs(30, 256, 300, 8, 8, 0, "e4m3", seed=5)
    want = ops.MoeLayer(router, *ws, top_k=2, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2]).forward(x)
    ws[0].view(torch.uint8)[3, 200, 17] = 0x7F
    got = ops.MoeLayer(router, *ws, top_k=2, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2]).forward(x)
    hit = (got["ids"] == 3).any(1)
    assert hit.any() and not hit.all()
    assert torch.isnan(got["out"][hit].float()).all() and torch.equal(got["out"][~hit], want["out"][~hit])
    for m in ws:
        m.view(torch.uint8)[:] = 0
    got = ops.MoeLayer(router, *ws, top_k=2, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2]).forward(x)
    assert torch.all(got["out"] == 0)
