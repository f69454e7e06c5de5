"""pf_moe_forward against the layer in 64 bits.

Tolerances, from the formula.  Let e1 be the relative error of a product's terms and sums: H 2^-23 (fp32 sums), for e4m3 weights 2^-11 more (tokens in
fp16).  With A_g = |x| . |g|, A_u likewise: |dg| <= e1 A_g, |du| <= e1 A_u; |silu'| <= 1.1, so
|dh| <= e1 (1.1 A_g |u| + |silu(g)| A_u) + e2 |h| + e3 max|h|, where e2 is what h keeps for the second product (2^-16 as two bf16 numbers, 2^-11 as fp16) plus its
fp32 evaluation (2^-20), and e3 = 2^-36 fp16's least step against the row's largest.  |dout| <= sum w |d| (|dh| + F 2^-23 |h|) + 2^-18 sum w |y| + half a
unit of bf16.  Weights: logits carry H 2^-23 |x| . |r|."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu


def blocks(w, scale):
    return scale.repeat_interleave(128, 1)[:, :w.shape[1]].repeat_interleave(128, 2)[:, :, :w.shape[2]].double()


def layer_inputs(T, H, F, E, local, shared, wtype, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = local + shared
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, router = rn(T, H).to(torch.bfloat16), rn(E, H).mul(H ** -0.5).to(torch.bfloat16)
    shapes = ((n, F, H), (n, F, H), (n, H, F))
    if wtype == "bf16":
        return x, router, [rn(*s).mul(s[2] ** -0.5).to(torch.bfloat16) for s in shapes], [None] * 3
    ws = [rn(*s).mul(100).clamp(-448, 448).to(torch.float8_e4m3fn) for s in shapes]
    sc = [torch.exp(rn(n, -(-s[1] // 128), -(-s[2] // 128)) * 0.4) / (100 * s[2] ** 0.5) for s in shapes]
    return x, router, ws, sc


def reference(x, xv, router, ws, sc, ids, first, local, shared, wtype):
    """The layer in 64 bits for the experts in `ids`; returns (out, error bound, weights)."""
    import torch
    T, H = x.shape
    F = ws[0].shape[1]
    logits = x.double() @ router.double().T
    chosen = logits.gather(1, ids.long())
    wts = torch.softmax(chosen, 1)
    out, tol = (torch.zeros(T, H, dtype=torch.float64, device=x.device) for _ in range(2))
    e1 = H * 2.0 ** -23 + (2.0 ** -11 if wtype == "e4m3" else 0)
    e2 = (2.0 ** -11 if wtype == "e4m3" else 2.0 ** -16) + 2.0 ** -20
    for e in range(local + shared):
        w = (wts * (ids == first + e)).sum(1) if e < local else torch.ones(T, dtype=torch.float64, device=x.device)
        rows = w.nonzero()[:, 0]
        if not rows.numel():
            continue
        gate, up, down = (m[e:e + 1].double() if s is None else m[e:e + 1].double() * blocks(m[e:e + 1], s[e:e + 1]) for m, s in zip(ws, sc))
        v = xv[rows]
        g, u = v @ gate[0].T, v @ up[0].T
        ag, au = v.abs() @ gate[0].abs().T, v.abs() @ up[0].abs().T
        silu = g * torch.sigmoid(g)
        h = silu * u
        dh = e1 * (1.1 * ag * u.abs() + (silu.abs() + 1.1 * e1 * ag) * au) + e2 * h.abs() + 2.0 ** -36 * h.abs().amax(1, keepdim=True) * (wtype == "e4m3")
        y = h @ down[0].T
        out[rows] += w[rows, None] * y
        tol[rows] += w[rows, None] * ((dh + F * 2.0 ** -23 * h.abs()) @ down[0].abs().T + 2.0 ** -18 * y.abs())
    return out, tol + 2.0 ** -8 * (out.abs() + tol), wts


def run(T, H, F, E, K, local=None, first=0, shared=0, wtype="bf16", xq=True, seed=0, edit=None):
    import torch
    from paper_2607_18631_b200 import ops
    local = E if local is None else local
    x, router, ws, sc = layer_inputs(T, H, F, E, local, shared, wtype, seed)
    if edit:
        edit(x, router)
    layer = ops.MoeLayer(router, *ws, top_k=K, first_expert=first, n_shared=shared, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2])
    xv, args = x.double(), ()
    if wtype == "e4m3" and xq and H % 128 == 0:
        n = ops.pf_add_rms_norm(x, group=128)
        args = (n["q"], n["scale"])
        xv = n["q"].double() * n["scale"].double().repeat_interleave(128, 1)
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    got = layer.forward(x, *args, status=status)
    assert int(status) == 0
    # the choice: any set whose logits are the largest within the logits' error, in falling order
    logits = x.double() @ router.double().T
    dl = H * 2.0 ** -23 * (x.double().abs() @ router.double().abs().T).amax(1)
    ids = got["ids"].long()
    assert ids.min() >= 0 and ids.max() < E and all(len(set(r)) == K for r in ids.tolist())
    chosen = logits.gather(1, ids)
    best = torch.sort(logits, 1, descending=True).values[:, :K]
    assert torch.all((chosen - best).abs() <= 2 * dl[:, None])
    out, tol, wts = reference(x, xv, router, ws, sc, got["ids"], first, local, shared, wtype)
    assert torch.all((got["weights"].double() - wts).abs() <= wts * (4 * dl[:, None] + 2.0 ** -20) + 1e-30)
    err = (got["out"].double() - out).abs()
    assert torch.all(err <= tol + 1e-30), float((err / (tol + 1e-30)).max())
    again = layer.forward(x, *args)
    assert all(torch.equal(again[n], got[n]) for n in got)
    return got, layer, x


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 17, 33, 64, 130])
@pytest.mark.parametrize("wtype", ["bf16", "e4m3"])
def test_token_counts(T, wtype):
    run(T, 512, 200, 16, 4, shared=1, wtype=wtype, seed=T)


@pytest.mark.parametrize("T", [1, 20])
@pytest.mark.parametrize("wtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("H,F", [(16, 1), (64, 8), (80, 7), (128, 129), (144, 100), (1024, 2816), (1040, 176), (2048, 1411)])
def test_widths(T, wtype, H, F):
    run(T, H, F, 8, 2, wtype=wtype, seed=H + F)


@pytest.mark.parametrize("T", [3, 50])
@pytest.mark.parametrize("wtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("E,K,local,first,shared", [(8, 2, 2, 6, 0), (8, 8, 8, 0, 0), (64, 6, 64, 0, 2), (37, 5, 12, 20, 1), (512, 8, 16, 100, 1), (8, 2, 0, 3, 1), (1, 1, 1, 0, 0),
                                                   (40, 14, 40, 0, 2), (256, 8, 1, 255, 0)])
def test_experts(T, wtype, E, K, local, first, shared):
    run(T, 256, 72, E, K, local, first, shared, wtype, seed=E)


@pytest.mark.parametrize("wtype", ["bf16", "e4m3"])
def test_full_width_single_token_and_most_tokens(wtype):
    run(1, 7168, 256, 32, 8, 4, 8, 1, wtype)
    run(512, 256, 40, 16, 8, shared=3, wtype=wtype)
    run(512, 128, 40, 300, 13, 200, 50, 3, wtype)


def test_tokens_in_bf16_with_e4m3_weights():
    run(5, 384, 96, 8, 2, wtype="e4m3", xq=False)
    run(40, 384, 96, 8, 2, wtype="e4m3", xq=False)


@pytest.mark.parametrize("T", [4, 40])
def test_token_without_a_local_expert_is_zero(T):
    import torch

    def edit(x, router):
        router.zero_()
        router[:2] = 1.0                # every token with a positive sum goes to experts 0 and 1, every other elsewhere
        x.copy_(x.abs())
        x[1::2] *= -1
    got, _, _ = run(T, 256, 64, 8, 2, local=2, first=0, edit=edit)
    assert torch.all(got["out"][1::2] == 0) and torch.all(got["out"][0::2].float().abs().sum(1) > 0)


@pytest.mark.parametrize("T", [3, 30])
def test_ties_take_the_lowest_index(T):
    import torch

    def edit(x, router):
        router[:] = router[0]
    got, _, _ = run(T, 128, 32, 24, 5, edit=edit)
    assert torch.equal(got["ids"].cpu(), torch.arange(5, dtype=torch.int32).repeat(T, 1))
    assert torch.all(got["weights"] == torch.full_like(got["weights"], 0.2))


@pytest.mark.parametrize("T", [5, 30])
@pytest.mark.parametrize("wtype", ["bf16", "e4m3"])
def test_a_token_that_is_not_finite_spoils_only_itself(T, wtype):
    import torch
    from paper_2607_18631_b200 import ops
    x, router, ws, sc = layer_inputs(T, 256, 64, 8, 8, 1, wtype)
    layer = ops.MoeLayer(router, *ws, top_k=2, n_shared=1, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2])
    want = layer.forward(x)
    x[2, 3] = float("nan")
    x[4, 9] = float("inf")
    got = layer.forward(x)
    ok = [t for t in range(T) if t not in (2, 4)]
    assert torch.equal(got["out"][ok], want["out"][ok]) and torch.equal(got["ids"][ok], want["ids"][ok])
    assert torch.isnan(got["out"][2]).any() and not torch.isfinite(got["out"][4]).all()
    assert got["ids"].min() >= 0 and got["ids"].max() < 8


@pytest.mark.parametrize("mul", [1e-6, 1e6])
@pytest.mark.parametrize("T", [3, 30])
def test_large_and_small_tokens(mul, T):
    def edit(x, router):
        x.mul_(mul)
        x[1].mul_(1e-3)
    run(T, 256, 64, 8, 2, wtype="e4m3", xq=False, edit=edit)
    run(T, 256, 64, 8, 2, wtype="bf16", edit=edit)


def test_strided_tokens_buffers_streams_and_refusals():
    import torch
    from paper_2607_18631_b200 import PlanfrontError, ops
    x, router, ws, sc = layer_inputs(11, 256, 64, 8, 4, 1, "bf16")
    layer = ops.MoeLayer(router, *ws, top_k=2, first_expert=2, n_shared=1)
    want = layer.forward(x)
    wide = torch.zeros(11, 512, dtype=torch.bfloat16, device="cuda")
    wide[:, 128:384] = x
    out, work = torch.empty_like(x), torch.empty(8 << 20, dtype=torch.uint8, device="cuda").fill_(0xFF)
    got = layer.forward(wide[:, 128:384], out=out, workspace=work)
    assert got["out"].data_ptr() == out.data_ptr() and all(torch.equal(got[n], want[n]) for n in want)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = layer.forward(x, stream=s)
    s.synchronize()
    assert torch.equal(got["out"], want["out"])
    assert layer.forward(x[:0])["out"].shape == (0, 256)
    one = layer.forward(x[3:4])                        # a token's result may differ only in the order of its sums
    assert torch.allclose(one["out"].float(), want["out"][3:4].float(), rtol=2.0 ** -7, atol=1e-3)
    for bad in (lambda: layer.forward(x.float()), lambda: layer.forward(x[:, :128]), lambda: layer.forward(x, workspace=work[:256]), lambda: layer.forward(x, workspace=work[8:]),
                lambda: layer.forward(x.cpu()), lambda: layer.forward(torch.zeros(513, 256, dtype=torch.bfloat16, device="cuda")),
                lambda: layer.forward(x, x.to(torch.float8_e4m3fn), torch.ones(11, 2, device="cuda")), lambda: layer.forward(wide[:, 1:257]),
                lambda: ops.MoeLayer(router, *ws, top_k=2, first_expert=5, n_shared=1), lambda: ops.MoeLayer(router, *ws, top_k=9),
                lambda: ops.MoeLayer(router, ws[0], ws[1], ws[0], top_k=2), lambda: ops.MoeLayer(router.float(), *ws, top_k=2),
                lambda: ops.MoeLayer(router, *ws, top_k=2, gate_scale=torch.ones(5, 1, 2, device="cuda"))):
        with pytest.raises(PlanfrontError):
            bad()


def test_in_a_graph():
    import torch
    from paper_2607_18631_b200 import ops
    x, router, ws, sc = layer_inputs(6, 512, 96, 16, 16, 0, "e4m3")
    layer = ops.MoeLayer(router, *ws, top_k=4, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2])
    layer.forward(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer.forward(x)
    x.copy_(torch.randn_like(x.float()).to(torch.bfloat16))
    graph.replay()
    torch.cuda.synchronize()
    want = layer.forward(x)
    assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("T,E,wtype", [(50, 64, "e4m3"), (50, 64, "bf16"), (7, 16, "bf16"), (7, 16, "e4m3"), (90, 20, "e4m3")])
def test_short_items_give_the_same_bits_call_after_call(T, E, wtype):
    """Experts of one or two stages: the blocks' warps hand their partial sums over as often as they can."""
    import torch
    from paper_2607_18631_b200 import ops
    x, router, ws, sc = layer_inputs(T, 256, 72, E, E, 2, wtype, seed=E)
    layer = ops.MoeLayer(router, *ws, top_k=6, n_shared=2, gate_scale=sc[0], up_scale=sc[1], down_scale=sc[2])
    want = layer.forward(x)
    out, tol, _ = reference(x, x.double(), router, ws, sc, want["ids"], 0, E, 2, wtype)
    assert torch.all((want["out"].double() - out).abs() <= tol + 1e-30)
    for _ in range(100):
        assert torch.equal(layer.forward(x)["out"], want["out"])


def test_overlapping_token_rows_are_refused():
    import torch
    from paper_2607_18631_b200 import PlanfrontError, ops
    x, router, ws, _ = layer_inputs(1, 128, 32, 4, 4, 0, "bf16")
    layer = ops.MoeLayer(router, *ws, top_k=2)
    with pytest.raises(PlanfrontError):
        layer.forward(x.expand(5, 128))
