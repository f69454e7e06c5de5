"""pf_add_rms_norm against the formula in 64 bits.

Tolerances.  Let u = 2^-24.  The sum of squares is a tree over at most 64 products a thread, then 10 shuffles: relative error
below 80 u; its root halves that, rsqrt and the two products add 4 u: y is within 64 u = 2^-18 before its own rounding.  The stored
types add half a unit: 2^-8 (bf16, 8 significant bits), 2^-11 (fp16; 2^-25 below the normals), u (fp32).  A scale carries y's error and a
division.  e4m3 has 3 mantissa bits: |q s - y| <= 2^-4 |y|, or half of its least step 2^-9 s, and y's own error."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

Y_REL = 2.0 ** -18
HALF = {"bfloat16": (2.0 ** -8, 0.0), "float16": (2.0 ** -11, 2.0 ** -25), "float32": (2.0 ** -24, 0.0)}


def reference(x, res, w, eps, group):
    import torch
    a = x.double() if res is None else x.double() + res.double()
    y = a / torch.sqrt((a * a).mean(1, keepdim=True) + eps)
    if w is not None:
        y = y * w.double()
    step = group or x.shape[1]
    scale = torch.stack([p.abs().amax(1) / 448.0 for p in y.split(step, 1)], 1)
    return a, y, torch.where(scale > 0, scale.clamp(min=2.0 ** -100), torch.ones_like(scale))


def check(out, x, res, w, eps, group, where):
    import torch
    a, y, scale = reference(x, res, w, eps, group)
    rel, least = HALF[str(x.dtype).replace("torch.", "")]
    if "sum" in out:
        assert torch.all((out["sum"].double() - a).abs() <= a.abs() * (rel + 2.0 ** -23) + least), where
    if "y" in out:
        assert torch.all((out["y"].double() - y).abs() <= y.abs() * (rel + Y_REL) + least), where
    if "q" in out:
        assert out["q"].dtype == torch.float8_e4m3fn and out["scale"].shape == scale.shape
        assert torch.all((out["scale"].double() - scale).abs() <= scale * 2 * Y_REL), where
        s = out["scale"].double().repeat_interleave(group or x.shape[1], 1)[:, :x.shape[1]]
        err = (out["q"].double() * s - y).abs()
        assert torch.all(err <= y.abs() * (2.0 ** -4 + 2 * Y_REL) + s * 2.0 ** -10), where


SHAPES = [(1, 1), (3, 7), (2, 8), (5, 100), (4, 127), (3, 128), (2, 129), (7, 1000), (1, 1024), (6, 1032), (149, 2048), (3, 2049), (150, 4096), (2, 5120), (200, 7168),
          (1, 7168), (5, 7175), (149, 8192), (3, 8200), (151, 16384), (2, 16384), (2, 16383)]


@pytest.mark.parametrize("rows,H", SHAPES)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_norm_matches_the_formula(rows, H, dtype):
    import torch
    from paper_2607_18631_b200 import ops
    dt = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(rows * 31 + H)
    x, res = (torch.randn(rows, H, generator=g, device="cuda").mul(s).to(dt) for s in (1.0, 4.0))
    w = (1 + 0.3 * torch.randn(H, generator=g, device="cuda")).to(dt)
    for r, wt, group in ((res, w, 128), (None, w, 0), (res, None, 0), (None, None, 128)):
        out = ops.pf_add_rms_norm(x, r, wt, eps=1e-5, group=group, y=True)
        check(out, x, r, wt, 1e-5, group, (r is not None, wt is not None, group))
        assert ("sum" in out) == (r is not None)
        again = ops.pf_add_rms_norm(x, r, wt, eps=1e-5, group=group, y=True)
        assert all(torch.equal(out[n].view(torch.uint8), again[n].view(torch.uint8)) for n in out)


@pytest.mark.parametrize("H,off", [(7168, 0), (1000, 8), (1000, 1), (130, 3)])
def test_strided_rows_and_in_place_sums(H, off):
    import torch
    from paper_2607_18631_b200 import ops
    big = torch.randn(9, H + 64, device="cuda").to(torch.bfloat16)
    res = torch.randn(9, H + 40, device="cuda").to(torch.bfloat16)
    x, r = big[:, off:off + H], res[:, off:off + H]
    want = ops.pf_add_rms_norm(x.contiguous(), r.contiguous(), group=128, y=True)
    keep_x, keep_r = big.clone(), res.clone()
    got = ops.pf_add_rms_norm(x, r, group=128, y=True, sum_out=r)      # the residual stream, updated in place
    assert got["sum"].data_ptr() == r.data_ptr()
    for n in ("y", "q", "scale"):
        assert torch.equal(got[n].view(torch.uint8), want[n].view(torch.uint8)), n
    assert torch.equal(r, want["sum"]) and torch.equal(big, keep_x)
    keep_r[:, off:off + H] = want["sum"]
    assert torch.equal(res, keep_r)                                    # nothing beside the rows was written
    x2 = keep_x.clone()
    v = x2[:, off:off + H]
    got = ops.pf_add_rms_norm(v, keep_r[:, off:off + H].sub(want["sum"]), group=0, q=True, sum_out=v)   # x itself
    assert torch.equal(got["sum"], x) and torch.equal(v, x)


def test_zero_tiny_and_non_finite_rows():
    import torch
    from paper_2607_18631_b200 import ops
    x = torch.randn(8, 512, device="cuda")
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    x[4] *= 1e-30
    x[5, 128:256] = 0                                                   # one group without anything
    w = torch.ones(512, device="cuda")
    for group in (0, 128):
        out = ops.pf_add_rms_norm(x, None, w, eps=1e-6, group=group, y=True)
        ok = [0, 1, 4, 5, 6, 7]
        check({n: v[ok] for n, v in out.items()}, x[ok], None, w, 1e-6, group, group)
        assert torch.all(out["q"][1].float() == 0) and torch.all(out["scale"][1] == 1)
        if group:
            assert out["scale"][5, 1] == 1 and torch.all(out["q"][5, 128:256].float() == 0)
        assert torch.isnan(out["y"][2]).all() and torch.isnan(out["q"][2].float()).all()
        assert torch.isnan(out["y"][3, 7]) and torch.all(out["y"][3, :7] == 0)


def test_refusals_and_empty_calls():
    import torch
    from paper_2607_18631_b200 import PlanfrontError, ops
    x = torch.randn(4, 64, device="cuda").to(torch.bfloat16)
    out = ops.pf_add_rms_norm(x[:0], y=True)
    assert out["y"].shape == (0, 64) and out["scale"].shape == (0, 1)
    for bad in (lambda: ops.pf_add_rms_norm(x.to(torch.float64)), lambda: ops.pf_add_rms_norm(x, x[:2]), lambda: ops.pf_add_rms_norm(x, x.float()),
                lambda: ops.pf_add_rms_norm(x, None, x[0, :32]), lambda: ops.pf_add_rms_norm(x.t()), lambda: ops.pf_add_rms_norm(x[0]),
                lambda: ops.pf_add_rms_norm(x.cpu()), lambda: ops.pf_add_rms_norm(x, group=32), lambda: ops.pf_add_rms_norm(x, eps=-1.0),
                lambda: ops.pf_add_rms_norm(x, q=False), lambda: ops.pf_add_rms_norm(torch.zeros(2, 16385, device="cuda"))):
        with pytest.raises(PlanfrontError):
            bad()


def test_on_a_stream_of_its_own():
    import torch
    from paper_2607_18631_b200 import ops
    s = torch.cuda.Stream()
    x = torch.randn(300, 4096, device="cuda").to(torch.bfloat16)
    want = ops.pf_add_rms_norm(x, y=True)
    torch.cuda.synchronize()
    got = ops.pf_add_rms_norm(x, y=True, stream=s)
    s.synchronize()
    assert torch.equal(got["y"], want["y"])


def test_overlapping_rows_are_refused():
    """An expanded row has stride 0: taking it for contiguous rows would read past its end."""
    import torch
    from paper_2607_18631_b200 import PlanfrontError, ops
    row, x = torch.randn(1, 256, device="cuda"), torch.randn(6, 256, device="cuda")
    for bad in (lambda: ops.pf_add_rms_norm(row.expand(6, 256)), lambda: ops.pf_add_rms_norm(x, row.expand(6, 256)),
                lambda: ops.pf_add_rms_norm(x, x, sum_out=row.expand(6, 256)), lambda: ops.pf_add_rms_norm(row[0].unfold(0, 128, 16))):
        with pytest.raises(PlanfrontError):
            bad()
