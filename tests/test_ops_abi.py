"""CPU checks of the decode-layer operators' C ABI: exports, and refusals that never reach a device."""
from __future__ import annotations

import ctypes as C
import os
import re

import pytest

from paper_2607_18631_b200 import binding as B
from paper_2607_18631_b200 import build as pf_build
from paper_2607_18631_b200 import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 1 << 20          # a 256-byte aligned address that no refused call looks at


@pytest.fixture(scope="module")
def lib():
    pf_build.build()
    return ops.declare(B.load_library())


def test_library_exports_every_declared_operator(lib):
    text = open(os.path.join(ROOT, "include", "planfront_ops.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(pf_[a-z0-9_]+)\s*\(", text))
    assert names == set(ops.EXPORTS)
    assert all(hasattr(lib, n) for n in names)
    assert not names & set(B.EXPORTS)


def norm(lib, dtype=0, rows=4, H=64, x=PTR, xs=64, res=None, rs=64, w=None, eps=1e-6, group=128, s=None, ss=64, y=PTR, ys=64, q=None, scale=None):
    return lib.pf_add_rms_norm(dtype, rows, H, x, xs, res, rs, w, eps, group, s, ss, y, ys, q, scale, None)


def test_norm_refusals(lib):
    assert norm(lib, rows=0) == B.PF_OK
    for bad in (dict(dtype=3), dict(dtype=-1), dict(group=64), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(y=None),
                dict(xs=63), dict(ys=63), dict(res=PTR, rs=10), dict(s=PTR, ss=1), dict(q=PTR), dict(x=PTR + 1), dict(w=PTR + 1)):
        assert norm(lib, **bad) == B.PF_EINVAL, bad
    for bad in (dict(H=0), dict(H=16385, xs=16385, ys=16385), dict(rows=-1), dict(rows=1 << 31)):
        assert norm(lib, **bad) == B.PF_ERANGE, bad


def cache(**kw):
    f = dict(n_pages=8, n_kv=2, page=64, hd=128, d_k=PTR, d_v=PTR, d_k_scale=PTR, d_v_scale=PTR)
    f.update(kw)
    return ops.PfKvCache(**f)


BAD_CACHES = [dict(n_pages=0), dict(n_kv=0), dict(page=24), dict(page=256), dict(hd=96), dict(hd=256), dict(d_k=None), dict(d_v=None), dict(d_k_scale=None),
              dict(d_v_scale=None), dict(d_k=PTR + 8), dict(d_v=PTR + 1), dict(d_k_scale=PTR + 2)]


def append(lib, c=None, dtype=0, n_seq=2, n_new=3, max_new=2, k=PTR, ks=256, v=PTR, vs=256, cu=PTR, ln=PTR, table=PTR, cols=4):
    return lib.pf_kv_append(c if c is not None else cache(), dtype, n_seq, n_new, max_new, k, ks, v, vs, cu, ln, table, cols, None)


def test_append_refusals(lib):
    for none in (dict(n_seq=0), dict(n_new=0), dict(max_new=0), dict(cols=0)):
        assert append(lib, **none) == B.PF_OK
    assert lib.pf_kv_append(None, 0, 1, 1, 1, PTR, 256, PTR, 256, PTR, PTR, PTR, 1, None) == B.PF_EINVAL
    for bad in BAD_CACHES:
        assert append(lib, cache(**bad)) == B.PF_EINVAL, bad
    for bad in (dict(dtype=2), dict(k=None), dict(v=None), dict(cu=None), dict(ln=None), dict(table=None), dict(k=PTR + 2), dict(v=PTR + 8), dict(ks=255), dict(ks=260),
                dict(vs=128), dict(cu=PTR + 1)):
        assert append(lib, **bad) == B.PF_EINVAL, bad
    for bad in (dict(n_seq=-1), dict(n_new=-1), dict(max_new=-1), dict(cols=-1), dict(n_seq=1 << 30, n_new=1 << 30, max_new=1 << 30, cols=1 << 20)):
        assert append(lib, **bad) == B.PF_ERANGE, bad


def attention(lib, c=None, dtype=0, n_seq=2, heads=8, q=PTR, qs=1024, ln=PTR, table=PTR, cols=4, sm=0.1, out=PTR, os_=1024, lse=None, ws=PTR, wb=1 << 40):
    return lib.pf_decode_attention(c if c is not None else cache(), dtype, n_seq, heads, q, qs, ln, table, cols, sm, out, os_, lse, ws, wb, None)


def test_attention_refusals(lib):
    assert attention(lib, n_seq=0) == B.PF_OK and attention(lib, heads=0) == B.PF_OK
    for bad in BAD_CACHES:
        assert attention(lib, cache(**bad)) == B.PF_EINVAL, bad
    for bad in (dict(dtype=2), dict(heads=7), dict(sm=float("nan")), dict(sm=float("inf")), dict(q=None), dict(out=None), dict(ln=None), dict(table=None), dict(q=PTR + 2),
                dict(out=PTR + 8), dict(qs=1000), dict(qs=1028), dict(os_=512), dict(lse=PTR + 1)):
        assert attention(lib, **bad) == B.PF_EINVAL, bad
    for bad in (dict(n_seq=-1), dict(n_seq=8193), dict(heads=-8), dict(cols=-1), dict(cols=1 << 26)):
        assert attention(lib, **bad) == B.PF_ERANGE, bad


def test_attention_refuses_tables_whose_tiles_pass_32_bits(lib):
    """The kernels add up tiles of 32 tokens over all sequences as 32-bit numbers: 2^31 of them and more are refused."""
    for n_seq, page, cols in ((8192, 64, 1 << 17), (8192, 16, 1 << 19), (4096, 128, 1 << 17), (33, 64, (1 << 25) - 1), (64, 16, 1 << 26), (64, 128, (1 << 24) - 1)):
        assert attention(lib, cache(page=page), n_seq=n_seq, cols=cols) == B.PF_ERANGE, (n_seq, page, cols)


def moe(**kw):
    f = dict(H=64, F=24, n_experts=8, first=2, n_local=4, n_shared=1, top_k=2, wtype=0)
    f.update(kw)
    return ops.PfMoe(**f)


BAD_MOES = [dict(H=0), dict(H=24), dict(F=0), dict(n_experts=0), dict(n_experts=513), dict(first=-1), dict(first=5), dict(n_local=-1), dict(n_local=9), dict(n_shared=-1),
            dict(top_k=0), dict(top_k=9), dict(n_experts=64, top_k=16), dict(n_local=0, n_shared=0), dict(wtype=1), dict(wtype=2)]


def forward(lib, m=None, T=3, x=PTR, xs=64, xq=None, xsc=None, router=PTR, packed=PTR, out=PTR, ids=PTR, w=PTR, st=None, ws=PTR, wb=1 << 40):
    return lib.pf_moe_forward(m if m is not None else moe(), T, x, xs, xq, xsc, router, packed, out, ids, w, st, ws, wb, None)


def test_moe_refusals(lib):
    assert forward(lib, T=0) == B.PF_OK
    assert lib.pf_moe_forward(None, 1, *([PTR, 64] + [PTR] * 8 + [PTR, 1 << 40, None])) == B.PF_EINVAL
    for bad in BAD_MOES:
        assert forward(lib, moe(**bad)) == B.PF_EINVAL, bad
        assert lib.pf_moe_packed_bytes(moe(**bad)) == 0
        assert lib.pf_moe_pack(moe(**bad), PTR, PTR, PTR, None, None, None, PTR, None) == B.PF_EINVAL
    for bad in (dict(x=None), dict(router=None), dict(packed=None), dict(out=None), dict(ids=None), dict(w=None), dict(x=PTR + 2), dict(xs=63), dict(xs=68), dict(packed=PTR + 16),
                dict(router=PTR + 2), dict(out=PTR + 2), dict(xq=PTR, xsc=PTR), dict(xq=PTR), dict(xsc=PTR), dict(st=PTR + 1)):
        assert forward(lib, **bad) == B.PF_EINVAL, bad
    m8 = moe(wtype=3)
    assert forward(lib, m8, xq=PTR) == B.PF_EINVAL and forward(lib, m8, xsc=PTR) == B.PF_EINVAL
    for scales in ((None, PTR, PTR), (PTR, None, PTR), (PTR, PTR, None), (PTR + 1, PTR, PTR)):
        assert lib.pf_moe_pack(m8, PTR, PTR, PTR, *scales, PTR, None) == B.PF_EINVAL
    assert forward(lib, T=-1) == B.PF_ERANGE and forward(lib, T=513) == B.PF_ERANGE
    for args in ((None, PTR, PTR, PTR), (PTR, None, PTR, PTR), (PTR, PTR, None, PTR), (PTR, PTR, PTR, None), (PTR + 1, PTR, PTR, PTR), (PTR, PTR, PTR, PTR + 16)):
        assert lib.pf_moe_pack(moe(), *args[:3], None, None, None, args[3], None) == B.PF_EINVAL
    assert lib.pf_moe_pack(moe(), PTR, PTR, PTR, PTR, PTR, PTR, PTR, None) == B.PF_EINVAL


def test_packed_sizes(lib):
    # 3 matrices of every expert, rows to tiles of 8 (gate and up) and 16, columns to slices of 128 bytes
    m = moe(H=64, F=24, n_local=4, n_shared=1)
    assert lib.pf_moe_packed_bytes(m) == 5 * 2048 * (3 * 1 + 4 * 1)
    m = moe(H=7168, F=2048, n_experts=256, first=32, n_local=32, n_shared=1, top_k=8, wtype=3)
    assert lib.pf_moe_packed_bytes(m) == 33 * (3 * 7168 * 2048 + 4 * (3 * 56 * 16 + 2))
    m = moe(H=4096, F=1408, n_experts=64, first=0, n_local=64, n_shared=2, top_k=6, wtype=0)
    assert lib.pf_moe_packed_bytes(m) == 66 * 3 * 4096 * 1408 * 2


def test_operators_fail_loudly_without_a_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    with pytest.raises(B.PlanfrontError):
        ops.pf_add_rms_norm(x)
    with pytest.raises(B.PlanfrontError):
        ops.MoeLayer(x, x, x, x, top_k=1)


def test_struct_layouts_match_the_header():
    assert C.sizeof(ops.PfKvCache) == 4 * 4 + 4 * 8 and ops.PfKvCache.d_k.offset == 16
    assert C.sizeof(ops.PfMoe) == 8 * 4 and ops.PfMoe.wtype.offset == 28
