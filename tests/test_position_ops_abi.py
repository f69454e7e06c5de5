"""CPU checks of the rotary and shared-prefix operators' C ABI: refusals that never reach a device, and the frequencies."""
from __future__ import annotations

import ctypes as C
import math
from fractions import Fraction

import pytest

from paper_2607_18631_b200 import binding as B
from paper_2607_18631_b200 import build as pf_build
from paper_2607_18631_b200 import ops
from test_ops_abi import BAD_CACHES, PTR, cache


@pytest.fixture(scope="module")
def lib():
    pf_build.build()
    return ops.declare(B.load_library())


def rotary(**kw):
    f = dict(rot=64, layout=0, amplitude=1.0, d_phase=PTR)
    f.update(kw)
    return ops.PfRotary(**f)


BAD_ROTARIES = [dict(rot=-2), dict(rot=63), dict(rot=130), dict(layout=2), dict(layout=-1), dict(amplitude=float("nan")), dict(amplitude=float("inf")), dict(d_phase=None),
                dict(d_phase=PTR + 4)]


def rope(lib, r=None, tr=0, dtype=0, tokens=3, heads=4, hd=128, x=PTR, xt=512, xh=128, pos=PTR, y=PTR, yt=512, yh=128):
    return lib.pf_rope(r if r is not None else rotary(), tr, dtype, tokens, heads, hd, x, xt, xh, pos, y, yt, yh, None)


def test_rope_refusals(lib):
    assert rope(lib, tokens=0) == B.PF_OK and rope(lib, heads=0) == B.PF_OK
    assert lib.pf_rope(None, 0, 0, 1, 1, 64, PTR, 64, 64, PTR, PTR, 64, 64, None) == B.PF_EINVAL
    for bad in BAD_ROTARIES:
        assert rope(lib, rotary(**bad)) == B.PF_EINVAL, bad
    for bad in (dict(dtype=3), dict(dtype=-1), dict(x=None), dict(y=None), dict(pos=None), dict(x=PTR + 1), dict(y=PTR + 1), dict(pos=PTR + 2), dict(dtype=2, x=PTR + 2), dict(xt=511),
                dict(xh=127), dict(yt=0), dict(yh=0), dict(xt=128, xh=128), dict(yt=128, yh=383), dict(yt=-512)):
        assert rope(lib, **bad) == B.PF_EINVAL, bad
    for bad in (dict(tokens=-1), dict(tokens=1 << 31), dict(heads=-1), dict(heads=65536), dict(hd=0), dict(hd=1025)):
        assert rope(lib, **bad) == B.PF_ERANGE, bad


def append(lib, c=None, r=None, dtype=0, n_seq=2, n_new=3, max_new=2, heads=4, q=PTR, qs=512, qo=PTR, qos=512, k=PTR, ks=256, v=PTR, vs=256, cu=PTR, ln=PTR, table=PTR, cols=4, pos=None):
    return lib.pf_kv_append_rope(c if c is not None else cache(), r if r is not None else rotary(), dtype, n_seq, n_new, max_new, heads, q, qs, qo, qos, k, ks, v, vs, cu, ln, table,
                                 cols, pos, None)


def test_append_refusals(lib):
    for none in (dict(n_seq=0), dict(n_new=0), dict(max_new=0), dict(heads=0, cols=0)):
        assert append(lib, **none) == B.PF_OK
    for bad in BAD_CACHES:
        assert append(lib, cache(**bad)) == B.PF_EINVAL, bad
    for bad in BAD_ROTARIES + [dict(rot=8), dict(rot=34)]:
        assert append(lib, r=rotary(**bad)) == B.PF_EINVAL, bad
    for bad in (dict(dtype=2), dict(k=None), dict(v=None), dict(cu=None), dict(ln=None), dict(table=None), dict(k=PTR + 2), dict(v=PTR + 8), dict(ks=255), dict(ks=260),
                dict(vs=128), dict(cu=PTR + 1), dict(pos=PTR + 2), dict(q=None), dict(qo=None), dict(q=PTR + 2), dict(qo=PTR + 8), dict(qs=511), dict(qos=516)):
        assert append(lib, **bad) == B.PF_EINVAL, bad
    for bad in (dict(n_seq=-1), dict(n_new=-1), dict(max_new=-1), dict(cols=-1), dict(heads=-1), dict(heads=65536), dict(n_new=1 << 31),
                dict(n_seq=1 << 30, n_new=1 << 30, max_new=1 << 30, cols=1 << 20)):
        assert append(lib, **bad) == B.PF_ERANGE, bad


def prefix(lib, c=None, dtype=0, n_seq=2, heads=8, q=PTR, qs=1024, ln=PTR, table=PTR, cols=4, groups=1, cu=PTR, pl=PTR, pt=PTR, pcols=8, sm=0.1, out=PTR, os_=1024, lse=None, ws=PTR,
           wb=1 << 50):
    return lib.pf_prefix_attention(c if c is not None else cache(), dtype, n_seq, heads, q, qs, ln, table, cols, groups, cu, pl, pt, pcols, sm, out, os_, lse, ws, wb, None)


def test_prefix_refusals(lib):
    assert prefix(lib, n_seq=0) == B.PF_OK and prefix(lib, heads=0) == B.PF_OK
    for bad in BAD_CACHES:
        assert prefix(lib, cache(**bad)) == B.PF_EINVAL, bad
    for bad in (dict(dtype=2), dict(heads=7), dict(sm=float("nan")), dict(sm=float("inf")), dict(q=None), dict(out=None), dict(ln=None), dict(table=None), dict(q=PTR + 2),
                dict(out=PTR + 8), dict(qs=1000), dict(qs=1028), dict(os_=512), dict(lse=PTR + 1), dict(groups=2, cu=None), dict(pl=None), dict(pt=None), dict(cu=PTR + 2),
                dict(pl=PTR + 1), dict(pt=PTR + 3)):
        assert prefix(lib, **bad) == B.PF_EINVAL, bad
    for bad in (dict(n_seq=-1), dict(n_seq=8193), dict(heads=-8), dict(cols=-1), dict(cols=1 << 26), dict(groups=-1), dict(groups=1025), dict(pcols=-1), dict(pcols=1 << 26), dict(pcols=(1 << 25) - 63),
                dict(n_seq=8192, cols=1 << 17), dict(n_seq=8192, heads=1 << 20, qs=1 << 27, os_=1 << 27)):
        assert prefix(lib, **bad) == B.PF_ERANGE, bad


def test_phases_are_the_fractions_of_a_turn(lib):
    pi = Fraction(3141592653589793238462643383279502884197, 10 ** 39)
    freq = ops.rotary_frequencies(128) + [0.0, -0.25, 7.5, 2 * math.pi, 100.0, -1e-12]
    out = (C.c_uint64 * len(freq))()
    assert lib.pf_rotary_phases(len(freq), (C.c_double * len(freq))(*freq), out) == B.PF_OK
    for f, p in zip(freq, out):
        turns = Fraction(f) / (2 * pi)
        off = (Fraction(p, 2 ** 64) - turns) % 1
        assert min(off, 1 - off) <= Fraction(max(1, abs(int(turns)) + 1) * 2, 2 ** 64), f      # a 64-bit quotient, rounded twice
    assert lib.pf_rotary_phases(0, None, None) == B.PF_OK and lib.pf_rotary_phases(-1, None, None) == B.PF_ERANGE and lib.pf_rotary_phases(1, None, out) == B.PF_EINVAL
    assert lib.pf_rotary_phases(1, (C.c_double * 1)(float("inf")), out) == B.PF_EINVAL


def test_frequencies():
    f = ops.rotary_frequencies(8, base=16.0)
    assert f == [1.0, 16.0 ** -0.25, 0.25, 16.0 ** -0.75]
    assert ops.rotary_frequencies(8, base=16.0, scaling="linear", factor=4.0) == [x / 4 for x in f]
    # the new base stretches the slowest pair by the factor and leaves the fastest
    g = ops.rotary_frequencies(8, base=16.0, scaling="base", factor=4.0)
    assert g[0] == 1.0 and math.isclose(g[3], f[3] / 4)
    # 100 positions: 15.9, 8.0, 4.0 and 2.0 turns; from 10 turns on kept, up to 3 divided, in between mixed
    h = ops.rotary_frequencies(8, base=16.0, scaling="parts", factor=4.0, original=100, low=3.0, high=10.0)
    r = [100 * x / (2 * math.pi) for x in f]
    assert h[0] == f[0] and h[3] == f[3] / 4 and all(math.isclose(h[i], f[i] * ((r[i] - 3) / 7 + (10 - r[i]) / 7 / 4)) for i in (1, 2))
    assert ops.rotary_frequencies(0) == [] and ops.rotary_frequencies(2, scaling="base", factor=2.0) == [1.0]
    for bad in (dict(rot=3), dict(rot=-2), dict(rot=8, base=0.0), dict(rot=8, base=float("nan")), dict(rot=8, factor=0.0), dict(rot=8, scaling="other"),
                dict(rot=8, scaling="parts", low=4.0, high=4.0)):
        with pytest.raises(B.PlanfrontError):
            ops.rotary_frequencies(**bad)


def test_struct_layout_matches_the_header():
    assert C.sizeof(ops.PfRotary) == 24 and ops.PfRotary.d_phase.offset == 16
