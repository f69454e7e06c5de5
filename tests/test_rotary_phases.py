"""CPU checks of pf_rotary_phases for frequencies next to 0 and next to whole turns."""
from __future__ import annotations

import ctypes as C
import math
from fractions import Fraction

import pytest

from paper_2607_18631_b200 import binding as B
from paper_2607_18631_b200 import build as pf_build
from paper_2607_18631_b200 import ops


@pytest.fixture(scope="module")
def lib():
    pf_build.build()
    return ops.declare(B.load_library())


@pytest.mark.parametrize("f", [-1e-18, -3e-19, -1.7e-19, -1e-19, -1e-20, -1e-30, -5e-324, 5e-324, 1e-20, -0.0, -2 * math.pi, math.nextafter(2 * math.pi, 0), math.nextafter(2 * math.pi, 7)])
def test_phases_next_to_a_whole_turn(lib, f):
    """Within two units of 2^-64 turns, modulo a turn; a frequency that is nearer to 0 than half a unit has phase 0."""
    pi = Fraction(3141592653589793238462643383279502884197, 10 ** 39)
    out = (C.c_uint64 * 1)(12345)
    assert lib.pf_rotary_phases(1, (C.c_double * 1)(f), out) == B.PF_OK
    turns = Fraction(f) / (2 * pi)
    off = (Fraction(out[0], 2 ** 64) - turns) % 1
    assert min(off, 1 - off) <= Fraction(2, 2 ** 64)
    if abs(turns) < Fraction(1, 2 ** 65):
        assert out[0] == 0
