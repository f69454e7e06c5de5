"""CPU checks of pf_prefix_attention_status: the refusals of pf_prefix_attention, and a status that no word can be written to."""
from __future__ import annotations

import pytest

import test_position_ops_abi as P
from paper_2607_18631_b200 import binding as B
from test_ops_abi import PTR


class WithStatus:
    """The library, with pf_prefix_attention calls going to the form with a status."""

    def __init__(self, L, status):
        self.L, self.status = L, status

    def pf_prefix_attention(self, *args):
        return self.L.pf_prefix_attention_status(*args[:18], self.status, *args[18:])


@pytest.fixture(scope="module")
def lib():
    from paper_2607_18631_b200 import build as pf_build
    from paper_2607_18631_b200 import ops
    pf_build.build()
    return ops.declare(B.load_library())


def test_status_refusals(lib):
    P.test_prefix_refusals(WithStatus(lib, None))
    for bad in (PTR + 1, PTR + 2):
        assert P.prefix(WithStatus(lib, bad)) == B.PF_EINVAL
    assert P.prefix(WithStatus(lib, PTR), q=None) == B.PF_EINVAL and P.prefix(WithStatus(lib, PTR), n_seq=-1) == B.PF_ERANGE
