"""pf_prefix_attention with value scales up to the append's largest, and tokens that hold nearly all the weight.

Scales: references and tolerances as in test_gpu_prefix_attention.  A token that is not there has weight 0 whatever the others' scales."""
from __future__ import annotations

import pytest

from test_gpu_prefix_attention import build, compare, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e", [-60, 70, 80, 100, 118])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("length", [8, 100, 1000, 3001])
def test_large_value_scales(e, page, length):
    """Ragged ends, and pages that are not there."""
    for holes in (False, True):
        args = build(2, 64, page, [5, 30], [length, length + 37], [3 * i for i in range(35)], 10, seed=e + length)
        args[1][3].fill_(2.0 ** e)
        if holes:
            args[5][:, ::3] = -1
        compare(run(*args), *args, 0.125)


def test_value_scales_of_all_sizes_in_one_prefix():
    import torch
    args = build(1, 128, 16, [12, 140], [900, 2000], [20] * 152, 3, seed=5)
    vs = args[1][3]
    vs.copy_(torch.exp2(torch.randint(60, 119, vs.shape, device="cuda").float()))
    args[5][:, 5::7] = -1
    compare(run(*args), *args, 128 ** -0.5)
