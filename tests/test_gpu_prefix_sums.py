"""pf_prefix_attention: the log of a row's sum has 32-bit accuracy, whichever way a token's power of two is computed.

Tolerance.  Scores below are exact and at most 4, so a reference is about -10 and a weight's exponent at most 15.9.  A weight is off by 2^-22 of it (special-function unit or polynomial),
its exponent by half units in the last place of three numbers below 16, 2^-21 each, and the result's logarithm (below 32 in base 2) by 2^-20:
2^-22 + ln 2 (3 x 2^-21 + 2^-20)."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("odd", [0, 1, 2, 3])
@pytest.mark.parametrize("hd", [64, 128])
def test_sums_of_weights_of_all_fractions(hd, odd):
    """A tile in which one token has the largest score and each fourth pair of tokens (all four places in turn) a smaller one; 512 such distances within three binary orders."""
    import torch
    from paper_2607_18631_b200 import ops
    k = torch.zeros(8, 1, 16, hd, device="cuda")
    pairs = torch.arange(16, device="cuda") // 2 % 4
    k[..., 0], first = -448.0, (2 * odd + 2) % 8
    k[:, :, pairs == odd, :2] = 1.0
    k[0, 0, first, :2] = torch.tensor([1.0, 0.0], device="cuda")
    v = torch.ones_like(k)
    cache = [t.to(torch.float8_e4m3fn) for t in (k, v)] + [torch.ones(8, 1, device="cuda") for _ in range(2)]
    n = 512
    q = torch.zeros(n, 1, hd, device="cuda", dtype=torch.float16)
    q[:, 0, 0], q[:, 0, 1] = 4.0, -torch.arange(n, device="cuda") / 240
    d = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    got = ops.pf_prefix_attention(q, *cache, zero, zero[:, None].contiguous(), d(128), d(*range(8))[None], sm_scale=1.0, lse=True)
    want = 4 + torch.log1p(32 * torch.exp(q[:, 0, 1].double()))
    err = (got["lse"][:, 0].double() - want).abs()
    assert torch.all(err <= 2.0 ** -22 + math.log(2) * (3 * 2.0 ** -21 + 2.0 ** -20)), float(err.max())
    assert torch.all((got["out"].float() - 1).abs() <= 2.0 ** -10)      # the weights' and the output's roundings
