"""pf_decode_attention and pf_kv_append: calls at the edge of what they take."""
from __future__ import annotations

import math

import pytest

from test_gpu_kv_attention import make_cache

pytestmark = pytest.mark.gpu


def test_a_table_without_columns_gives_empty_rows():
    """Sequences that have no page yet: all rows are empty, whatever their lengths say."""
    import torch
    from paper_2607_18631_b200 import ops
    cache = make_cache(4, 2, 16, 64)
    q = torch.randn(3, 4, 64, device="cuda").to(torch.bfloat16)
    none = torch.zeros(3, 0, dtype=torch.int32, device="cuda")
    got = ops.pf_decode_attention(q, *cache, torch.tensor([0, 5, -1], dtype=torch.int32, device="cuda"), none, lse=True)
    assert torch.all(got["out"] == 0) and torch.all(got["lse"] == -math.inf)
