"""The workspace of pf_prefix_attention: partial results take what the rows need, calls stay inside it, and what it holds does not matter."""
from __future__ import annotations

import pytest

from test_gpu_prefix_attention import build, compare, run

pytestmark = pytest.mark.gpu


def size_of(n_kv, page, hd, n_seq, heads, groups, cols):
    from paper_2607_18631_b200 import ops
    return ops._lib()[0].pf_prefix_attention_workspace(ops.PfKvCache(8, n_kv, page, hd), n_seq, heads, groups, cols)


@pytest.mark.parametrize("n_kv,hd,page,groups,plen,heads", [(1, 64, 16, [1], 100, 1), (2, 128, 64, [127], 1000, 2), (2, 128, 64, [128], 1000, 2), (2, 64, 32, [129], 1000, 2), (1, 64, 16, [1] * 1024, 40, 2),
                                                            (2, 64, 64, [1, 200, 0, 3, 257, 128] * 5, 900, 8), (1, 128, 128, [2] * 300, 5000, 16), (4, 128, 64, [3], 40000, 32)])
def test_calls_stay_inside(n_kv, hd, page, groups, plen, heads):
    import torch
    B = sum(groups)
    args = build(n_kv, hd, page, groups, [max(0, plen - 7 * i) for i in range(len(groups))], [5 * i % 60 for i in range(B)], heads, seed=B)
    size = size_of(n_kv, page, hd, B, heads, len(groups), args[5].shape[1])
    room = torch.full((size + 512,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN, wherever it is read as a number
    got = run(*args, workspace=room[256:256 + size])
    assert torch.all(room[:256] == 0xFF) and torch.all(room[256 + size:] == 0xFF)
    if B * plen < 400_000:
        compare(got, *args, hd ** -0.5)
    want = run(*args)
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])


def test_what_is_asked_for():
    """What pf_decode_attention asks for, three rows of hd + 2 numbers for each row (own tokens, and the prefix up to twice), and for each piece of the list (one an SM, and one for 512 tiles) the
    rows of a tile; not a tile of 256 rows for each group."""
    import torch
    from paper_2607_18631_b200 import ops
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for n_kv, hd, n_seq, heads, groups, cols in ((16, 64, 4, 16, 1, 13), (8, 128, 128, 64, 128, 128), (8, 128, 1024, 64, 1024, 64), (8, 128, 256, 64, 1, 512)):
        one = ops._lib()[0].pf_decode_attention_workspace(ops.PfKvCache(8, n_kv, 64, hd), n_seq, heads)
        tasks, tiles = n_kv * (n_seq * heads // n_kv // 256 + groups), cols // 2 + 1
        tile = min(256, 2 * n_seq * heads // n_kv)
        rows = 3 * n_seq * heads + (tasks * tiles // 512 + sms) * tile
        assert size_of(n_kv, 64, hd, n_seq, heads, groups, cols) <= one + rows * (hd + 2) * 4 + 4096
