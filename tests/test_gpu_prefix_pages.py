"""pf_prefix_attention where pages of full tiles are not there: whatever lies in shared memory where nothing was copied counts for nothing.

References and tolerances as in test_gpu_prefix_attention."""
from __future__ import annotations

import pytest

from test_gpu_kv_attention import make_cache
from test_gpu_prefix_attention import build, compare, d32, run

pytestmark = pytest.mark.gpu


def patterns(page):
    """Which pages of a tile of 128 tokens are there: every first few, every last few, one missing, one there."""
    n = 128 // page
    some = [[i < j for i in range(n)] for j in range(n + 1)] + [[i >= j for i in range(n)] for j in range(n + 1)]
    some += [[i != j for i in range(n)] for j in range(n)] + [[i == j for i in range(n)] for j in range(n)]
    return some


def leave_nan_behind(hd, page):
    """Calls whose keys and values are NaN throughout, on every SM: what they copy stays in shared memory."""
    import torch
    q, cache, own, table, plen, ptable, cu = build(1, hd, page, [4], [400 * 128], [0] * 4, 1, seed=9)
    for c in cache[:2]:
        c.view(torch.uint8).fill_(0x7F)
    assert torch.isnan(run(q, cache, own, table, plen, ptable, cu)["out"].float()).all()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("B,heads,n_kv", [(3, 4, 2), (40, 4, 1), (70, 8, 2)])
def test_every_pattern_of_missing_pages_in_full_tiles(page, hd, B, heads, n_kv):
    """Each tile has the next pattern.  Few tiles: each is its block's first; the longer prefix gives every block several."""
    for repeat in (1, 6):
        some = patterns(page) * repeat
        args = build(n_kv, hd, page, [B], [128 * len(some)], [11 * i % 50 for i in range(B)], heads, seed=page + B)
        ptable = args[5]
        flat = [there for tile in some for there in tile]
        for i, there in enumerate(flat):
            if not there:
                ptable[0, i] = (-1, 1 << 30)[i % 2]
        leave_nan_behind(hd, page)
        compare(run(*args), *args, hd ** -0.5)


@pytest.mark.parametrize("page", [16, 32, 64])
def test_a_tile_behind_another_groups_nan(page):
    """Groups whose pages are NaN take turns with groups of which pages are missing, several of them to a block: each sees its own tokens only."""
    import torch
    some = patterns(page)
    n = 300
    q, _, own, _, plen, _, cu = build(1, 64, page, [1] * n, [384] * n, [0] * n, 2, seed=page)
    per = 384 // page
    cache = make_cache(2 * per, 1, page, 64, page)
    for c in cache[:2]:
        c.view(torch.uint8)[per:] = 0x7F
    rows = []
    for g in range(n):
        if g % 2 == 0:
            rows.append(list(range(per, 2 * per)))
        else:
            tile = [some[(3 * g + t) % len(some)] for t in range(3)]
            there = [x for t in tile for x in t]
            rows.append([i if there[i] else -1 for i in range(per)])
    ptable, table = d32(rows), d32([[0]] * n)
    got = run(q, cache, own, table, plen, ptable, cu)
    assert torch.isnan(got["out"][::2].float()).all()
    odd = slice(1, None, 2)
    half = {k: v[odd] for k, v in got.items()}
    compare(half, q[odd], cache, own[odd], table[odd], plen[odd], ptable[odd], list(range(n // 2 + 1)), 0.125)
