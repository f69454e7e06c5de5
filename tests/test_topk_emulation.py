"""The block top-k that reduces long key lists, run on the host under arbitrary warp orders.

A list of more than 16,384 keys (the unconstrained large space's search leaves some 30,000, the constrained one's fits the
short path) is walked tile by tile, and a block prunes its buffer when a tile would overflow it.  All warps have to take that
decision alike whatever the order in which they get to it."""
from __future__ import annotations

import ctypes as C
import os
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2607_18631_b200", "csrc")


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("topk") / "topk.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wno-unknown-pragmas", "-I" + CSRC, "-shared", "-fPIC", "-o", lib, os.path.join(HERE, "topk_emulation.cpp")],
                   check=True)
    fn = C.CDLL(lib).topk_walk
    fn.restype = C.c_int
    fn.argtypes = [C.c_void_p, C.c_uint, C.c_int, C.c_uint, C.c_void_p]

    def run(keys, k, seed):
        out = np.zeros(2048, dtype=np.uint64)
        n = fn(keys.ctypes.data, len(keys), k, seed, out.ctypes.data)
        return n, out[:max(0, n)]
    return run


# a segment as pass 1 cuts it from 30,000 to 45,000 keys at k = 1024 (16 blocks), short ones, and ones of many tiles
@pytest.mark.parametrize("n,k", [(1, 1), (31, 5), (1024, 1024), (1025, 16), (1880, 1024), (2048, 1024), (2049, 1024), (2820, 1024), (3073, 1000), (6000, 100)])
def test_any_warp_order_gives_the_k_best(walk, n, k):
    rng = np.random.default_rng(n * 7 + k)
    for seed in range(4):
        keys = rng.permutation(np.arange(1, n + 1, dtype=np.uint64) * np.uint64(2654435761))
        if seed == 1:
            keys = np.sort(keys)           # every tile's keys beat the ones before
        got, best = walk(np.ascontiguousarray(keys), k, seed)
        assert got == min(n, k), {-1: "warps of the block wait at different barriers", -2: "a collective that not all threads reach"}.get(got, got)
        np.testing.assert_array_equal(best, np.sort(keys)[::-1][:k])
