"""Which kernels the gated part and the products in blocks choose, on the host: the sizes that
the GPU tests run reach each of them."""
import ctypes
import os
import shutil
import subprocess

import pytest

from tests.linear_plan import CSRC, TILES, Plan
from tests.test_gpu_blocks import SHAPES as BLOCKS
from tests.test_gpu_glu import SHAPES as GLU

SHIM = """#include "pk_linear_plan.h"
extern "C" void blocks(int exact, long long M, long long N, long long K, int* tile, int* splits, long long* k_split) {
  const pk::BlocksPlan p = pk::blocks_plan(exact, M, N, K);
  *tile = p.tile;
  *splits = p.splits;
  *k_split = p.k_split;
}
"""


@pytest.fixture(scope="module")
def folder(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    return str(tmp_path_factory.mktemp("plan"))


@pytest.fixture(scope="module")
def blocks_plan(folder):
    src, lib = os.path.join(folder, "blocks.cpp"), os.path.join(folder, "blocks.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", lib], check=True)
    fn = ctypes.CDLL(lib).blocks
    fn.argtypes = [ctypes.c_int] + [ctypes.c_longlong] * 3 + [ctypes.c_void_p] * 3

    def plan(exact, M, N, K):
        t, s, k = ctypes.c_int(), ctypes.c_int(), ctypes.c_longlong()
        fn(exact, M, N, K, ctypes.byref(t), ctypes.byref(s), ctypes.byref(k))
        return TILES[t.value], s.value, k.value
    return plan


def test_glu_tiles(folder):
    plan = Plan(folder)
    for dt in ("f32", "bf16", "e4m3"):
        reached = {"few rows" if T <= 8 else plan.product(dt, T, 2 * N) for T, N, K in GLU}
        assert reached == {"few rows", *TILES}, dt


def test_blocks_tiles(blocks_plan):
    exact = {("few rows", False) if T <= 8 else (p[0], p[1] > 1) for T, N, K in BLOCKS for p in [blocks_plan(1, T, N, K)]}
    assert exact == {("few rows", False), ("128_k2", False), ("64", False), ("32", False), ("128_k2", True)}
    assert {blocks_plan(0, T, N, K)[0] for T, N, K in BLOCKS if T > 8} == set(TILES)


def test_blocks_splits(blocks_plan):
    """Parts are whole numbers of 256 k (two groups of waves with whole blocks of scales each),
    none is empty, their tiles fit the chip at once, and results in bf16 are never split."""
    for T in (9, 64, 100, 500, 1000, 2048, 5000):
        for N in (8, 256, 1000, 1024, 4096):
            for K in (16, 1024, 2032, 2048, 5008, 8192, 16400, 65536, 1 << 20):
                tile, splits, k = blocks_plan(1, T, N, K)
                assert blocks_plan(0, T, N, K)[1:] == (1, K)
                if splits > 1:
                    assert tile == "128_k2" and k % 256 == 0 and (splits - 1) * k < K <= splits * k
                    assert splits * -(-T // 128) * -(-N // 128) <= 256
                else:
                    assert k == K and tile not in ("256", "128")
