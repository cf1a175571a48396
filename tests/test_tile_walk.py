"""The sizes of test_gpu_tile_walk.py give workgroups a second tile and more, in both widths of
the tiles of two steps; on the host."""
import ctypes
import os
import shutil
import subprocess

import pytest

from tests.linear_plan import CSRC, TILES
from tests.test_gpu_tile_walk import BLOCKS, GLU

SHIM = """#include "pk_linear_plan.h"
extern "C" int tile(long long M, long long N) { return pk::blocks_plan(false, M, N, 1024).tile; }
extern "C" int glu(long long M, long long N) { return pk::pick_tile(false, M, 2 * N); }
extern "C" int places(int tile) { return pk::step_tile_places(tile); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    folder = str(tmp_path_factory.mktemp("walk"))
    src, lib = os.path.join(folder, "walk.cpp"), os.path.join(folder, "walk.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", lib], check=True)
    so = ctypes.CDLL(lib)
    for fn in (so.tile, so.glu):
        fn.argtypes = [ctypes.c_longlong] * 2
    return so


@pytest.mark.parametrize("name,shapes", [("tile", BLOCKS), ("glu", GLU)])
def test_workgroups_walk(plan, name, shapes):
    most = {}
    for T, N, K in shapes:
        t = getattr(plan, name)(T, N)
        side = {"256": 256, "128": 128}[TILES[t]]
        across = -(-N // (side // 2 if name == "glu" else side))
        turns = -(-T // side) * across / plan.places(t)
        assert turns > 1, (T, N, K)
        most.setdefault(side, []).append(turns)
    assert sorted(most) == [128, 256] and all(len(v) >= 4 and max(v) > 3 for v in most.values())
