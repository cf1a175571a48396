"""The projections' rules for tiles and splits (csrc/pk_linear_plan.h), compiled for the
host and called through ctypes."""
import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2412_09764_amd", "csrc")
TILES = ("256", "128", "128_k2", "64", "32")  # in the order of the header's enum

SHIM = """#include "pk_linear_plan.h"
extern "C" int tile(int f32, long long M, long long N) { return pk::pick_tile(f32, M, N); }
extern "C" void grad(int bf16, long long T, int N, int K, int* tile, int* splits) {
  const pk::GradPlan p = pk::grad_plan(bf16, T, N, K);
  *tile = p.tile;
  *splits = p.splits;
}
"""


class Plan:
    def __init__(self, folder):
        src, lib = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan.so")
        with open(src, "w") as f:
            f.write(SHIM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{CSRC}", src, "-o", lib], check=True)
        self.lib = ctypes.CDLL(lib)
        self.lib.tile.argtypes = [ctypes.c_int, ctypes.c_longlong, ctypes.c_longlong]
        self.lib.grad.argtypes = [ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_int,
                                  ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int)]

    def product(self, dtype, rows, cols):
        """The tile of a product with rows x cols results (the forward's, dx's)."""
        return TILES[self.lib.tile(dtype == "f32", rows, cols)]

    def grad(self, dtype, T, N, K):
        """(tile, splits) of the weight gradient."""
        t, s = ctypes.c_int(), ctypes.c_int()
        self.lib.grad(dtype == "bf16", T, N, K, ctypes.byref(t), ctypes.byref(s))
        return TILES[t.value], s.value
