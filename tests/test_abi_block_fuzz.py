"""Random argument tuples through the norm, projection and optimizer calls on a
host without a GPU: every call returns one of the documented status codes and
never crashes (fake pointers, never dereferenced on the host)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk

CODES = {0, -1, -2, -3, -4}


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("fake device pointers: host-only test")
    return pk.load()


def _ptr(rng):
    return int(rng.choice([0, 0x10000, 0x10000, 0x10000, 0x10008, 0x10004, 0x10001]))


def _size(rng):
    return int(rng.choice([-8, 0, 1, 7, 8, 16, 64, 128, 200, 1024, 4096, 16384, 16392, 1 << 20, (1 << 20) + 8, (1 << 31) - 8]))


@pytest.mark.parametrize("seed", range(4))
def test_random_calls(lib, seed):
    rng = np.random.default_rng(seed)
    p, n = lambda: _ptr(rng), lambda: _size(rng)  # noqa: E731
    dt = lambda: int(rng.choice([0, 1, 1, 2, 7]))  # noqa: E731
    ws = lambda: int(rng.choice([0, 1000, 1 << 40]))  # noqa: E731
    eps = lambda: float(rng.choice([0.0, 1e-5, -1.0, np.nan, np.inf]))  # noqa: E731
    rows = lambda: int(rng.choice([-1, 0, 1, 333, 1 << 20, (1 << 31) - 1, 1 << 31, 1 << 40]))  # noqa: E731
    for _ in range(500):
        assert lib.mem_rmsnorm(p(), p(), p(), dt(), rows(), n(), eps(), p(), p(), dt(), p(), None) in CODES
        assert lib.mem_rmsnorm_backward(p(), p(), p(), dt(), rows(), n(), eps(), p(), p(), p(), p(), ws(), None) in CODES
        assert lib.mem_quantize_rows(p(), dt(), rows(), n(), p(), p(), None) in CODES
        assert lib.mem_linear(p(), p(), dt(), p(), p(), p(), p(), rows(), n(), n(), int(rng.integers(-1, 5)), p(), p(), dt(), None) in CODES
        assert lib.mem_act_backward(p(), p(), dt(), int(rng.integers(-1, 5)), rows(), n(), p(), None) in CODES
        assert lib.mem_linear_backward(p(), p(), p(), dt(), rows(), n(), n(), p(), p(), p(), p(), p(), ws(), None) in CODES
        t = pk._AdamwTensor(p(), p(), p(), p(), p(), p(), int(rng.choice([-1, 0, 5, 8192, 1 << 30, 1 << 41])), dt(), dt(), dt())
        o = pk._AdamwOpts(eps(), 0.9, float(rng.choice([0.999, 1.0])), 1e-8, eps(), int(rng.integers(-1, 3)), 5, p(), p(), p())
        assert lib.mem_adamw(ctypes.addressof(t), int(rng.integers(-1, 2)), ctypes.addressof(o), None) in CODES
        assert lib.mem_adamw_rows(ctypes.addressof(t), n(), n(), p(), rows(), ctypes.addressof(o), None) in CODES


def test_workspace_sizes_of_any_shape(lib):
    for T in (-1, 0, 1, 777, 1 << 20, (1 << 31) - 1):
        for N in (-8, 0, 8, 1032, 1 << 20):
            assert lib.mem_rmsnorm_backward_workspace_size(T, N) >= 0
            for K in (-8, 8, 1 << 20):
                for dt in (0, 1, 2, 9):
                    assert lib.mem_linear_backward_workspace_size(T, N, K, dt) >= 0
