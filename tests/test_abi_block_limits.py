"""Sizes that one launch (fewer than 2^32 threads) cannot hold are refused on the host as
unsupported, and the largest ones that it can are not (fake pointers, nothing is launched:
on a host without a GPU an accepted call ends in a HIP error)."""
import ctypes

import pytest
import torch

import paper_2412_09764_amd as pk

UNSUPPORTED, HIP = -2, -4
F32, BF16, E4M3 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("fake device pointers: host-only test")
    return pk.load()


@pytest.mark.parametrize("numel,rc", [((1 << 36) - 4096, HIP), ((1 << 36) - 4095, UNSUPPORTED), (1 << 40, UNSUPPORTED)])
@pytest.mark.parametrize("at", [0, 1])
def test_adamw_elements(lib, numel, rc, at):
    big = pk._AdamwTensor(1 << 44, 1 << 45, 1 << 46, 1 << 47, 1 << 48, 1 << 49, numel, BF16, BF16, E4M3)
    small = pk._AdamwTensor(1 << 20, 1 << 21, 1 << 22, 1 << 23, None, None, 100, F32, F32, F32)
    ts = (pk._AdamwTensor * 2)(*((big, small) if at == 0 else (small, big)))
    o = pk._AdamwOpts(1e-3, 0.9, 0.999, 1e-8, 0.1, 1, 0)
    assert lib.mem_adamw(ctypes.addressof(ts), 2, ctypes.addressof(o), None) == rc
    if rc == UNSUPPORTED:
        assert f"tensor {at}" in lib.mem_last_error().decode()


P = [e << 50 for e in range(1, 8)]  # far apart for the largest of these buffers (4 TiB)


@pytest.mark.parametrize("T,N,K,rc", [
    ((1 << 31) - 256, 256, 8, HIP), ((1 << 31) - 255, 8, 8, UNSUPPORTED), ((1 << 31) - 1, 8, 1 << 20, UNSUPPORTED),
    (1 << 30, 512, 8, UNSUPPORTED), ((1 << 30) - 256, 512, 8, HIP), (1 << 30, 8, 1 << 10, HIP)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_linear_tiles(lib, T, N, K, rc, dt):
    assert lib.mem_linear(P[0], P[1], dt, None, None, None, None, T, N, K, 0, None, P[2], dt, None) == rc
    assert rc != UNSUPPORTED or "tiles" in lib.mem_last_error().decode()


@pytest.mark.parametrize("T,N,K,rc", [
    ((1 << 31) - 256, 8, 256, HIP), ((1 << 31) - 255, 8, 8, UNSUPPORTED), (1 << 30, 8, 512, UNSUPPORTED),
    (64, 1 << 20, 1 << 20, UNSUPPORTED), (64, 1 << 20, 1 << 19, UNSUPPORTED), (64, 1 << 19, (1 << 20) - 256, HIP)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_linear_backward_tiles(lib, T, N, K, rc, dt):
    assert lib.mem_linear_backward(P[0], P[1], P[2], dt, T, N, K, None, P[3], P[4], P[5], P[6], 1 << 45, None) == rc
    assert rc != UNSUPPORTED or "tiles" in lib.mem_last_error().decode()
