"""Outputs that lie over what a norm, projection or optimizer call still reads, or
over each other, are refused on the host (fake pointers, nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2412_09764_amd as pk

INVALID = -1
F32, BF16, E4M3 = 0, 1, 2
A, B, C, D, E = (0x100000 * (1 << i) for i in range(5))  # 1 MiB or more apart


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("fake device pointers: host-only test")
    return pk.load()


def refused(lib, rc, text):
    return rc == INVALID and text in lib.mem_last_error().decode()


@pytest.mark.parametrize("x,res,w,s,y,ydt,bad", [
    (A, None, B, None, A, E4M3, True),   # 8-bit rows over wider ones
    (A, C, B, None, C, E4M3, True),
    (A, C, B, None, B, BF16, True),
    (A, C, B, B, D, BF16, True),
    (A, None, B, None, A, BF16, False),  # in place, row by row
    (A, C, B, None, C, BF16, False),
    (A, C, B, A, D, E4M3, False),        # the stream in place
])
def test_norm(lib, x, res, w, s, y, ydt, bad):
    rc = lib.mem_rmsnorm(x, res, w, BF16, 4, 64, 1e-5, s, y, ydt, E if ydt == E4M3 else None, None)
    assert refused(lib, rc, "may not be weight") if bad else rc != INVALID


def test_quantize_rows(lib):
    assert refused(lib, lib.mem_quantize_rows(A, BF16, 4, 64, A, B, None), "q_out may not be x")


@pytest.mark.parametrize("z,y", [(None, C), (C, D)])
def test_linear_over_bias(lib, z, y):
    assert refused(lib, lib.mem_linear(A, B, BF16, None, None, C, None, 4, 64, 64, 0, z, y, BF16, None), "operand")


@pytest.mark.parametrize("gw", [A, B, C, D, E])
def test_linear_backward_weight_gradient(lib, gw):
    rc = lib.mem_linear_backward(A, B, C, F32, 4, 64, 64, None, D, gw, E, 1 << 30, 1 << 40, None)
    assert refused(lib, rc, "no other buffer")


def tensor(p, m, v, n=1000, pd=F32, sd=F32, sm=None, sv=None):
    return pk._AdamwTensor(p, 1 << 40, m, v, sm, sv, n, pd, F32, sd)


def step(lib, ts):
    o = pk._AdamwOpts(1e-3, 0.9, 0.999, 1e-8, 0.1, 1, 0)
    array = (pk._AdamwTensor * len(ts))(*ts)
    return lib.mem_adamw(ctypes.addressof(array), len(ts), ctypes.addressof(o), None)


FIRST = tensor(A, A + 4000, A + 8000)


@pytest.mark.parametrize("second", [
    tensor(A, B, C),                                       # a parameter listed twice
    tensor(B, A + 4000, C),                                # another one's state
    tensor(B, B, C),                                       # its own state
    tensor(B, C, A + 11996),                               # by one element
    tensor(A - 1996, B, C, pd=BF16),
    tensor(B, C, D, sd=E4M3, sm=E, sv=E + 28),             # 8 scales of 4 bytes each
    tensor(B, C, B + 3996, sd=E4M3, sm=D, sv=E),
])
@pytest.mark.parametrize("more", [0, 40])
def test_adamw_overlap(lib, second, more):
    far = [tensor(*((1 << 30) + (i * 3 + j) * 4096 for j in range(3))) for i in range(more)]
    assert refused(lib, step(lib, [*far, FIRST, tensor(A, A, A, n=0), second]), "overlap")
    assert refused(lib, step(lib, [second, *far, FIRST]), "overlap")


@pytest.mark.parametrize("second", [
    tensor(A + 12000, A + 16000, A + 20000),               # end to end
    tensor(A - 2000, B, C, pd=BF16),
    tensor(B, C, D, sd=E4M3, sm=E, sv=E + 32),
    tensor(B, B + 4000, B + 5000, sd=E4M3, sm=B + 6000, sv=B + 6032),
])
def test_adamw_neighbours(lib, second):
    assert step(lib, [FIRST, second]) != INVALID


def test_adamw_rows_overlap(lib):
    o = pk._AdamwOpts(1e-3, 0.9, 0.999, 1e-8, 0.1, 1, 0)
    t = tensor(A, A + 64 * 64 * 4 - 16, B, n=64 * 64)
    assert refused(lib, lib.mem_adamw_rows(ctypes.addressof(t), 64, 64, C, 5, ctypes.addressof(o), None), "overlap")
