"""GELU and its derivative far below zero, where 1 + erf(z / sqrt 2) has no digits left:
relative to the value itself, against erfc in 64 bits.

u = 2^-24.  fp32: the argument |z| / sqrt 2 is off by 1.5 u (a product and its constant),
which moves erfc(a) by 2 a^2 = z^2 times that at most; the tail's own polynomial, reciprocal
and exponential are within 34 u, two products 2 u.  The derivative's second term has z^2 / 2 as the argument of an exponential
(2 u of it) and 8 u more.  Where bf16 is stored the functions are within 2^-12 of themselves,
the rounding adds half a step, 2^-8.  Results below 2^-118 may be 0."""
import math

import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -118
tail = np.vectorize(lambda z: 0.5 * math.erfc(-z / math.sqrt(2)), otypes=[float])  # Phi(z)


def points(dt):
    """Every 1/64 (in bf16 what is left of that) from -14 to 6."""
    z = (torch.arange(-14 * 64, 6 * 64 + 1).float() / 64).to(dt).unique()
    return torch.cat([z, z.new_zeros(-len(z) % 8)])


@pytest.mark.parametrize("dt,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32),
                                    (torch.bfloat16, torch.bfloat16)], ids=["f32", "bf16-f32", "bf16"])
@pytest.mark.parametrize("rows", [4, 40])  # both kernels' epilogues
def test_forward(gpu_lib, dt, out, rows):
    z = points(dt)
    w = torch.zeros((len(z), 8), dtype=dt)
    w[:, 0] = z
    x = torch.zeros((rows, 8), dtype=dt)
    x[:, 0] = 1
    y, got_z = pk.mem_linear(x.cuda(), w.cuda(), act="gelu", out_dtype=out, want_z=True)
    z = z.double().numpy()
    assert torch.equal(got_z[0].cpu().double(), torch.from_numpy(z))
    want = z * tail(z)
    rel = (1.5 * z * z + 36) * U if out == torch.float32 else 2.0 ** -12 + 2.0 ** -8
    for row in (y[0], y[-1]):
        assert np.all(np.abs(row.cpu().double().numpy() - want) <= rel * np.abs(want) + TINY)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_backward(gpu_lib, dt):
    z = points(dt).view(-1, 8)
    d = pk.mem_act_backward(torch.ones_like(z).cuda(), z.cuda(), "gelu").cpu().double().numpy()
    z = z.double().numpy()
    p, f = tail(z), np.abs(z) * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    want = p + np.sign(z) * f
    if dt == torch.float32:
        tol = (1.5 * z * z + 36) * U * p + (z * z + 8) * U * f + U * np.abs(want)
    else:
        tol = 2.0 ** -12 * (p + f) + 2.0 ** -8 * np.abs(want)
    assert np.all(np.abs(d - want) <= tol + TINY)
