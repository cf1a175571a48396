"""Rows in 8 bits of any fp32 numbers: every code is the e4m3 number nearest to
448 y / max|y|, formed in 64 bits and rounded to fp32 first.  Two computations in 64
bits differ by 2^-51 of the quotient, which meets a border of fp32 once in 2^27
elements and one of e4m3 only if that border is its own: all codes have to be equal."""
import pytest
import torch

import paper_2412_09764_amd as pk

pytestmark = pytest.mark.gpu

SHAPES = [(4001, 1032), (3000, 2048), (1500, 4104), (700, 8192), (20000, 72)]


def nearest(u):
    top = u.abs().amax(-1, keepdim=True)
    return (u * 448 / top).float().to(torch.float8_e4m3fn).float()


def rand(shape, seed, std=1.0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * std


@pytest.mark.parametrize("T,D", SHAPES)
def test_quantize_rows(gpu_lib, T, D):
    x = rand((T, D), 1) * 2.0 ** torch.randint(-40, 40, (T, 1), device="cuda", generator=torch.Generator("cuda").manual_seed(2)).float()
    q, s = pk.mem_quantize_rows(x)
    assert torch.equal(q.float(), nearest(x.double()))
    assert torch.equal(s, (x.double().abs().amax(-1) / 448).float())


@pytest.mark.parametrize("T,D", SHAPES)
def test_norm(gpu_lib, T, D):
    x, r, w = rand((T, D), 3), rand((T, D), 4, 2.0), 1 + rand((D,), 5, 0.1)
    q, h, s = pk.mem_rmsnorm(x, w, r, quantize=True)
    assert torch.equal(q.float(), nearest(h.double() * w.double()))
    # the scale is that of the norm itself: 44 u of the root of the mean square, and its own rounding
    y = h.double() * w.double() / (h.double().square().mean(-1, keepdim=True) + 1e-5).sqrt()
    want = y.abs().amax(-1) / 448
    assert torch.all((s.double() - want).abs() <= 46 * 2.0 ** -24 * want)
