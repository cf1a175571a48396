"""mem_glu and mem_glu_backward against the fp64 oracle.

Whole-number inputs give sums that fp32 holds exactly in any order: there the products have
to be equal.  For others, with u = 2^-24, a sum of K products in any order is within K u of
the sum of their sizes and the scales and bias add 4 u; activations are within 16 u of
|z| + |act| in fp32 and within 2^-12 of them where bf16 is stored, none is steeper than
1.13, and the rounding to the stored type is half a step (bf16 2^-8).  For 8-bit operands with
bf16 results the instruction cuts each of 8 products 13 bits below the largest of them: a sum
is then within 8 * 2^-13 of the sum of its sizes as a bound."""
import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk
from oracle import block_oracle as bo
from tests.test_gpu_linear import BF16, E4M3, F32, HALF, NAMES, U, exact_mm, f64, ints, randn

pytestmark = pytest.mark.gpu

# T, N, K: every tile (see test_more_plan.py), its edges, k shorter than a stage and of many
SHAPES = [(1, 8, 16), (1, 2048, 512), (3, 520, 1040), (8, 24, 48), (9, 24, 48), (17, 136, 80), (33, 40, 128), (65, 264, 208),
          (129, 256, 32), (255, 1032, 144), (300, 72, 16), (1000, 328, 272), (1000, 1032, 80), (2000, 1048, 400),
          (4100, 520, 80), (6500, 1032, 80), (25700, 264, 272)]


@pytest.mark.parametrize("dt", [F32, BF16, E4M3], ids=NAMES.get)
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_whole_numbers(gpu_lib, T, N, K, dt):
    x, w = ints((T, K), dt, 1, 3), ints((2 * N, K), dt, 2, 3)
    kw, scale = {}, 1.0
    if dt == E4M3:  # powers of two as scales keep the sums exact
        sx, sw = (2.0 ** torch.arange(n, device="cuda").remainder(3).sub(1) for n in (T, 2 * N))
        kw, scale = dict(x_scale=sx.float(), w_scale=sw.float()), sx.double()[:, None] * sw.double()
    b = ints((2 * N,), F32, 3)
    want = exact_mm(x.float(), w.float()) * scale + b.double()
    for act, f in (("relu", lambda z: z.clamp(min=0)), ("none", lambda z: z)):
        y, z = pk.mem_glu(x, w, b, act=act, out_dtype=F32, want_z=True, **kw)
        assert y.shape == (T, N) and torch.equal(z.double(), want)
        # one product of exact numbers, rounded once
        assert torch.equal(y, (f(want[:, :N]) * want[:, N:]).float())
    y, none = pk.mem_glu(x, w, act="relu", out_dtype=F32, **kw)
    want -= b.double()
    assert none is None and torch.equal(y, (want[:, :N].clamp(min=0) * want[:, N:]).float())
    if dt != F32:
        y, z = pk.mem_glu(x, w, act="relu", out_dtype=BF16, want_z=True, **kw)
        assert torch.equal(z, want.to(BF16))
        assert torch.equal(y, (want[:, :N].clamp(min=0) * want[:, N:]).float().to(BF16))


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dt", [F32, BF16, E4M3], ids=NAMES.get)
@pytest.mark.parametrize("T,N,K", [(1, 40, 48), (7, 136, 512), (200, 264, 336), (6500, 1032, 80)])
def test_epilogue(gpu_lib, T, N, K, dt, act):
    x, w = randn((T, K), F32, 1), randn((2 * N, K), F32, 2, 2.0 / K ** 0.5)
    kw, sx, sw = {}, 1.0, 1.0
    if dt == E4M3:
        (x, a), (w, b) = pk.mem_quantize_rows(x), pk.mem_quantize_rows(w)
        kw, sx, sw = dict(x_scale=a, w_scale=b), a.double()[:, None], b.double()
    else:
        x, w = x.to(dt), w.to(dt)
    for out in ((F32,) if dt == F32 else (BF16, F32)):
        bias = randn((2 * N,), out, 3)
        y, z = pk.mem_glu(x, w, bias, act=act, out_dtype=out, want_z=True, **kw)
        assert y.dtype == z.dtype == out
        want_z = exact_mm(x.float(), w.float()) * sx * sw + bias.double()
        size = exact_mm(x.float().abs(), w.float().abs()) * sx * sw
        ez = (K + 4) * U * (size + bias.double().abs())
        if dt == E4M3 and out == BF16:  # each of 8 products within 2^-13 of the largest of them
            ez = ez + 2.0 ** -10 * size
        assert torch.all((z.double() - want_z).abs() <= ez + HALF[out] * want_z.abs())
        gate, up = want_z[:, :N], want_z[:, N:]
        a = torch.from_numpy(bo.act(f64(gate), act)).cuda()
        fast = 0.0 if act in ("none", "relu") else 16 * U if out == F32 else 2.0 ** -12
        ea = 1.13 * ez[:, :N] + fast * (gate.abs() + a.abs())
        want = a * up
        tol = ea * (up.abs() + ez[:, N:]) + a.abs() * ez[:, N:] + (U + HALF[out]) * want.abs() + HALF[out] * ea * up.abs()
        assert torch.all((y.double() - want).abs() <= tol + 1e-30)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dt", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("T,N", [(1, 8), (1001, 24), (333, 1032)])
def test_backward(gpu_lib, T, N, dt, act):
    z, dy = randn((T, 2 * N), F32, 5, 3.0), randn((T, N), dt, 6)
    if T > 1:
        z[0, :8] = torch.tensor([0.0, -0.0, 30.0, -30.0, 100.0, -100.0, 1e4, -1e4])
    z = z.to(dt)
    dz = pk.mem_glu_backward(dy, z, act)
    zz = f64(z)
    if act in ("silu", "gelu"):  # exp in the oracle; both sides are 0 below
        zz[:, :N] = np.clip(zz[:, :N], -700, None)
    want = bo.glu_backward(f64(dy), zz, act)
    d, a = np.abs(bo.act_grad(zz[:, :N], act)), np.abs(bo.act(zz[:, :N], act))
    fast = 0.0 if act in ("none", "relu") else 16 * U
    ady, up = np.abs(f64(dy)), np.abs(zz[:, N:])
    tol = np.concatenate([ady * up * fast * (1 + d), ady * fast * (np.abs(zz[:, :N]) + a)], 1) + (HALF[dt] + 3 * U) * np.abs(want)
    assert np.all(np.abs(f64(dz) - want) <= tol + 1e-38)
    into = z.clone()
    assert pk.mem_glu_backward(dy, into, act, dz_out=into) is into and torch.equal(into, dz)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_through(gpu_lib, act):
    """Forward and backward in fp32 against autograd in 64 bits: each number is a sum of at most
    400 products of up to three factors, below 2^10 roundings of 2^-24 of the largest."""
    T, N, K = 200, 136, 72
    x, w, b, dy = randn((T, K), F32, 1), randn((2 * N, K), F32, 2, 0.1), randn((2 * N,), F32, 3), randn((T, N), F32, 4)
    y, z = pk.mem_glu(x, w, b, act=act, want_z=True)
    dz = pk.mem_glu_backward(dy, z, act)
    dx, gw, gb = pk.mem_linear_backward(dz, x, w)
    t = [v.cpu().double().requires_grad_() for v in (x, w, b)]
    zz = t[0] @ t[1].t() + t[2]
    f = torch.nn.functional.silu if act == "silu" else torch.nn.functional.gelu
    yy = f(zz[:, :N]) * zz[:, N:]
    (yy * dy.cpu().double()).sum().backward()
    for got, want in ((y, yy.detach()), (dx, t[0].grad), (gw, t[1].grad), (gb, t[2].grad)):
        assert float((got.cpu().double() - want).abs().max()) <= 2.0 ** -14 * float(want.abs().max())


def test_infinities_and_nan_stay_in_their_row(gpu_lib):
    T, N, K = 300, 72, 64
    x, w = randn((T, K), BF16, 1), randn((2 * N, K), BF16, 2)
    clean, _ = pk.mem_glu(x, w)
    x[7, 3], x[200, 0] = float("nan"), float("inf")
    y, _ = pk.mem_glu(x, w)
    rest = [i for i in range(T) if i not in (7, 200)]
    assert torch.isnan(y[7]).all() and not torch.isfinite(y[200]).any()
    assert torch.equal(y[rest], clean[rest])


def test_no_rows(gpu_lib):
    w = randn((48, 16), BF16, 1)
    y, z = pk.mem_glu(torch.empty((0, 16), dtype=BF16, device="cuda"), w, want_z=True)
    assert y.shape == (0, 24) and z.shape == (0, 48)
    assert pk.mem_glu_backward(y, z).shape == (0, 48)
