"""mem_linear, mem_act_backward and mem_linear_backward against the fp64 oracle.

Whole-number inputs give sums that fp32 holds exactly in any order: there the
products have to be equal.  For others, with u = 2^-24, a sum of K products in any
order is within K u of the sum of their sizes; the epilogue adds 4 u of its terms
and the rounding to the stored type half a step (bf16 2^-8).  Activations are within
16 u of |z| + |act| in fp32 and within 2^-12 of them where bf16 is stored (a fast
exponential and an approximated erf)."""
import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk
from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
NAMES = {F32: "f32", BF16: "bf16", E4M3: "e4m3"}
U = 2.0 ** -24
HALF = {F32: U, BF16: 2.0 ** -8}
# T, N, K: one row, edges of the 32-, 128- and 256-wide blocks, k shorter than a
# stage, at its edges, and of many stages; the last ones fill the large tiles
SHAPES = [(1, 8, 16), (1, 2048, 512), (2, 24, 48), (3, 520, 1040), (17, 136, 80), (31, 64, 64), (33, 128, 128), (65, 264, 208),
          (127, 8, 2048), (129, 256, 32), (255, 1032, 144), (300, 72, 16), (1000, 328, 272), (6500, 2056, 80),
          (25700, 520, 272)]


def f64(t):
    return t.detach().cpu().double().numpy()


def ints(shape, dt, seed, most=4):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).float().to(dt).cuda()


def randn(shape, dt, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dt)


def exact_mm(a, b):
    """a b^T in 64 bits, as a tensor on the GPU."""
    return a.double() @ b.double().t().contiguous()


@pytest.mark.parametrize("dt", [F32, BF16, E4M3], ids=NAMES.get)
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_whole_numbers(gpu_lib, T, N, K, dt):
    x, w = ints((T, K), dt, 1), ints((N, K), dt, 2)
    kw, scale = {}, 1.0
    if dt == E4M3:  # powers of two as scales keep the sums exact
        sx, sw = (2.0 ** torch.arange(n, device="cuda").remainder(5).sub(2) for n in (T, N))
        kw, scale = dict(x_scale=sx.float(), w_scale=sw.float()), sx.double()[:, None] * sw.double()
    out = F32
    b, r = ints((N,), out, 3), ints((T, N), out, 4)
    y, z = pk.mem_linear(x, w, b, residual=r, act="relu", out_dtype=out, want_z=True, **kw)
    want = exact_mm(x.float(), w.float()) * scale + b.double()
    assert torch.equal(z.double(), want)
    assert torch.equal(y.double(), want.clamp(min=0) + r.double())
    y, none = pk.mem_linear(x, w, out_dtype=out, **kw)
    assert none is None and torch.equal(y.double(), want - b.double())


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dt", [F32, BF16, E4M3], ids=NAMES.get)
@pytest.mark.parametrize("T,N,K", [(1, 40, 48), (7, 136, 512), (200, 264, 336), (6500, 2048, 80)])
def test_epilogue(gpu_lib, T, N, K, dt, act):
    x, w = randn((T, K), F32, 1), randn((N, K), F32, 2, 2.0 / K ** 0.5)
    kw, sx, sw = {}, 1.0, 1.0
    if dt == E4M3:
        (x, a), (w, b) = pk.mem_quantize_rows(x), pk.mem_quantize_rows(w)
        kw, sx, sw = dict(x_scale=a, w_scale=b), a.double()[:, None], b.double()
    else:
        x, w = x.to(dt), w.to(dt)
    for out in ((F32,) if dt == F32 else (BF16, F32)):
        bias, res = randn((N,), out, 3), randn((T, N), out, 4)
        y, z = pk.mem_linear(x, w, bias, residual=res, act=act, out_dtype=out, want_z=True, **kw)
        assert y.dtype == z.dtype == out
        want_z = exact_mm(x.float(), w.float()) * sx * sw + bias.double()
        sizes = exact_mm(x.float().abs(), w.float().abs()) * sx * sw + bias.double().abs()
        ez = (K + 4) * U * sizes
        assert torch.all((z.double() - want_z).abs() <= ez + HALF[out] * want_z.abs())
        a = torch.from_numpy(bo.act(f64(want_z), act)).cuda()
        want = a + res.double()
        fast = 0.0 if act in ("none", "relu") else 16 * U if out == F32 else 2.0 ** -12
        # no activation is steeper than 1.13
        tol = 1.13 * ez + fast * (want_z.abs() + a.abs()) + 2 * U * (a.abs() + res.double().abs()) + HALF[out] * want.abs()
        assert torch.all((y.double() - want).abs() <= tol + 1e-30)
        into = res.clone()
        y2, _ = pk.mem_linear(x, w, bias, residual=into, act=act, out_dtype=out, y_out=into, **kw)
        assert y2 is into and torch.equal(y2, y)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dt", [F32, BF16], ids=NAMES.get)
def test_act_backward(gpu_lib, dt, act):
    z = randn((1001, 24), F32, 5, 3.0)
    z[0, :8] = torch.tensor([0.0, -0.0, 30.0, -30.0, 100.0, -100.0, 1e4, -1e4])
    z, dy = z.to(dt), randn((1001, 24), dt, 6)
    dz = pk.mem_act_backward(dy, z, act)
    d = bo.act_grad(np.clip(f64(z), -700, 700), act)
    want = f64(dy) * d
    fast = 0.0 if act in ("none", "relu") else 16 * U if dt == F32 else 2.0 ** -12
    tol = np.abs(f64(dy)) * fast * (1 + np.abs(d)) + (HALF[dt] + 2 * U) * np.abs(want)
    assert np.all(np.abs(f64(dz) - want) <= tol + 1e-38)
    for into in (dy.clone(), z.clone()):
        a, b = (into, z) if torch.equal(into, dy) else (dy, into)
        assert torch.equal(pk.mem_act_backward(a, b, act, dz_out=into), dz)


@pytest.mark.parametrize("dt", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("T,N,K", SHAPES + [(4100, 1024, 1032), (8192, 1288, 1024)])
def test_backward_whole_numbers(gpu_lib, T, N, K, dt):
    dz, x, w, add = ints((T, N), dt, 1, 2), ints((T, K), dt, 2, 2), ints((N, K), dt, 3, 2), ints((T, K), dt, 4)
    gw, gb = ints((N, K), F32, 5), ints((N,), F32, 6)
    want_w = exact_mm(dz.float().t().contiguous(), x.float().t().contiguous()) + gw.double()
    want_b = dz.double().sum(0) + gb.double()
    dx, got_w, got_b = pk.mem_linear_backward(dz, x, w, dx_add=add, grad_w=gw, grad_bias=gb)
    assert got_w is gw and got_b is gb
    assert torch.equal(gw.double(), want_w) and torch.equal(gb.double(), want_b)
    want = exact_mm(dz.float(), w.float().t().contiguous()) + add.double()
    assert torch.equal(dx, want.to(dt))
    into = add.clone()
    assert torch.equal(pk.mem_linear_backward(dz, x, w, dx_add=into, dx=into, want_grad_w=False, want_grad_bias=False)[0], dx)


@pytest.mark.parametrize("dt", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("T,N,K", [(1, 8, 8), (100, 264, 72), (3000, 136, 520), (9000, 1032, 1024)])
def test_backward(gpu_lib, T, N, K, dt):
    dz, x, w = randn((T, N), dt, 1), randn((T, K), dt, 2), randn((N, K), dt, 3, 0.05)
    dx, gw, gb = pk.mem_linear_backward(dz, x, w)
    a, b = dz.float(), x.float()
    want = exact_mm(a, w.float().t().contiguous())
    size = exact_mm(a.abs(), w.float().abs().t().contiguous())
    assert torch.all((dx.double() - want).abs() <= N * U * size + HALF[dt] * want.abs())
    at, bt = a.t().contiguous(), b.t().contiguous()
    assert torch.all((gw.double() - exact_mm(at, bt)).abs() <= (T + 70) * U * exact_mm(at.abs(), bt.abs()))
    # a thread adds at most T / 16 of the rows, a workgroup 32 threads, the call 64 splits of 9 tiles
    assert torch.all((gb.double() - a.double().sum(0)).abs() <= (T / 16 + 700) * U * a.double().abs().sum(0))
    for _ in range(3):
        again = pk.mem_linear_backward(dz, x, w)
        assert torch.equal(again[0], dx) and torch.equal(again[1], gw) and torch.equal(again[2], gb)
    for want in ((True, False, False), (False, True, False), (False, False, True)):
        some = pk.mem_linear_backward(dz, x, w, want_dx=want[0], want_grad_w=want[1], want_grad_bias=want[2])
        for got, ref, on in zip(some, (dx, gw, gb), want):
            assert (got is None) != on
            if on and ref is gb:  # alone it is summed in another order
                assert torch.all((got.double() - a.double().sum(0)).abs() <= (T / 512 + 80) * U * a.double().abs().sum(0))
            elif on:
                assert torch.equal(got, ref)


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_gradients_against_differences(gpu_lib, act):
    """Central differences of the fp32 forward through a loss sum(dy y) in 64 bits: a step h
    on one entry moves the loss by its gradient, off by the third derivative (h^2) and by the
    forward's rounding over 2 h."""
    T, N, K = 40, 72, 48
    x, w, b, dy = randn((T, K), F32, 1), randn((N, K), F32, 2, 0.2), randn((N,), F32, 3), randn((T, N), F32, 4)
    z = pk.mem_linear(x, w, b, act=act, want_z=True)[1]
    dx, gw, gb = pk.mem_linear_backward(pk.mem_act_backward(dy, z, act), x, w)
    loss = lambda: float((dy.double() * pk.mem_linear(x, w, b, act=act)[0].double()).sum())  # noqa: E731
    h = 2.0 ** -7
    for t, g, at in ((x, dx, (3, 5)), (w, gw, (70, 47)), (b, gb, (11,))):
        old = float(t[at])
        t[at] = old + h
        up = loss()
        t[at] = old - h
        down = loss()
        t[at] = old
        # outputs of one row or column: at most 72 terms of size ~4, each off by K u of 10 and by
        # h^2 / 6 * 2 of a slope's change; a kink of relu inside the step counts h of its term
        kink = 72 * 4 * 0.2 * h if act == "relu" else 0.0
        assert abs((up - down) / (2 * h) - float(g[at])) <= 72 * 4 * (K * U * 10 / h + h * h / 3) + kink


def test_fp32_of_any_scale(gpu_lib):
    """Powers of two go through the product untouched: operands scaled by 2^e and 2^-e give
    the same bits, and products far from one in size stay within the bound of fp32."""
    T, N, K = 200, 136, 264
    x, w, dz = randn((T, K), F32, 1), randn((N, K), F32, 2), randn((T, N), F32, 3)
    y, _ = pk.mem_linear(x, w)
    want = exact_mm(x, w)
    assert torch.all((y.double() - want).abs() <= (K + 4) * U * exact_mm(x.abs(), w.abs()))
    dx, gw, _ = pk.mem_linear_backward(dz, x, w)
    for e in (40, 80, -80):
        s = 2.0 ** e
        assert torch.equal(pk.mem_linear(x * s, w / s)[0], y)
        got = pk.mem_linear_backward(dz * s, x / s, w / s)
        assert torch.equal(got[0], dx) and torch.equal(got[1], gw)
    # entries of one row from 2^-30 to 2^30
    x = x * 2.0 ** torch.randint(-30, 31, x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(4)).float()
    assert torch.all((pk.mem_linear(x, w)[0].double() - exact_mm(x, w)).abs() <= (K + 4) * U * exact_mm(x.abs(), w.abs()))


def test_special_values(gpu_lib):
    """A NaN or infinity reaches the outputs that use it and no others, also where
    rows and k end inside a tile."""
    for dt in (F32, BF16):
        x, w = randn((70, 40), dt, 1), randn((136, 40), dt, 2)
        x[5, 39] = float("inf")
        w[130, 0] = float("nan")
        y, _ = pk.mem_linear(x, w)
        bad = torch.zeros(70, 136, dtype=torch.bool, device="cuda")
        bad[5] = True
        bad[:, 130] = True
        assert torch.equal(~torch.isfinite(y), bad)
        dz = randn((70, 136), dt, 3)
        dz[69, 135] = float("inf")
        dx, gw, gb = pk.mem_linear_backward(dz, x[:, :40].clone().fill_(1.0), w.nan_to_num(1.0))
        assert torch.equal((~torch.isfinite(dx)).any(1).nonzero().flatten(), torch.tensor([69], device="cuda"))
        assert torch.equal((~torch.isfinite(gw)).any(1).nonzero().flatten(), torch.tensor([135], device="cuda"))
        assert torch.equal((~torch.isfinite(gb)).nonzero().flatten(), torch.tensor([135], device="cuda"))


def test_rows_behind_the_last_stay(gpu_lib):
    big = torch.full((300, 136), 7.0, device="cuda")
    x, w = randn((129, 72), F32, 1), randn((136, 72), F32, 2)
    pk.mem_linear(x, w, y_out=big[:129])
    assert torch.all(big[129:] == 7)
    dx = torch.full((300, 72), 7.0, device="cuda")
    pk.mem_linear_backward(randn((129, 136), F32, 3), x, w, dx=dx[:129])
    assert torch.all(dx[129:] == 7)


def test_empty_and_refusals(gpu_lib):
    x, w = torch.zeros((0, 64), device="cuda"), torch.zeros((32, 64), device="cuda")
    y, _ = pk.mem_linear(x, w)
    assert y.shape == (0, 32)
    dx, gw, gb = pk.mem_linear_backward(y, x, w)
    assert dx.shape == (0, 64) and not gw.any() and not gb.any()
    x = torch.zeros((4, 64), device="cuda")
    for args, kw in (((x, w[:, :32].contiguous()), {}), ((x, w.bfloat16()), {}), ((x, w.t()), {}), ((x, w, w[0]), {}),
                     ((x, w), dict(residual=x)), ((x, w), dict(y_out=torch.zeros(4, 31, device="cuda"))),
                     ((x.to(E4M3), w.to(E4M3)), {}), ((x.cpu(), w), {})):
        with pytest.raises(ValueError):
            pk.mem_linear(*args, **kw)
    with pytest.raises(KeyError):
        pk.mem_linear(x, w, act="tanh")
    with pytest.raises(pk.PkmemError):
        pk.mem_linear(x, w, act=9)
    with pytest.raises(pk.PkmemError):
        pk.mem_linear(x, w, out_dtype=BF16)
    with pytest.raises(pk.PkmemError):
        pk.mem_linear(x[:, :60].contiguous(), w[:, :60].contiguous())
    with pytest.raises(ValueError):
        pk.mem_linear_backward(torch.zeros(4, 32, device="cuda"), x, w, grad_w=torch.zeros(32, 64, device="cuda").bfloat16())
    with pytest.raises(ValueError):
        pk.mem_linear_backward(torch.zeros(4, 32, device="cuda"), x, w, workspace=torch.zeros(1, device="cuda"))
