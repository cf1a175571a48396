"""Products in blocks and the gated part at sizes whose workgroups take tile after tile (more
tiles than the chip holds at once; test_tile_walk.py counts them): results of one tile leave while
the next one's codes arrive.

Whole numbers, with powers of two as scales: codes up to 4 give products up to 16, which the 8-bit
instruction keeps whole (13 bits below the largest), sums of up to 528 of them in steps of 2^-4
are below 2^18 and so exact in fp32 in any order, and each result is rounded once.  Others are
held to the bounds of test_gpu_blocks.py and test_gpu_glu.py.  Outputs are filled with NaN before
and stand in front of rows that have to stay as they were."""
import pytest
import torch

import paper_2412_09764_amd as pk
from oracle import block_oracle as bo
from tests.test_gpu_blocks import scales, spread
from tests.test_gpu_linear import BF16, E4M3, HALF, U, exact_mm, f64, ints, randn

pytestmark = pytest.mark.gpu

# T, N, K: 128-wide tiles, two and four a workgroup; 256-wide ones, two and four.  Steps of 128 k
# (64 of bf16): one, an even and an odd number, the last of them partly empty.
BLOCKS = [(3000, 3848, 400), (3001, 3848, 528), (3000, 3840, 16), (100, 200008, 272),
          (8200, 2312, 400), (8201, 2312, 528), (8200, 2304, 128), (16500, 3080, 272)]
GLU = [(3000, 1928, 400), (3001, 1928, 528), (3000, 1920, 16), (100, 100008, 272),
       (8200, 1160, 400), (8201, 1160, 528), (8200, 1152, 128), (16500, 1544, 272)]
GUARD = 3  # rows behind an output


def fresh(T, N, dt=BF16):
    """An output of T rows and the buffer that it begins."""
    whole = torch.full((T + GUARD, N), float("nan"), dtype=dt, device="cuda")
    whole[T:] = 77
    return whole[:T], whole


def kept(*wholes):
    return all(bool((w[-GUARD:] == 77).all()) for w in wholes)


@pytest.mark.parametrize("tile", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("T,N,K", BLOCKS)
def test_blocks(gpu_lib, T, N, K, tile):
    x, w = ints((T, K), E4M3, 1), ints((N, K), E4M3, 2)
    kb, nb = -(-K // 128), -(-N // 128) if tile else N
    sx, sw = scales((kb, T), 3), scales((kb, nb), 4)
    want = (x.double() * spread(sx, 1, T, K)) @ (w.double() * spread(sw, 128 if tile else 1, N, K)).t().contiguous()
    bias, res = ints((N,), BF16, 5), ints((T, N), BF16, 6)
    wz = want + bias.double()
    with_z, with_res, both = wz.to(BF16), (want + res.double()).to(BF16), (wz.clamp(min=0) + res.double()).to(BF16)
    relu, plain = wz.clamp(min=0).to(BF16), want.to(BF16)
    del want, wz
    for _ in range(2):
        (y, whole), (z, zwhole) = fresh(T, N), fresh(T, N)
        pk.mem_linear_blocks(x, w, sx, sw, bias, residual=res, act="relu", y_out=y, z_out=z)
        assert torch.equal(y, both) and torch.equal(z, with_z) and kept(whole, zwhole)
        (y, whole), (z, zwhole) = fresh(T, N), fresh(T, N)
        pk.mem_linear_blocks(x, w, sx, sw, bias, act="relu", y_out=y, z_out=z)
        assert torch.equal(y, relu) and torch.equal(z, with_z) and kept(whole, zwhole)
        y, whole = fresh(T, N)
        y.copy_(res)
        pk.mem_linear_blocks(x, w, sx, sw, residual=y, y_out=y)
        assert torch.equal(y, with_res) and kept(whole)
        y, whole = fresh(T, N)
        pk.mem_linear_blocks(x, w, sx, sw, y_out=y)
        assert torch.equal(y, plain) and kept(whole)


@pytest.mark.parametrize("dt", [BF16, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,N,K", GLU)
def test_glu(gpu_lib, T, N, K, dt):
    x, w = ints((T, K), dt, 1, 3), ints((2 * N, K), dt, 2, 3)
    kw, scale = {}, 1.0
    if dt == E4M3:
        sx, sw = (2.0 ** torch.arange(n, device="cuda").remainder(3).sub(1) for n in (T, 2 * N))
        kw, scale = dict(x_scale=sx.float(), w_scale=sw.float()), sx.double()[:, None] * sw.double()
    b = ints((2 * N,), BF16, 3)
    want = exact_mm(x.float(), w.float()) * scale
    plain = (want[:, :N].clamp(min=0) * want[:, N:]).float().to(BF16)
    want += b.double()
    with_z, with_bias = want.to(BF16), (want[:, :N].clamp(min=0) * want[:, N:]).float().to(BF16)
    del want
    for _ in range(2):
        (y, whole), (z, zwhole) = fresh(T, N), fresh(T, 2 * N)
        pk.mem_glu(x, w, b, act="relu", y_out=y, z_out=z, **kw)
        assert torch.equal(y, with_bias) and torch.equal(z, with_z) and kept(whole, zwhole)
        y, whole = fresh(T, N)
        pk.mem_glu(x, w, act="relu", y_out=y, **kw)
        assert torch.equal(y, plain) and kept(whole)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("tile", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("T,N,K", [(3000, 3848, 400), (8200, 2312, 400)])
def test_blocks_of_any_numbers(gpu_lib, T, N, K, tile, act):
    (x, sx, _, _), (w, sw, _, _) = pk.mem_quantize_blocks(randn((T, K), BF16, 1)), pk.mem_quantize_blocks(randn((N, K), BF16, 2) / K ** 0.5, tile=tile)
    a, b = x.double() * spread(sx.double(), 1, T, K), w.double() * spread(sw.double(), 128 if tile else 1, N, K)
    want_z, size = a @ b.t().contiguous(), a.abs() @ b.abs().t().contiguous()
    bias, res = randn((N,), BF16, 3), randn((T, N), BF16, 4)
    want_z += bias.double()
    ez = ((K / 32 + 140) * U + 2.0 ** -10) * size + 4 * U * bias.double().abs()
    f = torch.from_numpy(bo.act(f64(want_z), act)).cuda()
    for add in (None, res):
        y, z = pk.mem_linear_blocks(x, w, sx, sw, bias, residual=add, act=act, want_z=True)
        assert torch.all((z.double() - want_z).abs() <= ez + HALF[BF16] * (want_z.abs() + ez))
        r = 0.0 if add is None else add.double()
        want = f + r
        tol = 1.13 * ez + 2.0 ** -12 * (want_z.abs() + f.abs()) + 2 * U * (f.abs() + res.double().abs())
        assert torch.all((y.double() - want).abs() <= tol + HALF[BF16] * (want.abs() + tol))
        again, _ = pk.mem_linear_blocks(x, w, sx, sw, bias, residual=add, act=act)  # without z
        assert torch.equal(again, y)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("dt", [BF16, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,N,K", [(3000, 1928, 400), (8200, 1160, 400)])
def test_glu_of_any_numbers(gpu_lib, T, N, K, dt, act):
    x, w = randn((T, K), torch.float32, 1), randn((2 * N, K), torch.float32, 2, 2.0 / K ** 0.5)
    kw, s = {}, 1.0
    if dt == E4M3:
        (x, a), (w, b) = pk.mem_quantize_rows(x), pk.mem_quantize_rows(w)
        kw, s = dict(x_scale=a, w_scale=b), a.double()[:, None] * b.double()
    else:
        x, w = x.to(dt), w.to(dt)
    bias = randn((2 * N,), BF16, 3)
    y, z = pk.mem_glu(x, w, bias, act=act, want_z=True, **kw)
    want_z = exact_mm(x.float(), w.float()) * s + bias.double()
    size = exact_mm(x.float().abs(), w.float().abs()) * s
    ez = (K + 4) * U * (size + bias.double().abs()) + (2.0 ** -10 * size if dt == E4M3 else 0.0)
    assert torch.all((z.double() - want_z).abs() <= ez + HALF[BF16] * (want_z.abs() + ez))
    gate, up = want_z[:, :N], want_z[:, N:]
    f = torch.from_numpy(bo.act(f64(gate), act)).cuda()
    ea = 1.13 * ez[:, :N] + (0.0 if act == "none" else 2.0 ** -12) * (gate.abs() + f.abs())
    want = f * up
    tol = ea * (up.abs() + ez[:, N:]) + f.abs() * ez[:, N:] + U * want.abs()
    assert torch.all((y.double() - want).abs() <= tol + HALF[BF16] * (want.abs() + tol))
    again, _ = pk.mem_glu(x, w, bias, act=act, **kw)  # without z
    assert torch.equal(again, y)
