"""mem_quantize_blocks and mem_linear_blocks against the fp64 oracle.

Codes are the oracle's, all of them; scales are one division in fp32 (u = 2^-24).  With
whole-number codes and powers of two as scales every sum is exact in fp32 in any order and
products have to be equal.  For others: products of codes are exact, a block's sum of 128 is
within 128 u of its sizes, its two scales and its addition are 3 u, the blocks' sum
ceil(K / 128) u (and twice that for sums in halves of a block and groups of waves): together
(K / 32 + 140) u of the sum of all sizes, 4 u for the bias.  Where bf16 is stored, each
product is moreover within 2^-13 of the largest of 8, hence their sum within 8 * 2^-13 of all
sizes as a bound, and activations are within 2^-12 of |z| + |act| (16 u in fp32), none
steeper than 1.13; the stored type takes half a step."""
import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk
from oracle import block_oracle as bo
from tests.test_gpu_linear import BF16, E4M3, F32, HALF, U, exact_mm, f64, ints, randn

pytestmark = pytest.mark.gpu

IDS = {F32: "f32", BF16: "bf16"}


def uneven(R, C, dt, seed):
    x = randn((R, C), F32, seed) * torch.exp(randn((R, C), F32, seed + 100) * 2)
    if R > 2 and C >= 32:
        x[1] = 0
        x[2, :16] = 3.0e-39  # below the least scale
        x[2, 16:] = 0
    return x.to(dt)


def check_codes(x, rows, q, s, want_t):
    """q, s of x's rows (want_t: of its columns) in blocks of `rows` x 128."""
    v = f64(x).T if want_t else f64(x)
    wq, _, ws = bo.quantize_blocks(v, rows)
    n = v.shape[1]
    got = f64(q.float())
    assert got.shape == (v.shape[0], -(-n // 16) * 16 if want_t else n) and tuple(s.shape) == ws.shape
    assert np.array_equal(got[:, :n], wq) and not got[:, n:].any()
    assert np.all(np.abs(f64(s) - ws) <= U * ws)


@pytest.mark.parametrize("dt", [F32, BF16], ids=IDS.get)
@pytest.mark.parametrize("R,C", [(1, 16), (3, 48), (17, 128), (5, 144), (128, 2048), (129, 272), (300, 112), (777, 1040), (16, 4112)])
def test_codes(gpu_lib, R, C, dt):
    x = uneven(R, C, dt, R + C)
    for tile, rows in ((False, 1), (True, 128)):
        q, s, qt, st = pk.mem_quantize_blocks(x, tile=tile, want_cols=True)
        check_codes(x, rows, q, s, False)
        check_codes(x, rows, qt, st, True)
        q1, s1, none, none2 = pk.mem_quantize_blocks(x, tile=tile)
        assert none is None and none2 is None and torch.equal(q1.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s1, s)
        none, none2, q1, s1 = pk.mem_quantize_blocks(x, tile=tile, want_rows=False, want_cols=True)
        assert none is None and none2 is None and torch.equal(q1.view(torch.uint8), qt.view(torch.uint8)) and torch.equal(s1, st)


@pytest.mark.parametrize("top", [448.0, 1.0, 3.0, 1.75 * 2.0 ** 100, 1.1 * 2.0 ** -110, 449.5 * 2.0 ** -126, 447.0 * 2.0 ** -126,
                                 2.0 ** -149, 3.0e38, 1.0 + 2.0 ** -23, 7.0 / 3.0])
def test_borders(gpu_lib, top):
    """fp32 numbers on, right below and right above every border between two codes, for
    largest numbers of many kinds."""
    top = np.float32(top)
    grid = np.unique(np.abs(bo.e4m3_values()[np.isfinite(bo.e4m3_values())]))
    mid = (grid[1:] + grid[:-1]) / 2
    scale = max(float(top) / 448, 2.0 ** -126)
    v = (mid * scale).astype(np.float32)
    v = np.concatenate([v, np.nextafter(v, np.float32(0)), np.nextafter(v, np.float32(np.inf)),
                        np.nextafter(np.nextafter(v, np.float32(0)), np.float32(0))])
    v = v[v < top]
    v = np.concatenate([v, -v])
    rows = [np.concatenate([[top], v[i:i + 127], np.zeros(127 - len(v[i:i + 127]), np.float32)]) for i in range(0, max(len(v), 1), 127)]
    x = torch.from_numpy(np.stack(rows).astype(np.float32)).cuda()
    q, s, _, _ = pk.mem_quantize_blocks(x)
    check_codes(x, 1, q, s, False)
    t = torch.cat([x, x.new_zeros((-len(x) % 16, 128))]).t().contiguous()
    _, _, q, s = pk.mem_quantize_blocks(t, want_cols=True, want_rows=False)
    check_codes(t, 1, q, s, True)


def test_borders_of_bf16(gpu_lib):
    """Every bf16 number between 2^-10 and 1 in a block with each of 128 largest numbers."""
    tops = (1 + torch.arange(128).float() / 128).bfloat16()
    vals = torch.arange(0x3A80, 0x3F80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    vals = torch.cat([vals, vals.new_zeros(-len(vals) % 127)]).view(-1, 127)
    x = torch.cat([torch.cat([tops[i].expand(len(vals), 1), vals], 1) for i in range(128)]).cuda()
    q, s, _, _ = pk.mem_quantize_blocks(x)
    check_codes(x, 1, q, s, False)


def test_nan_and_infinity_stay_in_their_block(gpu_lib):
    x = randn((256, 256), F32, 1)
    clean = pk.mem_quantize_blocks(x, want_cols=True)
    x[3, 5], x[200, 130] = float("nan"), float("inf")
    got = pk.mem_quantize_blocks(x, want_cols=True)
    v = (got[0].float().view(256, 2, 128) * got[1].t()[:, :, None]).view(256, 256)
    w = (clean[0].float().view(256, 2, 128) * clean[1].t()[:, :, None]).view(256, 256)
    assert torch.isnan(v[3, 5]) and not torch.isfinite(v[200, 130])
    v[3, :128], v[200, 128:] = w[3, :128], w[200, 128:]
    assert torch.equal(v, w)


@pytest.mark.parametrize("tile", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_codes_beside_an_infinity(gpu_lib, dt, tile, sign):
    x = randn((128, 128), dt, 1)
    x[7, 9], x[70, 9], x[90, 3] = sign * float("inf"), float("nan"), -3.0e38
    q, s, qt, st = pk.mem_quantize_blocks(x, tile=tile, want_cols=True)
    for code, scale, line in ((q, s, 7), (qt.t(), st, 9)):
        v = code.float() if tile else code.float()[7] if line == 7 else code.float()[:, 9]
        hit = ~torch.isfinite(x if tile else x[7] if line == 7 else x[:, 9])
        assert torch.isnan(v[hit]).all() and (v[~hit] == 0).all()
        assert torch.isinf(scale).all() if tile else torch.isinf(scale[0, line]) and torch.isfinite(scale).sum() == 127


# T, N, K: one row to few, edges of the 32-, 64-, 128- and 256-wide tiles, k of a part of a stage,
# of a part of a block, of many blocks
SHAPES = [(1, 8, 16), (1, 2048, 528), (3, 520, 1040), (8, 136, 80), (9, 8, 144), (17, 136, 80), (33, 128, 128), (65, 264, 208),
          (129, 256, 32), (255, 1032, 144), (333, 1096, 400), (1000, 1032, 272), (1800, 1992, 272), (2000, 2056, 144),
          (4100, 1032, 272), (6500, 2056, 272), (40, 72, 2064), (777, 200, 1168),
          (9, 8, 16400), (300, 264, 8208), (2040, 1000, 9008), (130, 2048, 16400)]  # the first, third and fourth: k in parts


def scales(shape, seed):
    g = torch.Generator().manual_seed(seed)
    return (2.0 ** torch.randint(-2, 3, shape, generator=g)).float().cuda()


def spread(s, rows, n, k):
    """[blocks of k, rows or row blocks] to [n, k]."""
    s = s.t().repeat_interleave(128, 1)[:, :k]
    return s if rows == 1 else s.repeat_interleave(128, 0)[:n]


@pytest.mark.parametrize("tile", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_whole_numbers(gpu_lib, T, N, K, tile):
    x, w = ints((T, K), E4M3, 1), ints((N, K), E4M3, 2)
    kb, nb = -(-K // 128), -(-N // 128) if tile else N
    sx, sw = scales((kb, T), 3), scales((kb, nb), 4)
    a, b = x.double() * spread(sx, 1, T, K), w.double() * spread(sw, 128 if tile else 1, N, K)
    want = a @ b.t().contiguous()
    for out in (F32, BF16):
        bias, res = ints((N,), out, 5), ints((T, N), out, 6)
        y, z = pk.mem_linear_blocks(x, w, sx, sw, bias, residual=res, act="relu", out_dtype=out, want_z=True)
        wz = want + bias.double()
        assert torch.equal(z, wz.to(out))
        assert torch.equal(y, (wz.clamp(min=0) + res.double()).to(out))
        into = res.clone()
        y, none = pk.mem_linear_blocks(x, w, sx, sw, residual=into, y_out=into, out_dtype=out)
        assert y is into and none is None and torch.equal(y, (want + res.double()).to(out))


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("tile", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("T,N,K", [(1, 40, 48), (7, 136, 512), (200, 264, 336), (2000, 2056, 400), (6500, 2048, 144)])
def test_product(gpu_lib, T, N, K, tile, act):
    (x, sx, _, _), (w, sw, _, _) = pk.mem_quantize_blocks(uneven(T, K, BF16, 1)), pk.mem_quantize_blocks(uneven(N, K, F32, 2) / K ** 0.5, tile=tile)
    a, b = x.double() * spread(sx.double(), 1, T, K), w.double() * spread(sw.double(), 128 if tile else 1, N, K)
    z64, size = a @ b.t().contiguous(), a.abs() @ b.abs().t().contiguous()
    for out in (F32, BF16):
        bias, res = randn((N,), out, 3), randn((T, N), out, 4)
        y, z = pk.mem_linear_blocks(x, w, sx, sw, bias, residual=res, act=act, out_dtype=out, want_z=True)
        want_z = z64 + bias.double()
        ez = (K / 32 + 140) * U * size + 4 * U * bias.double().abs()
        if out == BF16 and T > 8:
            ez = ez + 2.0 ** -10 * size
        assert torch.all((z.double() - want_z).abs() <= ez + HALF[out] * (want_z.abs() + ez))
        if out == BF16:  # far less than the bound on the whole: a tenth of a step in the mean
            err = (z.double() - want_z).square().mean().sqrt()
            assert float(err) <= 1.1 * HALF[out] / 3 ** 0.5 * float(want_z.square().mean().sqrt())
        f = torch.from_numpy(bo.act(f64(want_z), act)).cuda()
        want = f + res.double()
        fast = 0.0 if act == "none" else 16 * U if out == F32 else 2.0 ** -12
        tol = 1.13 * ez + fast * (want_z.abs() + f.abs()) + 2 * U * (f.abs() + res.double().abs())
        assert torch.all((y.double() - want).abs() <= tol + HALF[out] * (want.abs() + tol) + 1e-30)


def test_training_step(gpu_lib):
    """y, dx and the weight's gradient of one layer, all in blocks, against the fp64 products
    of the numbers that the codes stand for."""
    T, N, K = 777, 272, 400
    x, w, dy = uneven(T, K, BF16, 1), uneven(N, K, F32, 2), uneven(T, N, BF16, 3)
    gw = randn((N, K), F32, 4)
    xq, xs, xqt, xst = pk.mem_quantize_blocks(x, want_cols=True)
    wq, ws, wqt, wst = pk.mem_quantize_blocks(w, tile=True, want_cols=True)
    dq, ds, dqt, dst = pk.mem_quantize_blocks(dy, want_cols=True)
    y, _ = pk.mem_linear_blocks(xq, wq, xs, ws, out_dtype=F32)
    dx, _ = pk.mem_linear_blocks(dq, wqt, ds, wst, out_dtype=F32)
    before = gw.double()
    g, _ = pk.mem_linear_blocks(dqt, xqt, dst, xst, residual=gw, y_out=gw, out_dtype=F32)
    assert g is gw
    val = lambda q, s, rows: q.double() * spread(s.double(), rows, q.shape[0], q.shape[1])  # noqa: E731
    for got, a, b, add in ((y, val(xq, xs, 1), val(wq, ws, 128), 0), (dx, val(dq, ds, 1), val(wqt, wst, 128)[:, :N], 0),
                           (gw, val(dqt, dst, 1), val(xqt, xst, 1), before)):
        want, size = a @ b.t().contiguous() + add, a.abs() @ b.abs().t().contiguous()
        assert got.shape == want.shape
        assert torch.all((got.double() - want).abs() <= (a.shape[1] / 32 + 140) * U * size + 2 * U * want.abs())


def test_no_rows(gpu_lib):
    x = torch.empty((0, 64), dtype=BF16, device="cuda")
    q, s, qt, st = pk.mem_quantize_blocks(x, want_cols=True)
    assert q.shape == (0, 64) and s.shape == (1, 0) and qt.shape == (64, 0) and st.shape == (0, 64)
    w, sw, _, _ = pk.mem_quantize_blocks(randn((24, 64), BF16, 1))
    y, _ = pk.mem_linear_blocks(q, w, s, sw)
    assert y.shape == (0, 24)
