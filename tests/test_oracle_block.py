"""Pins of the block oracle: gradients against central differences, the e4m3
grid against torch's conversion, the random rounding against its expectation."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo


def _diff(f, x, at, h=1e-6):
    a, b = x.copy(), x.copy()
    a[at] += h
    b[at] -= h
    return (f(a) - f(b)) / (2 * h)


def test_e4m3_grid_matches_torch():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(bo.e4m3_values(), codes, equal_nan=True)
    x = np.random.default_rng(0).standard_normal(20000) * 60
    x = np.clip(np.concatenate([x, x / 4096, (bo._POS[1:] + bo._POS[:-1]) / 2]), -448, 448)
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(bo.to_e4m3(x.astype(float)), want)


@pytest.mark.parametrize("eps", [1e-5, 0.0])
def test_rmsnorm_gradients(eps):
    rng = np.random.default_rng(1)
    h, dy, w = rng.standard_normal((3, 16)), rng.standard_normal((3, 16)), rng.standard_normal(16)
    dx, gw = bo.rmsnorm_backward(dy, h, w, eps)
    for at in [(0, 0), (1, 7), (2, 15)]:
        assert abs(_diff(lambda v: (dy * bo.rmsnorm(v, w, eps)).sum(), h, at) - dx[at]) < 1e-7
    for at in [(0,), (9,)]:
        assert abs(_diff(lambda v: (dy * bo.rmsnorm(h, v, eps)).sum(), w, at) - gw[at]) < 1e-7
    assert np.all(bo.rmsnorm(np.zeros((2, 8)), np.ones(8), 0.0) == 0)
    # scaling a row leaves its norm alone (eps = 0): dx is orthogonal to the row
    if eps == 0:
        assert np.abs((dx * h).sum(-1)).max() < 1e-12


@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu"])
def test_linear_gradients(name):
    rng = np.random.default_rng(2)
    x, w, b = rng.standard_normal((4, 6)), rng.standard_normal((5, 6)), rng.standard_normal(5)
    res, dy = rng.standard_normal((4, 5)), rng.standard_normal((4, 5))
    _, z = bo.linear(x, w, b, res, name)
    dz = dy * bo.act_grad(z, name)
    dx, gw, gb = bo.linear_backward(dz, x, w)
    f = lambda x_, w_, b_: (dy * bo.linear(x_, w_, b_, res, name)[0]).sum()  # noqa: E731
    assert abs(_diff(lambda v: f(v, w, b), x, (1, 2)) - dx[1, 2]) < 1e-7
    assert abs(_diff(lambda v: f(x, v, b), w, (3, 4)) - gw[3, 4]) < 1e-7
    assert abs(_diff(lambda v: f(x, w, v), b, (2,)) - gb[2]) < 1e-7


def test_adamw_first_step_is_the_sign():
    """Without decay and with zero states the first step is lr * g / (|g| + eps)."""
    g = np.array([3.0, -0.5, 1e-3])
    p, m, v = bo.adamw(np.zeros(3), g, np.zeros(3), np.zeros(3), 0.1, (0.9, 0.999), 1e-8, 0.0, 1)
    assert np.allclose(p, -0.1 * g / (np.abs(g) + 1e-8), rtol=1e-12)
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 1e-3 * g * g)


def test_random_bits_are_even():
    """Each of the 32 bits of 2^18 elements is set half of the time, for each step
    and tensor and across two of them: off by at most 6 standard deviations
    (sqrt(2^18) / 2 = 256 of a count of 2^17)."""
    n = 1 << 18
    at = np.arange(n) + (1 << 32) - n // 2  # places on both sides of 2^32
    a = bo.random_bits(at, 12345, 1)
    others = [bo.random_bits(at, 12345, 2), bo.random_bits(at, 12345, 1, tensor=1),
              bo.random_bits(at, 12346, 1), bo.random_bits(at + 1, 12345, 1)]
    for b in range(32):
        assert abs(int((a >> b & 1).sum()) - n // 2) < 6 * 256
        for o in others:
            assert abs(int(((a ^ o) >> b & 1).sum()) - n // 2) < 6 * 256


def test_random_rounding_keeps_the_mean():
    """The mean of 4096 elements rounded at random differs from the value by at most
    6 standard deviations of a step's coin (step * sqrt(1/4 / 4096)) plus half of a
    random bit's weight (step / 4096 or / 256)."""
    n = 4096
    for val, t in [(0.7321, 3), (0.0101, 4), (0.0004, 5)]:
        x = np.full(n, val)
        x[::128] = 1.0  # the largest of every block
        bits = bo.random_bits(np.arange(n), 99, t)
        for width, b in ((12, bits >> 12 & 0xFFF), (8, bits >> 24 & 0xFF)):
            s, lo, hi, up, _ = bo.state_up(x, b, width, False)
            got = np.where(up, hi, lo) * np.repeat(s, 128)
            keep = np.arange(n) % 128 != 0
            step = (hi - lo)[1] * s[0]
            assert abs(got[keep].mean() - val) <= step * (6 * 0.5 / np.sqrt(keep.sum()) + 0.5 / 2 ** width)
        lo, hi, up, _ = bo.bf16_up(x, bits)
        got = np.where(up, hi, lo)
        keep = np.arange(n) % 128 != 0
        step = (hi - lo)[1]
        assert abs(got[keep].mean() - val) <= step * (6 * 0.5 / np.sqrt(keep.sum()) + 0.5 / 4096)
