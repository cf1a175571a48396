"""Pins of the block oracle's layer norm, gated part and 8-bit blocks: torch's layer norm
and autograd in 64 bits, central differences, closed forms, blocks by hand."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo


@pytest.mark.parametrize("eps", [1e-5, 0.1])
def test_layernorm_against_torch(eps):
    rng = np.random.default_rng(1)
    h, dy = rng.standard_normal((5, 24)) * 3 + 1, rng.standard_normal((5, 24))
    w, b = rng.standard_normal(24), rng.standard_normal(24)
    t = [torch.from_numpy(v).requires_grad_() for v in (h, w, b)]
    y = torch.nn.functional.layer_norm(t[0], (24,), t[1], t[2], eps)
    (y * torch.from_numpy(dy)).sum().backward()
    assert np.allclose(bo.layernorm(h, w, b, eps), y.detach().numpy(), rtol=1e-12, atol=1e-12)
    for got, want in zip(bo.layernorm_backward(dy, h, w, eps), t):
        assert np.allclose(got, want.grad.numpy(), rtol=1e-10, atol=1e-10)
    dsum = rng.standard_normal(h.shape)
    assert np.allclose(bo.layernorm_backward(dy, h, w, eps, dsum)[0] - dsum, t[0].grad.numpy(), atol=1e-10)


def test_layernorm_closed_forms():
    h = np.array([[1.0, 2, 3, 4], [7, 7, 7, 7]])
    y = bo.layernorm(h, np.ones(4), np.zeros(4), 0.0)
    assert np.allclose(y[0], np.array([-3, -1, 1, 3]) / np.sqrt(5)) and np.all(y[1] == 0)
    assert np.all(bo.layernorm(h, np.ones(4), np.arange(4.0), 0.0)[1] == np.arange(4))


@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu"])
def test_glu_gradients(name):
    rng = np.random.default_rng(2)
    x, w, b, dy = rng.standard_normal((4, 6)), rng.standard_normal((10, 6)), rng.standard_normal(10), rng.standard_normal((4, 5))
    y, z = bo.glu(x, w, b, name)
    assert y.shape == (4, 5) and np.allclose(y, bo.act(x @ w[:5].T + b[:5], name) * (x @ w[5:].T + b[5:]))
    dz, step = bo.glu_backward(dy, z, name), 1e-6
    for at in [(0, 0), (1, 4), (2, 5), (3, 9)]:
        f = []
        for s in (step, -step):
            v = z.copy()
            v[at] += s
            f.append((dy * bo.act(v[:, :5], name) * v[:, 5:]).sum())
        assert abs((f[0] - f[1]) / (2 * step) - dz[at]) < 1e-7


def test_blocks_by_hand():
    x = np.zeros((3, 136))
    x[0, 0], x[0, 5] = 448.0, 1.0625     # scale 1: a tie between 1 and 1.125, to the even 1
    x[1, 0], x[1, 127], x[1, 128] = -3.5, 7.0, 2.0 ** -140  # scale 2^-6; then below 2^-126
    q, each, s = bo.quantize_blocks(x, 1)
    assert s.shape == (2, 3)
    assert s[0, 0] == 1 and s[0, 1] == 2.0 ** -6 and s[0, 2] == s[1, 0] == s[1, 1] == 2.0 ** -126
    assert q[0, 5] == 1 and q[1, 0] == -224 and q[1, 127] == 448 and q[1, 128] == 0 and np.all(q[2] == 0)
    assert each[1, 127] == 2.0 ** -6 and each[1, 128] == 2.0 ** -126
    q, each, s = bo.quantize_blocks(x, 128)
    assert s.shape == (2, 1) and s[0, 0] == 1 and q[1, 127] == 7 and np.all(each[:, :128] == 1)


def test_blocks_round_to_nearest():
    x = np.random.default_rng(3).standard_normal((40, 300)) * np.exp(np.random.default_rng(4).standard_normal((40, 300)) * 3)
    for rows in (1, 128):
        q, each, _ = bo.quantize_blocks(x, rows)
        grid = bo.e4m3_values()
        grid = grid[np.isfinite(grid)]
        v = x / each
        best = np.abs(v[..., None] - grid).min(-1)
        assert np.all(np.abs(q - v) <= best + 1e-12) and np.abs(q).max() == 448
