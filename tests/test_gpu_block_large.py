"""Offsets past 32 bits: outputs, rows and tables of more than 2^31 or 2^32 elements
through the norm, the projections and the optimizer.  Whole numbers make the products
exact, so that the last rows of a large call equal those rows alone."""
import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk
from tests.test_gpu_adamw import HYPER, check, values

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def ints(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(BF16)


def test_linear_of_many_rows(gpu_lib):
    T, N, K = (1 << 20) + 77, 2056, 16
    x, w = ints((T, K), 1), ints((N, K), 2)
    y, _ = pk.mem_linear(x, w)
    assert y.numel() > 1 << 31
    for at in (slice(0, 100), slice(T - 100, T)):
        assert torch.equal(y[at].float(), x[at].float() @ w.float().t().contiguous())
    # backward: dz of the same size; grad_w's sums stay below 2^24
    dx, gw, gb = pk.mem_linear_backward(y, x, w)
    want = y[-100:].float() @ w.float()
    assert torch.equal(dx[-100:], want.to(BF16))
    ref = torch.zeros((N, K), dtype=torch.float64, device="cuda")
    for a in range(0, T, 1 << 17):
        ref += y[a:a + (1 << 17)].double().t().contiguous() @ x[a:a + (1 << 17)].double()
    assert float((gw.double() - ref).abs().max()) <= 2.0 ** -20 * float(ref.abs().max())


def test_norm_of_many_rows(gpu_lib):
    T, D = (1 << 20) + 3, 2056
    x = ints((T, D), 3)
    y, _, _ = pk.mem_rmsnorm(x)
    for at in (slice(0, 50), slice(T - 50, T)):
        assert torch.equal(y[at], pk.mem_rmsnorm(x[at].contiguous())[0])
    q, s = pk.mem_quantize_rows(x)
    tail = pk.mem_quantize_rows(x[-50:].contiguous())
    assert torch.equal(q[-50:].view(torch.uint8), tail[0].view(torch.uint8)) and torch.equal(s[-50:], tail[1])
    dx, _ = pk.mem_rmsnorm_backward(y, x)
    assert torch.equal(dx[-50:], pk.mem_rmsnorm_backward(y[-50:].contiguous(), x[-50:].contiguous())[0])


def test_adamw_on_a_large_table(gpu_lib):
    """Places past 2^32 reach the hash with their upper half, and rows there are found."""
    N, D = (1 << 21) + 5, 2048
    p = torch.full((N, D), 0.02, dtype=BF16, device="cuda")
    m, v, sm, sv = pk.mem_adamw_state(p, 8)
    assert p.numel() > 1 << 32
    rows = torch.tensor([0, 7, (1 << 21) - 1, 1 << 21, N - 1])
    g = torch.randn((5, D), generator=torch.Generator().manual_seed(5)) * 1e-3
    i = rows.cuda()
    p0 = p[i].cpu().double().numpy()
    pk.mem_adamw_rows(p, i, g.cuda(), m, v, step=1, seed=6, exp_avg_scale=sm, exp_avg_sq_scale=sv, **HYPER)
    pick = lambda s: s.view(N, -1)[i].reshape(-1)  # noqa: E731
    u8 = lambda t: t.view(torch.uint8)[i].view(t.dtype)  # noqa: E731
    zero = np.zeros_like(p0)
    check((p0, (zero, zero)), (p[i], u8(m), u8(v), pick(sm), pick(sv)), g.double().numpy(), 1, HYPER, 8,
          places=rows.numpy()[:, None] * D + np.arange(D), seed=6)
    assert torch.equal(p[1], p[2]) and torch.equal(p[1], p[N - 2])  # rows without a gradient
    # the dense step on the same table, its last elements against the oracle
    gd = torch.zeros((N, D), dtype=BF16, device="cuda")
    gd[-1] = g[4].to(BF16).cuda()
    last = p[-1:].cpu().double().numpy(), values(m[-1:], v[-1:], sm[-16:], sv[-16:])
    pk.mem_adamw([p], [gd], [m], [v], step=2, seed=6, exp_avg_scales=[sm], exp_avg_sq_scales=[sv], **HYPER)
    check(last, (p[-1:], m[-1:], v[-1:], sm[-16:], sv[-16:]), gd[-1:].cpu().double().numpy(), 2, HYPER, 8,
          places=(N - 1) * D + np.arange(D), seed=6)
