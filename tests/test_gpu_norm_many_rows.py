"""More rows than one launch holds (2^32 threads: 2^26 rows of one wave each, 2^24 of
four): the rows at the edges equal those rows alone."""
import pytest
import torch

import paper_2412_09764_amd as pk

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def u8(t):
    return t.contiguous().view(torch.uint8)


@pytest.mark.parametrize("T", [(1 << 25) + 1, (1 << 26) + 5])
def test_one_wave_a_row(gpu_lib, T):
    D = 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randn((T, D), generator=g, device="cuda", dtype=BF16) for _ in range(2))
    w = torch.linspace(0.5, 2.0, D, device="cuda").to(BF16)
    edges = [slice(0, 9), slice((1 << 25) - 6, (1 << 25) + 1), slice(T - 7, T)]
    y, h, _ = pk.mem_rmsnorm(x, w, r)
    q, _, s = pk.mem_rmsnorm(x, w, r, quantize=True, want_sum=False)
    c, sc = pk.mem_quantize_rows(x)
    for at in edges:
        a, b = x[at].clone(), r[at].clone()
        y1, h1, _ = pk.mem_rmsnorm(a, w, b)
        assert torch.equal(y[at], y1) and torch.equal(h[at], h1)
        q1, _, s1 = pk.mem_rmsnorm(a, w, b, quantize=True)
        assert torch.equal(u8(q[at]), u8(q1)) and torch.equal(s[at], s1)
        c1, sc1 = pk.mem_quantize_rows(a)
        assert torch.equal(u8(c[at]), u8(c1)) and torch.equal(sc[at], sc1)
    # no row between was left out: each mean square is 1
    pk.mem_rmsnorm(x, y_out=x)
    assert float(x.float().square().mean(-1).min()) > 0.98


def test_four_waves_a_row_in_place(gpu_lib):
    T, D = (1 << 24) + 3, 4104
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < T * D * 2 + (8 << 30):
        pytest.skip("138 GB of rows do not fit beside what is on the card")
    x = torch.empty((T, D), dtype=BF16, device="cuda")
    x[0], x[(1 << 23) - 2:(1 << 23) + 2], x[-5:] = 3, 5, 7
    x[100:200] = 0
    pk.mem_rmsnorm(x, y_out=x)
    for at in (slice(0, 1), slice((1 << 23) - 2, (1 << 23) + 2), slice(T - 5, T)):
        assert torch.all(x[at] == 1)
    assert not x[100:200].any()
