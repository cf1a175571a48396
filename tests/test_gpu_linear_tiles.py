"""Every kernel that the projections' rules can choose (operand layout, type, tile, k
split or not) with ragged rows, columns and k, on whole numbers: sums are exact in any
order, so results have to be equal.  test_linear_plan.py checks on the host that these
sizes reach every one of them."""
import pytest
import torch

import paper_2412_09764_amd as pk
from tests.test_gpu_linear import BF16, E4M3, F32, NAMES, exact_mm, ints

pytestmark = pytest.mark.gpu

# T, N, and the k of a fraction of a stage (whole groups of waves without work), of a few
# stages and of many with a ragged end
FORWARD = [(T, N, K) for T, N in ((5, 1048), (40, 72), (333, 1096), (1000, 1032), (1800, 1992), (2000, 2056), (4100, 1032), (6500, 2056))
           for K in (16, 80, 400)]
# dx and grad_w: T, N, K
BACKWARD = [(300, 40, 200), (333, 16, 1096), (1000, 80, 1032), (2000, 16, 2056), (2000, 144, 2056), (4100, 80, 1032),
            (6500, 48, 2056),  # dx
            (5, 264, 3360), (777, 520, 1720), (32384, 528, 72), (24451, 72, 352),  # grad_w in 128-wide tiles
            (3, 3248, 1160), (100, 2056, 2056), (16155, 1392, 136), (20354, 336, 336),  # 256
            (2887, 8, 8), (967, 8, 8), (3000, 24, 40),  # 32
            (1, 2752, 72), (70, 1000, 264), (4014, 272, 8), (4068, 72, 80)]  # 64


@pytest.mark.parametrize("dt", [F32, BF16, E4M3], ids=NAMES.get)
@pytest.mark.parametrize("T,N,K", FORWARD)
def test_forward(gpu_lib, T, N, K, dt):
    x, w = ints((T, K), dt, 1), ints((N, K), dt, 2)
    kw, scale = {}, 1.0
    if dt == E4M3:
        sx, sw = (2.0 ** torch.arange(n, device="cuda").remainder(5).sub(2) for n in (T, N))
        kw, scale = dict(x_scale=sx.float(), w_scale=sw.float()), sx.double()[:, None] * sw.double()
    b, r = ints((N,), F32, 3), ints((T, N), F32, 4)
    y, z = pk.mem_linear(x, w, b, residual=r, act="relu", out_dtype=F32, want_z=True, **kw)
    want = exact_mm(x.float(), w.float()) * scale + b.double()
    assert torch.equal(z.double(), want)
    assert torch.equal(y.double(), want.clamp(min=0) + r.double())
    if dt != F32:
        y, none = pk.mem_linear(x, w, out_dtype=BF16, **kw)
        assert none is None and torch.equal(y, (want - b.double()).to(BF16))


@pytest.mark.parametrize("dt", [F32, BF16], ids=NAMES.get)
@pytest.mark.parametrize("T,N,K", BACKWARD)
def test_backward(gpu_lib, T, N, K, dt):
    dz, x, w, add = ints((T, N), dt, 1, 2), ints((T, K), dt, 2, 2), ints((N, K), dt, 3, 2), ints((T, K), dt, 4)
    gw, gb = ints((N, K), F32, 5), ints((N,), F32, 6)
    want_w = exact_mm(dz.float().t().contiguous(), x.float().t().contiguous()) + gw.double()
    want_b = dz.double().sum(0) + gb.double()
    dx, _, _ = pk.mem_linear_backward(dz, x, w, dx_add=add, grad_w=gw, grad_bias=gb)
    assert torch.equal(gw.double(), want_w) and torch.equal(gb.double(), want_b)
    assert torch.equal(dx, (exact_mm(dz.float(), w.float().t().contiguous()) + add.double()).to(dt))
