"""mem_layernorm and its backward against the fp64 oracle.

Tolerances, from counting roundings of u = 2^-24 (fp32) and half a step of the stored type
(bf16 2^-8).  A row's sum is a chain of at most 64 fused adds per lane, 6 exchanges and 2
joins: 72 u of the sum of its terms' sizes.  The first mean, summed from the differences to the
first element, is off by e <= u |mean| + 73 u mean|h - h_0| (by nothing where all are equal).  The variance (squares: all of
one sign) and with it rstd is within 72 u / 2 + 4 u where e is below the deviation; the
deviation from the first mean is one rounding of itself, and the mean's correction within
72 u of the mean deviation from it, which is at most one standard deviation and e: an error
of y of 45 u |xh w| + 75 u (1 + e rstd) |w|, and with the last product and sum 2 u (|y| + |b|).  In dx both means are within 75 u of the means of their terms' sizes, the
second one's factor xh as y: 50 u |g| + 80 u mean|g| + (50 + 130) u |xh| mean|g xh| +
80 u (mean|g xh| + |xh| mean|g|), all times rstd.  A column's sum over the rows is a chain of
T / 2048 + 1 (a wave's rows), 4, 16 and 32 more adds of terms that are within 45 u |dy xh| +
75 u |dy|."""
import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk
from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
DTS = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]
# T, D: one group of elements, odd numbers of rows, every class of widths and its edges
SHAPES = [(1, 8), (3, 64), (5, 200), (257, 512), (4, 520), (130, 1024), (9, 2048), (33, 2056), (2, 4096),
          (7, 4104), (3, 8192), (2, 16384)]


def f64(t):
    return t.detach().cpu().double().numpy()


def _rows(T, D, dt, seed, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, D), generator=g) * scale + shift
    if T > 2:
        x[1] = 3.0 if seed == 1 else 0.0  # a constant row
        x[2] = 0
        x[2, D // 2] = 1e4  # one element alone
    return x.to(dt)


def _widths(D, dt):
    return min(D, 8184) if dt == torch.float32 else D


def first_mean(h, eps):
    """e rstd"""
    m = h.mean(-1, keepdims=True)
    e = U * np.abs(m) * (h != h[:, :1]).any(-1, keepdims=True) + 73 * U * np.abs(h - h[:, :1]).mean(-1, keepdims=True)
    var = ((h - m) ** 2).mean(-1, keepdims=True) + eps
    return e / np.sqrt(np.where(var == 0, 1, var))


def check_y(y, h, w, b, eps, dt):
    want = bo.layernorm(h, w, b, eps)
    xh = np.abs(bo.layernorm(h, 1.0, 0.0, eps))
    tol = U * (45 * xh * np.abs(w) + 75 * (1 + first_mean(h, eps)) * np.abs(w) + 2 * (np.abs(want) + np.abs(b))) + HALF[dt] * np.abs(want)
    assert np.all(np.abs(f64(y) - want) <= tol + 1e-44)


def check_backward(got, dy, h, w, eps, dsum, gw0, gb0, dt):
    dx, gw, gb = got
    T = len(h)
    want, want_w, want_b = bo.layernorm_backward(dy, h, w, eps, dsum)
    d = h - h.mean(-1, keepdims=True)
    var = (d * d).mean(-1, keepdims=True) + eps
    rstd = np.where(var == 0, 0, 1 / np.sqrt(np.where(var == 0, 1, var)))
    xh, g = np.abs(d * rstd), np.abs(dy * w)
    mg, mgx = g.mean(-1, keepdims=True), (g * xh).mean(-1, keepdims=True)
    assert np.all(first_mean(h, eps) < 1)
    tol = U * rstd * (50 * g + 80 * mg + 180 * xh * mgx + 80 * (mgx + xh * mg))
    add = 0 if dsum is None else np.abs(dsum)
    tol = tol + 2 * U * (np.abs(want) + add) + HALF[dt] * np.abs(want)
    assert np.all(np.abs(f64(dx) - want) <= tol + 1e-44)
    chain = T // 2048 + 1 + 4 + 16 + 32
    if gw is not None:
        size = (np.abs(dy) * xh).sum(0)
        err = U * ((chain + 45) * size + 75 * np.abs(dy).sum(0) + 2 * np.abs(want_w + gw0))
        assert np.all(np.abs(f64(gw) - want_w - gw0) <= err)
    if gb is not None:
        assert np.all(np.abs(f64(gb) - want_b - gb0) <= U * (chain * np.abs(dy).sum(0) + 2 * np.abs(want_b + gb0)))


@pytest.mark.parametrize("dt", DTS, ids=IDS)
@pytest.mark.parametrize("T,D", SHAPES)
def test_forward(gpu_lib, T, D, dt):
    D = _widths(D, dt)
    x, r = _rows(T, D, dt, 1), _rows(T, D, dt, 2, 3.0, 1.0)
    g = torch.Generator().manual_seed(3)
    w, b = (1 + 0.1 * torch.randn(D, generator=g)).to(dt), torch.randn(D, generator=g).to(dt)
    for res in (None, r):
        hh = x if res is None else (x.float() + r.float()).to(dt)
        for weight in (None, w):
            for bias in (None, b):
                y, h = pk.mem_layernorm(x.cuda(), *(None if t is None else t.cuda() for t in (weight, bias, res)), 1e-5)
                assert (h is None) == (res is None) and (h is None or torch.equal(h.cpu(), hh))
                check_y(y, f64(hh), 1.0 if weight is None else f64(w), 0.0 if bias is None else f64(b), 1e-5, dt)


@pytest.mark.parametrize("dt", DTS, ids=IDS)
@pytest.mark.parametrize("T,D", SHAPES + [(2500, 72), (5001, 264)])
def test_backward(gpu_lib, T, D, dt):
    D = _widths(D, dt)
    h, dy, ds = _rows(T, D, dt, 1, 2.0, 0.5), _rows(T, D, dt, 2), _rows(T, D, dt, 4)
    g = torch.Generator().manual_seed(3)
    w = (1 + 0.1 * torch.randn(D, generator=g)).to(dt)
    gw0, gb0 = torch.randn(D, generator=g), torch.randn(D, generator=g)
    for weight, dsum in ((None, None), (w, None), (w, ds)):
        gw, gb = gw0.cuda(), gb0.cuda()
        args = [t if t is None else t.cuda() for t in (dy, h, weight)]
        kw = dict(dsum=None if dsum is None else dsum.cuda(), eps=1e-5)
        got = pk.mem_layernorm_backward(*args, grad_weight=gw, grad_bias=gb, **kw)
        assert got[1] is gw and got[2] is gb
        check = [f64(dy), f64(h), 1.0 if weight is None else f64(w), 1e-5, None if dsum is None else f64(ds)]
        check_backward(got, *check, f64(gw0), f64(gb0), dt)
        # the same bits again, from zeros, one gradient alone, none
        two = pk.mem_layernorm_backward(*args, **kw)
        check_backward(two, *check, 0.0, 0.0, dt)
        for want in ((True, False), (False, True), (False, False)):
            one = pk.mem_layernorm_backward(*args, want_grad_weight=want[0], want_grad_bias=want[1], **kw)
            assert torch.equal(one[0], got[0])
            for i in (1, 2):
                assert torch.equal(one[i], two[i]) if want[i - 1] else one[i] is None


@pytest.mark.parametrize("dt", DTS, ids=IDS)
@pytest.mark.parametrize("D", [264, 8184])
def test_far_from_zero(gpu_lib, D, dt):
    """Rows whose mean is many times their deviation: the deviations keep their digits."""
    for shift in (100.0, 3e4, -1e6):
        h = _rows(6, D, dt, 5, 1.0, shift)
        ones, zeros = torch.ones(D, dtype=dt), torch.zeros(D, dtype=dt)
        y, _ = pk.mem_layernorm(h.cuda(), ones.cuda(), zeros.cuda(), eps=1e-5)
        check_y(y, f64(h), 1.0, 0.0, 1e-5, dt)
        dy = _rows(6, D, dt, 6)
        got = pk.mem_layernorm_backward(dy.cuda(), h.cuda(), ones.cuda(), 1e-5)
        check_backward(got, f64(dy), f64(h), 1.0, 1e-5, None, 0.0, 0.0, dt)


@pytest.mark.parametrize("dt", DTS, ids=IDS)
def test_constant_rows_and_extremes(gpu_lib, dt):
    D = 128
    h = torch.zeros((5, D))
    h[0] = 7.0
    h[1] = 3e38 if dt == torch.float32 else 2.9e38
    h[2] = torch.randn(D, generator=torch.Generator().manual_seed(1)) * 1e30
    h[3, 5] = float("nan")
    h[4] = torch.arange(D)
    h = h.to(dt).cuda()
    b = torch.arange(D).to(dt).cuda()
    y, _ = pk.mem_layernorm(h, None, b, eps=0.0)
    for row in (0, 1, 2):  # no deviation, or past the largest number: the bias alone
        assert torch.equal(y[row], b)
    assert torch.isnan(y[3]).all() and torch.isfinite(y[4]).all()
    dy = torch.ones((5, D), dtype=dt, device="cuda")
    dx, _, gb = pk.mem_layernorm_backward(dy, h, None, 0.0, dsum=dy)
    assert torch.equal(dx[:3], dy[:3]) and torch.isnan(dx[3]).all() and torch.equal(gb, torch.full_like(gb, 5.0))


@pytest.mark.parametrize("dt", DTS, ids=IDS)
@pytest.mark.parametrize("D", [1032, 8184])
def test_in_place(gpu_lib, D, dt):
    x, r, w = (_rows(9, D, dt, s).cuda() for s in (1, 2, 3))
    w = w[0].contiguous()
    y, h = pk.mem_layernorm(x, w, w, r)
    for into in ("x", "r"):
        a, c = x.clone(), r.clone()
        y2, h2 = pk.mem_layernorm(a, w, w, c, sum_out=a if into == "x" else c)
        assert torch.equal(y2, y) and torch.equal(h2, h) and h2.data_ptr() == (a if into == "x" else c).data_ptr()
        a, c = x.clone(), r.clone()
        y2, h2 = pk.mem_layernorm(a, w, w, c, y_out=a if into == "x" else c, want_sum=False)
        assert torch.equal(y2, y) and h2 is None
    s = torch.empty_like(x)
    assert torch.equal(pk.mem_layernorm(x, w, w, sum_out=s)[1], x)
    dx, gw, gb = pk.mem_layernorm_backward(x, h, w, dsum=r)
    for i in range(3):
        args = [x.clone(), h.clone(), r.clone()]
        got = pk.mem_layernorm_backward(args[0], args[1], w, dsum=args[2], dx=args[i])
        assert got[0] is args[i] and torch.equal(got[0], dx) and torch.equal(got[1], gw) and torch.equal(got[2], gb)


def test_no_rows(gpu_lib):
    x = torch.empty((0, 64), device="cuda")
    y, _ = pk.mem_layernorm(x)
    assert y.shape == (0, 64)
    gw = torch.ones(64, device="cuda")
    dx, got, _ = pk.mem_layernorm_backward(x, x, grad_weight=gw)
    assert dx.shape == (0, 64) and torch.equal(got, torch.ones_like(got))


@pytest.mark.parametrize("D,T", [(64, (1 << 25) + 9)])
def test_many_rows(gpu_lib, D, T):
    """More rows than a launch of four a workgroup holds."""
    x = torch.zeros((T, D), dtype=torch.bfloat16, device="cuda")
    x[:, 1::2] = 1.0
    x[-1] = torch.arange(D)
    y, _ = pk.mem_layernorm(x, eps=0.0)
    one = torch.ones(D, device="cuda", dtype=torch.bfloat16)
    one[0::2] = -1.0
    assert torch.equal(y[0], one) and torch.equal(y[T - 2], one)
    assert bool((y[:-1].view(torch.int64)[:, 0] == y[0].view(torch.int64)[0]).all())
    assert torch.equal(y[-1], pk.mem_layernorm(x[-1:].clone(), eps=0.0)[0][0])
