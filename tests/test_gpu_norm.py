"""mem_rmsnorm, its backward and mem_quantize_rows against the fp64 oracle.

Tolerances, from counting roundings of u = 2^-24 (fp32) and half a step of the
stored type (bf16 2^-8, e4m3 2^-4 relative or 2^-10 of the grid's unit):
the mean square is a chain of at most 64 fused adds per lane, 6 exchanges, 3
joins, a division and an addition: 76 u, half of that in rstd with 3 u for
root and division; with two products y is within 43 u < 64 u = 2^-18."""
import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk
from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

Y = 2.0 ** -18
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
# T, D: one element group, odd row counts, every row width class and its edges
SHAPES = [(1, 8), (3, 64), (5, 200), (257, 512), (4, 520), (130, 1024), (9, 2048), (33, 2056), (2, 4096),
          (7, 4104), (3, 8192)]
DTS = [torch.float32, torch.bfloat16]


def f64(t):
    return t.detach().cpu().double().numpy()


def _x(T, D, dt, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, D), generator=g) * scale
    if T > 2:
        x[1] = 0          # a row of zeros
        x[2] = 0
        x[2, D // 2] = 1e4  # one element only
    return x.to(dt)


@pytest.mark.parametrize("dt", DTS, ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D", SHAPES + [(2, 16384)])
def test_norm(gpu_lib, T, D, dt):
    if dt == torch.float32 and D > 8192:
        D = 8184
    x, r = _x(T, D, dt, 1), _x(T, D, dt, 2, 3.0)
    w = (1 + 0.1 * torch.randn(D, generator=torch.Generator().manual_seed(3))).to(dt)
    for res in (None, r):
        for weight in (None, w):
            y, h, s = pk.mem_rmsnorm(x.cuda(), None if weight is None else w.cuda(),
                                     None if res is None else r.cuda(), 1e-5)
            assert s is None and (h is None) == (res is None)
            hh = x if res is None else (x.float() + r.float()).to(dt)
            if res is not None:
                assert torch.equal(h.cpu(), hh)
            want = bo.rmsnorm(f64(hh), 1.0 if weight is None else f64(w), 1e-5)
            assert np.all(np.abs(f64(y) - want) <= (Y + HALF[dt]) * np.abs(want) + 1e-44)


@pytest.mark.parametrize("dt", DTS, ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D", SHAPES)
def test_norm_in_8_bits(gpu_lib, T, D, dt):
    x, r = _x(T, D, dt, 4), _x(T, D, dt, 5)
    w = (1 + 0.1 * torch.randn(D, generator=torch.Generator().manual_seed(6))).to(dt)
    q, h, s = pk.mem_rmsnorm(x.cuda(), w.cuda(), r.cuda(), 1e-5, quantize=True)
    assert q.dtype == torch.float8_e4m3fn and s.shape == (T,)
    want = bo.rmsnorm(f64(h), f64(w), 1e-5)
    _, sw = bo.quantize_rows(want)
    s = f64(s)
    assert np.all(np.abs(s - sw) <= Y * sw)
    err = np.abs(f64(q) * s[:, None] - want)
    assert np.all(err <= (2.0 ** -4 + 2 * Y) * np.abs(want) + 2.0 ** -10 * s[:, None])
    assert np.all(np.abs(f64(q)).max(-1)[want.any(-1)] == 448)


def test_norm_eps_zero_and_tiny(gpu_lib):
    x = torch.zeros(3, 64)
    x[1] = 1e-18
    x[2, 0] = 1e-30  # its square is 0 in fp32: so is the row
    y, _, _ = pk.mem_rmsnorm(x.cuda(), eps=0.0)
    assert not y[0].any() and not y[2].any()
    assert torch.allclose(y[1].cpu(), torch.ones(64), rtol=1e-5)
    dx, gw = pk.mem_rmsnorm_backward(torch.ones(3, 64).cuda(), x.cuda(), eps=0.0)
    assert not dx[0].any() and torch.isfinite(gw).all()
    q, s = pk.mem_quantize_rows(x.cuda())
    assert not q[0].float().any() and float(s[0]) == 2.0 ** -126


def test_norm_and_gradient_in_place(gpu_lib):
    x, r = _x(70, 1032, torch.bfloat16, 7).cuda(), _x(70, 1032, torch.bfloat16, 8).cuda()
    y, h, _ = pk.mem_rmsnorm(x, None, r)
    for into in (x.clone(), r.clone()):
        a, b = (into, r) if torch.equal(into, x) else (x, into)
        y2, h2, _ = pk.mem_rmsnorm(a, None, b, sum_out=into)
        assert h2 is into and torch.equal(h2, h) and torch.equal(y2, y)
    dy = _x(70, 1032, torch.bfloat16, 9).cuda()
    want, _ = pk.mem_rmsnorm_backward(dy, h, dsum=x)
    for name in ("dy", "h", "dsum"):
        a = dict(dy=dy.clone(), h=h.clone(), dsum=x.clone())
        got, _ = pk.mem_rmsnorm_backward(a["dy"], a["h"], dsum=a["dsum"], dx=a[name])
        assert torch.equal(got, want), name


@pytest.mark.parametrize("dt", DTS, ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D", SHAPES + [(2500, 1024)])
def test_norm_backward(gpu_lib, T, D, dt):
    h, dy, ds = _x(T, D, dt, 11, 2.0), _x(T, D, dt, 12), _x(T, D, dt, 13)
    w = (1 + 0.1 * torch.randn(D, generator=torch.Generator().manual_seed(14))).to(dt)
    g0 = torch.randn(D, generator=torch.Generator().manual_seed(15))
    for dsum in (None, ds):
        gw = g0.cuda()
        dx, got = pk.mem_rmsnorm_backward(dy.cuda(), h.cuda(), w.cuda(), 1e-5,
                                          dsum=None if dsum is None else ds.cuda(), grad_weight=gw)
        assert got is gw
        wx, ww = bo.rmsnorm_backward(f64(dy), f64(h), f64(w), 1e-5, None if dsum is None else f64(ds))
        # each of the two terms carries at most 128 u: both sums of the row,
        # rstd twice, four products and the difference
        hh = f64(h)
        rstd = 1 / np.sqrt((hh * hh).mean(-1, keepdims=True) + 1e-5)
        g, xh = np.abs(f64(dy) * f64(w)), np.abs(hh) * rstd
        size = rstd * (g + xh * (g * xh).mean(-1, keepdims=True))
        assert np.all(np.abs(f64(dx) - wx) <= 128 * 2.0 ** -24 * size + (HALF[dt] + 2.0 ** -23) * np.abs(wx))
        # rows in chains of T / 2048 + 1, 4 waves, 64 parts, 8 groups, the sum itself, and 43 u of each xh
        terms = (np.abs(f64(dy)) * xh).sum(0)
        assert np.all(np.abs(f64(gw) - g0.double().numpy() - ww) <= 128 * 2.0 ** -24 * (terms + g0.abs().numpy()))
        again, _ = pk.mem_rmsnorm_backward(dy.cuda(), h.cuda(), w.cuda(), 1e-5, grad_weight=g0.cuda())
        assert torch.equal(_, got)
    only, none = pk.mem_rmsnorm_backward(dy.cuda(), h.cuda(), w.cuda(), 1e-5, want_grad_weight=False)
    assert none is None and torch.equal(only, again)


@pytest.mark.parametrize("dt", DTS, ids=["f32", "bf16"])
@pytest.mark.parametrize("R,C", [(1, 8), (5, 264), (100, 2048), (3, 4104)])
def test_quantize_rows(gpu_lib, R, C, dt):
    x = _x(R, C, dt, 21, 0.02)
    q, s = pk.mem_quantize_rows(x.cuda())
    sw = np.maximum(np.abs(f64(x)).max(-1) / 448, 2.0 ** -126)
    s, v = f64(s), f64(x)
    assert np.all(np.abs(s - sw) <= 2.0 ** -22 * sw)
    assert np.all(np.abs(f64(q) * s[:, None] - v) <= (2.0 ** -4 + 2.0 ** -21) * np.abs(v) + 2.0 ** -10 * s[:, None])


def test_empty_and_refusals(gpu_lib):
    x = torch.zeros((0, 64), device="cuda")
    y, _, _ = pk.mem_rmsnorm(x)
    assert y.shape == (0, 64)
    dx, gw = pk.mem_rmsnorm_backward(x, x)
    assert dx.shape == (0, 64) and not gw.any()
    x = torch.zeros((4, 64), device="cuda")
    for bad in (dict(weight=x[0].bfloat16()), dict(residual=x[:2]), dict(y_out=x[:3]), dict(sum_out=x.t(), residual=x)):
        with pytest.raises(ValueError):
            pk.mem_rmsnorm(x, **bad)
    with pytest.raises(ValueError):
        pk.mem_rmsnorm(x.t())
    with pytest.raises(TypeError):
        pk.mem_rmsnorm(x.half())
    with pytest.raises(pk.PkmemError):
        pk.mem_rmsnorm(x[:, :4].contiguous())
    with pytest.raises(ValueError):
        pk.mem_rmsnorm_backward(x, x, grad_weight=torch.zeros(63, device="cuda"))
    with pytest.raises(ValueError):
        pk.mem_rmsnorm_backward(x, x, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dt", DTS, ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(1, 8), (33, 2056), (257, 512), (3, 8192)])
def test_norm_in_place(gpu_lib, T, D, dt):
    x, r = _x(T, D, dt, 11).cuda(), _x(T, D, dt, 12).cuda()
    w = torch.linspace(0.5, 1.5, D).to(dt).cuda()
    want, _, _ = pk.mem_rmsnorm(x, w)
    both, h, _ = pk.mem_rmsnorm(x, w, r)
    a = x.clone()
    assert torch.equal(pk.mem_rmsnorm(a, w, y_out=a)[0], want)
    b, c = x.clone(), r.clone()
    pk.mem_rmsnorm(b, w, c, sum_out=b, y_out=c)
    assert torch.equal(b, h) and torch.equal(c, both)


def test_outputs_over_inputs_are_refused(gpu_lib):
    x = torch.zeros((4, 64), device="cuda")
    with pytest.raises(pk.PkmemError):
        pk.mem_rmsnorm(x, quantize=True, y_out=x.view(torch.float8_e4m3fn).view(-1)[:256].view(4, 64))
    with pytest.raises(pk.PkmemError):
        pk.mem_quantize_rows(x, q_out=x.view(torch.float8_e4m3fn).view(-1)[:256].view(4, 64))
    g, m, v = (torch.zeros_like(x) for _ in range(3))
    with pytest.raises(pk.PkmemError):  # a parameter listed twice
        pk.mem_adamw([x, x], [g, g], [m, m.clone()], [v, v.clone()], lr=1e-3, step=1)
    with pytest.raises(pk.PkmemError):  # views that share an element
        f = x.view(-1)
        cut = lambda t: [t.clone().view(-1)[:100], t.clone().view(-1)[:157]]  # noqa: E731
        pk.mem_adamw([f[:100], f[99:]], cut(g), cut(m), cut(v), lr=1e-3, step=1)
