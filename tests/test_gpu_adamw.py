"""mem_adamw and mem_adamw_rows against the fp64 oracle.

Tolerances, in u = 2^-24 (one rounding of fp32): m is two products with
rounded constants and a sum, 5 u of its terms' sizes; v likewise with g^2, 6 u;
the root and the quotient add 8 u of the update, m's own error counts through
the quotient; p adds 3 u of itself and 4 u of the update.  States in 8 bits and
bf16 parameters are drawn by known bits: the result is the oracle's neighbour,
except where the decision lies within 2^-9 of a step of its border."""
import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk
from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HYPER = dict(lr=3e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)


def f64(t):
    return t.detach().cpu().double().numpy()


def make(shape, dt, bits, seed, gdt=torch.float32):
    g = torch.Generator().manual_seed(seed)
    p = (torch.randn(shape, generator=g) * 0.02).to(dt).cuda()
    gr = (torch.randn(shape, generator=g) * 1e-3).to(gdt).cuda()
    m, v, sm, sv = pk.mem_adamw_state(p, bits)
    return [p, gr, m, v, sm, sv]


def values(m, v, sm, sv):
    """States as fp64 (m, v)."""
    if sm is None:
        return f64(m), f64(v)
    n = m.numel()
    full = [np.repeat(f64(s), 128)[:n].reshape(m.shape) for s in (sm, sv)]
    return f64(m) * full[0], (f64(v) * full[1]) ** 2


def check(before, after, g, t, hyper, bits, places=None, tensor=0, seed=0):
    """before, after: (p, m, v, sm, sv) of one tensor as fp64 / tensors."""
    p0, (m0, v0) = before
    p1, m, v, sm, sv = after
    b1, b2 = hyper["betas"]
    wp, wm, wv = bo.adamw(p0, g, m0, v0, hyper["lr"], hyper["betas"], hyper["eps"], hyper["weight_decay"], t)
    am = b1 * np.abs(m0) + (1 - b1) * np.abs(g)
    den = np.sqrt(wv) / np.sqrt(1 - b2 ** t) + hyper["eps"]
    rate = hyper["lr"] / (1 - b1 ** t)
    tol = 4 * U * np.abs(p0) + rate * (5 * U * am + 16 * U * np.abs(wm)) / den
    h = bo.random_bits(np.arange(p0.size) if places is None else places, seed, t, tensor).reshape(p0.shape)
    if p1.dtype == torch.bfloat16:
        lo, hi, up, near = bo.bf16_up(wp, h)
        want = np.where(up, hi, lo)
        got = f64(p1)
        assert np.all((got == want) | ((got == lo) | (got == hi)) & (near <= 2.0 ** -9 + tol / np.maximum(np.abs(hi - lo), 1e-40)))
        assert np.mean(got != want) < 0.02
    else:
        assert np.all(np.abs(f64(p1) - wp) <= tol)
    if bits == 32:
        assert np.all(np.abs(f64(m) - wm) <= 5 * U * am)
        assert np.all(np.abs(f64(v) - wv) <= 6 * U * wv + 1e-44)
        return
    for q, s, x, b, width, nz in ((m, sm, wm, h >> 24 & 0xFF, 8, False), (v, sv, np.sqrt(wv), h >> 12 & 0xFFF, 12, True)):
        sw, lo, hi, up, near = bo.state_up(x, b, width, nz)
        # the largest of a block is within 5 u of its terms, the scale 2 u more
        size = np.repeat(sw, 128)[:x.size]
        assert np.all(np.abs(f64(s) - sw) <= 2.0 ** -20 * sw + 1e-44)
        got, want = f64(q).reshape(-1), np.where(up, hi, lo)
        err = (2.0 ** -18 * np.abs(want) + (5 * U * am.reshape(-1) if not nz else 0) / np.maximum(size, 1e-44))
        step = np.maximum(np.abs(hi - lo), 2.0 ** -9)
        # (both neighbours of the other side where the value itself is on the grid)
        ok = (got == want) | (np.abs(got - want) <= step * 1.01) & ((near <= 2.0 ** -9 + err / step) | (near >= 1 - 2.0 ** -9 - err / step))
        assert np.all(ok), (got[~ok][:4], want[~ok][:4], near[~ok][:4])
        assert np.mean(got != want) < 0.02


SIZES = [1, 7, 128, 129, 1000, 4096, (3, 5, 11), 100003]


@pytest.mark.parametrize("gdt", [torch.float32, torch.bfloat16], ids=["g32", "g16"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_adamw_steps(gpu_lib, dt, bits, gdt):
    ts = [make(s if isinstance(s, tuple) else (s,), dt, bits, i, gdt) for i, s in enumerate(SIZES)]
    for t in (1, 2, 3):
        before = [(f64(x[0]), values(*x[2:])) for x in ts]
        pk.mem_adamw(*[[x[j] for x in ts] for j in range(4)], step=t, seed=77, exp_avg_scales=[x[4] for x in ts],
                     exp_avg_sq_scales=[x[5] for x in ts], **HYPER)
        for i, (x, b) in enumerate(zip(ts, before)):
            check(b, (x[0], *x[2:]), f64(x[1]), t, HYPER, bits, tensor=i, seed=77)


def test_adamw_mixed_types_and_many(gpu_lib):
    """More tensors than one launch holds, of all types at once."""
    kinds = [(dt, bits, g) for dt in (torch.float32, torch.bfloat16) for bits in (32, 8)
             for g in (torch.float32, torch.bfloat16)]
    ts = [make((1 + 37 * i,), *kinds[i % 8][:2], i, kinds[i % 8][2]) for i in range(330)]
    before = [(f64(x[0]), values(*x[2:])) for x in ts]
    pk.mem_adamw(*[[x[j] for x in ts] for j in range(4)], step=5, seed=-3, exp_avg_scales=[x[4] for x in ts],
                 exp_avg_sq_scales=[x[5] for x in ts], **HYPER)
    for i in list(range(0, 330, 13)) + [329]:
        x = ts[i]
        check(before[i], (x[0], *x[2:]), f64(x[1]), 5, HYPER, kinds[i % 8][1], tensor=i, seed=(1 << 64) - 3)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_unaligned_tensors(gpu_lib, dt, bits):
    """Slices at odd offsets give what aligned copies give, and nothing around them moves."""
    n = 1001
    x = make((n,), dt, bits, 5)
    y = []
    for t in x[:4]:
        raw = torch.zeros(n + 16, dtype=t.dtype, device="cuda") if t.element_size() > 1 else \
            torch.zeros(n + 16, dtype=torch.uint8, device="cuda").view(t.dtype)
        raw[3:3 + n].view(torch.uint8 if t.element_size() == 1 else t.dtype).copy_(t.view(torch.uint8) if t.element_size() == 1 else t)
        y.append(raw)
    sm, sv = (None, None) if bits == 32 else (x[4].clone(), x[5].clone())
    pk.mem_adamw([x[0]], [x[1]], [x[2]], [x[3]], step=1, exp_avg_scales=[x[4]], exp_avg_sq_scales=[x[5]], **HYPER)
    pk.mem_adamw(*[[t[3:3 + n]] for t in y], step=1, exp_avg_scales=[sm], exp_avg_sq_scales=[sv], **HYPER)
    for a, b in zip((x[0], x[2], x[3]), (y[0], y[2], y[3])):
        raw = b.float()
        assert torch.equal(a.float(), raw[3:3 + n]) and not raw[:3].any() and not raw[3 + n:].any()


@pytest.mark.parametrize("bits", [32, 8])
def test_special_gradients(gpu_lib, bits):
    """A NaN or an infinity stays with its element; zeros leave zero states at zero."""
    x = make((512,), torch.float32, bits, 6)
    x[1][:] = 0
    x[1][5], x[1][140], x[1][300] = float("nan"), float("inf"), 1e-3
    p0 = x[0].clone()
    pk.mem_adamw(*[[t] for t in x[:4]], step=1, exp_avg_scales=[x[4]], exp_avg_sq_scales=[x[5]],
                 **{**HYPER, "weight_decay": 0.0})
    bad = torch.tensor([5, 140])
    keep = torch.ones(512, dtype=torch.bool)
    keep[bad] = False
    assert torch.isnan(x[0].cpu()[bad]).all() and torch.isnan(x[2].float().cpu()[5])
    assert torch.isfinite(x[0].cpu()[keep]).all() and torch.isfinite(x[2].float().cpu()[keep]).all()
    keep[300] = False
    assert torch.equal(x[0].cpu()[keep], p0.cpu()[keep])
    assert not x[2].float().cpu()[keep].any() and not x[3].float().cpu()[keep].any()


def test_grad_scale_and_device_scalars(gpu_lib):
    dev = torch.device("cuda")
    a, b, c = (make((3000,), torch.bfloat16, 8, 8) for _ in range(3))
    call = lambda x, g, **k: pk.mem_adamw([x[0]], [g], [x[2]], [x[3]], exp_avg_scales=[x[4]], exp_avg_sq_scales=[x[5]], seed=9,  # noqa: E731
                                          **{**HYPER, **k})
    for t in (1, 2, 3):
        call(a, a[1] * 0.5, step=t)
        call(b, b[1], step=t, grad_scale=torch.tensor(0.5, device=dev))
        call(c, c[1], step=torch.tensor([t], device=dev), lr=torch.tensor(HYPER["lr"], device=dev),
             grad_scale=torch.tensor([0.5], device=dev))
    for i in (0, 2, 3, 4, 5):
        u8 = lambda t: t.view(torch.uint8)  # noqa: E731
        assert torch.equal(u8(a[i]), u8(b[i]))
        # the rate is an fp32 scalar on the device: one rounding more in every update
        close = (a[i].float() - c[i].float()).abs() <= 0.14 * a[i].float().abs() + 1e-9
        assert close.all() and torch.equal(a[i].float(), c[i].float()) or (a[i].float() != c[i].float()).float().mean() < 0.02
    before = [t.clone() for t in a]
    for s in (0.0, float("inf"), float("nan")):
        call(a, a[1], step=4, grad_scale=torch.tensor(s, device=dev))
    call(a, a[1], step=torch.zeros(1, dtype=torch.int64, device=dev))  # a step number below 1
    for t, u in zip(a, before):
        if t is not None:
            assert torch.equal(t.view(torch.uint8), u.view(torch.uint8))


@pytest.mark.parametrize("N,D,U,dt,bits", [(1, 8, 1, torch.float32, 32), (50, 200, 17, torch.float32, 32),
                                           (64, 128, 64, torch.float32, 8), (300, 640, 100, torch.bfloat16, 8),
                                           (4096, 64, 1601, torch.bfloat16, 32), (33, 2048, 5, torch.bfloat16, 8)])
def test_rows(gpu_lib, N, D, U, dt, bits):
    p, _, m, v, sm, sv = make((N, D), dt, bits, 31)
    g = torch.Generator().manual_seed(32)
    rows = torch.randperm(N, generator=g)[:U].sort().values
    gr = torch.randn((U, D), generator=g) * 1e-3
    sc = {} if bits == 32 else dict(exp_avg_scale=sm, exp_avg_sq_scale=sv)
    for t in (1, 2):
        p0, (m0, v0) = p.clone(), values(m, v, sm, sv)
        raw0 = [x.clone() for x in (m, v)]
        pk.mem_adamw_rows(p, rows.cuda(), gr.cuda(), m, v, step=t, seed=4, **sc, **HYPER)
        i = rows.numpy()
        at = i[:, None] * D + np.arange(D)
        pick = lambda s: None if s is None else s.view(N, -1)[rows.cuda()].reshape(-1)  # noqa: E731
        check((f64(p0)[i], (m0[i], v0[i])),
              (p[rows.cuda()], m.float()[rows.cuda()], v.float()[rows.cuda()], pick(sm), pick(sv)),
              gr.double().numpy(), t, HYPER, bits, places=at, seed=4)
        rest = torch.ones(N, dtype=torch.bool)
        rest[rows] = False
        assert torch.equal(p[rest.cuda()], p0[rest.cuda()])
        for x, x0 in zip((m, v), raw0):
            assert torch.equal(x.float()[rest.cuda()], x0.float()[rest.cuda()])


def test_rows_equal_dense_where_all_are_touched(gpu_lib):
    a, b = make((40, 256), torch.bfloat16, 8, 41), make((40, 256), torch.bfloat16, 8, 41)
    pk.mem_adamw(*[[x] for x in a[:4]], step=3, exp_avg_scales=[a[4]], exp_avg_sq_scales=[a[5]], **HYPER)
    pk.mem_adamw_rows(b[0], torch.arange(40, device="cuda"), b[1], b[2], b[3], step=3, exp_avg_scale=b[4],
                      exp_avg_sq_scale=b[5], **HYPER)
    for x, y in zip(a, b):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_rows_twice_and_outside(gpu_lib):
    """Equal neighbours are one row with the sum of their gradients; rows outside are passed over."""
    a, b = make((30, 128), torch.float32, 8, 51), make((30, 128), torch.float32, 8, 51)
    g = torch.randn((6, 128), generator=torch.Generator().manual_seed(52)).cuda() * 1e-3
    rows = torch.tensor([-5, 3, 3, 3, 29, 30], device="cuda")
    pk.mem_adamw_rows(a[0], rows, g, a[2], a[3], step=1, exp_avg_scale=a[4], exp_avg_sq_scale=a[5], **HYPER)
    pk.mem_adamw_rows(b[0], torch.tensor([3, 29], device="cuda"), torch.stack([g[1] + g[2] + g[3], g[4]]), b[2], b[3],
                      step=1, exp_avg_scale=b[4], exp_avg_sq_scale=b[5], **HYPER)
    for x, y in zip(a, b):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    pk.mem_adamw_rows(a[0], rows[:0], g[:0], a[2], a[3], step=2, exp_avg_scale=a[4], exp_avg_sq_scale=a[5], **HYPER)
    assert torch.equal(a[0], b[0])


def test_rows_debug_check(gpu_lib, monkeypatch):
    x = make((30, 128), torch.float32, 32, 53)
    monkeypatch.setenv("PKMEM_DEBUG", "1")
    g = torch.zeros((3, 128), device="cuda")
    call = lambda r: pk.mem_adamw_rows(x[0], torch.tensor(r, device="cuda"), g, x[2], x[3], step=1, **HYPER)  # noqa: E731
    call([0, 0, 29])
    for bad in ([0, 2, 1], [-1, 0, 1], [0, 1, 30]):
        with pytest.raises(pk.PkmemError):
            call(bad)


def test_long_run_in_8_bits_follows_32_bits(gpu_lib):
    """200 steps of a constant gradient's decay: a state that nearest rounding would
    freeze decays as the 32-bit one does.  g = 0 after the first step, so v falls by
    0.999 a step to 0.819 of itself and r to 0.905; drawn in steps of at most 1/8 of a
    value, its mean over n = 4096 elements is within 6 / sqrt(n) * 1/8 * sqrt(200 * 0.008)
    (a step is drawn with a probability under 0.008 of one) of that, plus half of a
    random bit's weight (2^-13 of a step of 1/8) for each of the 200."""
    n = 4096
    p = torch.zeros(n, device="cuda")
    m, v, sm, sv = pk.mem_adamw_state(p, 8)
    g = torch.full((n,), 0.03, device="cuda")
    g[::128] = 1.0
    z = torch.zeros(n, device="cuda")
    for t in range(1, 202):
        pk.mem_adamw([p], [g if t == 1 else z], [m], [v], step=t, exp_avg_scales=[sm], exp_avg_sq_scales=[sv], lr=0.0)
    r = (v.float() * sv.repeat_interleave(128)).cpu().double()
    keep = torch.arange(n) % 128 != 0
    want = 0.03 * np.sqrt(1e-3) * 0.999 ** 100
    tol = 6 / np.sqrt(n) * 0.125 * np.sqrt(200 * 0.008 * 4) + 200 * 0.125 * 2.0 ** -13
    assert abs(float(r[keep].mean()) / want - 1) <= tol


def test_captured_step(gpu_lib):
    """A captured step whose step number and rate live on the device, replayed between
    eager work, equals the eager steps."""
    dev = torch.device("cuda")
    a, b = make((5000,), torch.bfloat16, 8, 61), make((5000,), torch.bfloat16, 8, 61)
    ta, tb = (torch.zeros(1, dtype=torch.int64, device=dev) for _ in range(2))
    lr = torch.tensor([1e-3], device=dev)

    def step(x, t):
        t.add_(1)
        pk.mem_adamw([x[0]], [x[1]], [x[2]], [x[3]], step=t, lr=lr, seed=3, exp_avg_scales=[x[4]], exp_avg_sq_scales=[x[5]])

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(b, tb)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for k in range(4):
        lr.fill_(1e-3 / (k + 1))
        step(a, ta)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k


def test_refusals(gpu_lib):
    x = make((256,), torch.float32, 32, 71)
    y = make((256,), torch.float32, 8, 71)
    with pytest.raises(ValueError):
        pk.mem_adamw([x[0]], [x[1][:100]], [x[2]], [x[3]], step=1, lr=1e-3)
    with pytest.raises(ValueError):
        pk.mem_adamw([y[0]], [y[1]], [y[2]], [y[3]], step=1, lr=1e-3)
    with pytest.raises(ValueError):
        pk.mem_adamw([y[0]], [y[1]], [y[2]], [y[3]], step=1, lr=1e-3, exp_avg_scales=[y[4][:1]], exp_avg_sq_scales=[y[5]])
    with pytest.raises(TypeError):
        pk.mem_adamw([x[0].half()], [x[1]], [x[2]], [x[3]], step=1, lr=1e-3)
    with pytest.raises(TypeError):
        pk.mem_adamw([x[0]], [x[1]], [x[2]], [y[3]], step=1, lr=1e-3)
    with pytest.raises(pk.PkmemError):
        pk.mem_adamw([x[0]], [x[1]], [x[2]], [x[3]], step=0, lr=1e-3)
    with pytest.raises(ValueError):
        pk.mem_adamw([x[0]], [x[1]], [x[2]], [x[3]], step=torch.tensor([1.0], device="cuda"), lr=1e-3)
