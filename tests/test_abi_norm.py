"""Argument checks of the norm and optimizer calls, on the host (fake pointers
that are never dereferenced; nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2412_09764_amd as pk

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
F32, BF16, E4M3 = 0, 1, 2
FAKE, BIG = 0x10000, 1 << 40


@pytest.fixture(scope="module")
def lib():
    return pk.load()


def msg(lib):
    return lib.mem_last_error().decode()


def norm(lib, x=FAKE, res=None, w=FAKE, dt=BF16, T=4, D=64, eps=1e-5, s=None, y=FAKE, ydt=BF16, sc=None):
    return lib.mem_rmsnorm(x, res, w, dt, T, D, eps, s, y, ydt, sc, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=2, ydt=2, sc=FAKE), INVALID, "dtype"),
    (dict(dt=7), INVALID, "dtype"),
    (dict(ydt=F32), INVALID, "y_dt"),
    (dict(T=-1), INVALID, "rows must be >= 0"),
    (dict(T=1 << 31), UNSUPPORTED, "2^31"),
    (dict(D=0), UNSUPPORTED, "multiple of 8"),
    (dict(D=12), UNSUPPORTED, "multiple of 8"),
    (dict(D=16392), UNSUPPORTED, "32 KiB"),
    (dict(dt=F32, ydt=F32, D=8200), UNSUPPORTED, "32 KiB"),
    (dict(eps=-1.0), INVALID, "eps"),
    (dict(eps=float("nan")), INVALID, "eps"),
    (dict(eps=float("inf")), INVALID, "eps"),
    (dict(x=None), INVALID, "null"),
    (dict(y=None), INVALID, "null"),
    (dict(ydt=E4M3), INVALID, "null"),
    (dict(sc=FAKE), INVALID, "scale_out"),
    (dict(x=FAKE + 8), INVALID, "aligned"),
    (dict(w=FAKE + 2), INVALID, "aligned"),
    (dict(res=FAKE + 4), INVALID, "aligned"),
    (dict(s=FAKE + 8), INVALID, "aligned"),
    (dict(s=FAKE), INVALID, "one buffer"),
    (dict(ydt=E4M3, sc=FAKE + 2), INVALID, "aligned"),
])
def test_norm_rejects(lib, kw, code, text):
    assert norm(lib, **kw) == code and text in msg(lib)


def norm_bwd(lib, dy=FAKE, h=FAKE, w=FAKE, dt=BF16, T=4, D=64, eps=1e-5, ds=None, dx=FAKE, gw=FAKE, ws=FAKE, n=BIG):
    return lib.mem_rmsnorm_backward(dy, h, w, dt, T, D, eps, ds, dx, gw, ws, n, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=2), INVALID, "dtype"),
    (dict(D=4), UNSUPPORTED, "multiple of 8"),
    (dict(T=-2), INVALID, "rows"),
    (dict(eps=-0.5), INVALID, "eps"),
    (dict(dy=None), INVALID, "null"),
    (dict(h=None), INVALID, "null"),
    (dict(dx=None), INVALID, "null"),
    (dict(dx=FAKE + 8), INVALID, "aligned"),
    (dict(ds=FAKE + 8), INVALID, "aligned"),
    (dict(gw=FAKE + 2), INVALID, "aligned"),
    (dict(ws=None), WORKSPACE, "workspace"),
    (dict(n=100), WORKSPACE, "workspace"),
    (dict(ws=FAKE + 16), INVALID, "256-byte"),
])
def test_norm_backward_rejects(lib, kw, code, text):
    assert norm_bwd(lib, **kw) == code and text in msg(lib)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=2), INVALID, "dtype"),
    (dict(C=20), UNSUPPORTED, "multiple of 8"),
    (dict(R=-1), INVALID, "rows"),
    (dict(x=None), INVALID, "null"),
    (dict(sc=None), INVALID, "null"),
    (dict(q=FAKE + 8), INVALID, "aligned"),
])
def test_quantize_rejects(lib, kw, code, text):
    a = dict(x=FAKE, dt=BF16, R=4, C=64, q=FAKE, sc=FAKE)
    a.update(kw)
    assert lib.mem_quantize_rows(a["x"], a["dt"], a["R"], a["C"], a["q"], a["sc"], None) == code
    assert text in msg(lib)


def test_empty_batches_are_noops(lib):
    assert norm(lib, T=0) == OK
    assert norm_bwd(lib, T=0, ws=None, n=0) == OK
    assert lib.mem_quantize_rows(None, BF16, 0, 64, None, None, None) == OK


TENSOR = dict(param=FAKE, grad=FAKE, exp_avg=FAKE, exp_avg_sq=FAKE, exp_avg_scale=None,
              exp_avg_sq_scale=None, numel=4096, param_dt=F32, grad_dt=F32, state_dt=F32)
OPTS = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=1, seed=0)


@pytest.mark.parametrize("t,o,code,text", [
    (dict(param_dt=E4M3), {}, INVALID, "dtype"),
    (dict(grad_dt=E4M3), {}, INVALID, "dtype"),
    (dict(state_dt=BF16), {}, INVALID, "dtype"),
    (dict(state_dt=E4M3), {}, INVALID, "null"),
    (dict(numel=-1), {}, INVALID, "numel"),
    (dict(numel=1 << 41), {}, UNSUPPORTED, "2^40"),
    (dict(param=None), {}, INVALID, "null"),
    (dict(grad=None), {}, INVALID, "null"),
    (dict(exp_avg_sq=None), {}, INVALID, "null"),
    (dict(param=FAKE + 2), {}, INVALID, "aligned"),
    (dict(exp_avg=FAKE + 1), {}, INVALID, "aligned"),
    ({}, dict(beta1=1.0), INVALID, "betas"),
    ({}, dict(beta2=-0.1), INVALID, "betas"),
    ({}, dict(beta1=float("nan")), INVALID, "betas"),
    ({}, dict(lr=-1.0), INVALID, "lr"),
    ({}, dict(lr=float("inf")), INVALID, "lr"),
    ({}, dict(eps=-1e-8), INVALID, "eps"),
    ({}, dict(weight_decay=float("nan")), INVALID, "weight_decay"),
    ({}, dict(step=0), INVALID, "step"),
    ({}, dict(lr_dev=FAKE + 2), INVALID, "aligned"),
    ({}, dict(step_dev=FAKE + 4), INVALID, "aligned"),
])
def test_adamw_rejects(lib, t, o, code, text):
    ts = (pk._AdamwTensor * 2)(pk._AdamwTensor(**{**TENSOR, "numel": 0}), pk._AdamwTensor(**{**TENSOR, **t}))
    opts = pk._AdamwOpts(**{**OPTS, **o})
    assert lib.mem_adamw(ctypes.addressof(ts), 2, ctypes.addressof(opts), None) == code
    assert text in msg(lib)


def test_adamw_lists(lib):
    opts = pk._AdamwOpts(**OPTS)
    empty = (pk._AdamwTensor * 1)(pk._AdamwTensor(numel=0))
    assert lib.mem_adamw(None, 0, ctypes.addressof(opts), None) == OK
    assert lib.mem_adamw(ctypes.addressof(empty), 1, ctypes.addressof(opts), None) == OK
    assert lib.mem_adamw(None, 1, ctypes.addressof(opts), None) == INVALID
    assert lib.mem_adamw(None, -1, ctypes.addressof(opts), None) == INVALID
    assert lib.mem_adamw(ctypes.addressof(empty), 1, None, None) == INVALID


@pytest.mark.parametrize("t,kw,code,text", [
    ({}, dict(N=0), INVALID, "N must"),
    ({}, dict(D=60), UNSUPPORTED, "multiple of 8"),
    ({}, dict(N=63), INVALID, "numel"),
    ({}, dict(N=1 << 40), INVALID, "numel"),
    (dict(grad_dt=BF16), {}, UNSUPPORTED, "fp32"),
    (dict(state_dt=E4M3, exp_avg_scale=FAKE, exp_avg_sq_scale=FAKE), {}, UNSUPPORTED, "multiple of 128"),
    (dict(param=FAKE + 8), {}, INVALID, "aligned"),
    (dict(grad=None), {}, INVALID, "null"),
    ({}, dict(rows=None), INVALID, "null"),
    ({}, dict(rows=FAKE + 4), INVALID, "aligned"),
    ({}, dict(U=-1), INVALID, "U must"),
    ({}, dict(U=1 << 31), UNSUPPORTED, "too many"),
    (dict(grad=None), dict(U=0, rows=None), OK, ""),
])
def test_adamw_rows_rejects(lib, t, kw, code, text):
    a = dict(N=64, D=64, rows=FAKE, U=5)
    a.update(kw)
    table = pk._AdamwTensor(**{**TENSOR, **t})
    opts = pk._AdamwOpts(**OPTS)
    rc = lib.mem_adamw_rows(ctypes.addressof(table), a["N"], a["D"], a["rows"], a["U"], ctypes.addressof(opts), None)
    assert rc == code and text in msg(lib)


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        pk.mem_rmsnorm(x)
    with pytest.raises(ValueError):
        pk.mem_rmsnorm_backward(x, x)
    with pytest.raises(ValueError):
        pk.mem_quantize_rows(x)
    with pytest.raises(ValueError):
        pk.mem_adamw([x], [x], [x], [x], lr=1e-3, step=1)
    with pytest.raises(ValueError):
        pk.mem_adamw([x], [], [x], [x], lr=1e-3, step=1)
    with pytest.raises(ValueError):
        pk.mem_adamw_rows(x, torch.zeros(2, dtype=torch.int64), x[:2], x, x, lr=1e-3, step=1)


def test_adamw_state_shapes():
    p = torch.zeros(3, 130)
    m, v, sm, sv = pk.mem_adamw_state(p)
    assert m.shape == v.shape == p.shape and sm is None and sv is None
    m, v, sm, sv = pk.mem_adamw_state(p, bits=8)
    assert m.dtype == v.dtype == torch.float8_e4m3fn and sm.shape == sv.shape == (4,)
    assert not m.float().any() and not sv.any()
    with pytest.raises(ValueError):
        pk.mem_adamw_state(p, bits=16)
