"""Argument checks of the projection calls, on the host (fake pointers that are
never dereferenced; nothing is launched)."""
import pytest
import torch

import paper_2412_09764_amd as pk

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
F32, BF16, E4M3 = 0, 1, 2
FAKE, BIG = 0x10000, 1 << 40
X, W, Y, DX = 0x20000, 0x30000, 0x40000, 0x50000  # buffers that have to differ


@pytest.fixture(scope="module")
def lib():
    return pk.load()


def msg(lib):
    return lib.mem_last_error().decode()


def linear(lib, x=X, w=W, dt=BF16, sx=None, sw=None, b=None, r=None, T=4, N=64, K=64, act=0, z=None, y=Y,
           ydt=BF16):
    return lib.mem_linear(x, w, dt, sx, sw, b, r, T, N, K, act, z, y, ydt, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=7), INVALID, "dtype"),
    (dict(dt=-1), INVALID, "dtype"),
    (dict(ydt=E4M3), INVALID, "y_dt"),
    (dict(dt=F32), INVALID, "y_dt"),
    (dict(T=-1), INVALID, "T must"),
    (dict(T=1 << 31), UNSUPPORTED, "2^31"),
    (dict(N=0), UNSUPPORTED, "multiple of 8"),
    (dict(N=20), UNSUPPORTED, "multiple of 8"),
    (dict(K=0), UNSUPPORTED, "multiple of 8"),
    (dict(K=12), UNSUPPORTED, "multiple of 8"),
    (dict(dt=E4M3, sx=FAKE, sw=FAKE, K=72), UNSUPPORTED, "multiple of 16"),
    (dict(N=(1 << 20) + 8), UNSUPPORTED, "2^20"),
    (dict(K=(1 << 20) + 8), UNSUPPORTED, "2^20"),
    (dict(T=(1 << 31) - 1, N=1 << 20), UNSUPPORTED, "tiles"),
    (dict(act=4), INVALID, "activation"),
    (dict(act=-1), INVALID, "activation"),
    (dict(sx=FAKE), INVALID, "scales"),
    (dict(dt=E4M3), INVALID, "null"),
    (dict(dt=E4M3, sx=FAKE), INVALID, "null"),
    (dict(x=None), INVALID, "null"),
    (dict(w=None), INVALID, "null"),
    (dict(y=None), INVALID, "null"),
    (dict(x=FAKE + 8), INVALID, "aligned"),
    (dict(w=FAKE + 2), INVALID, "aligned"),
    (dict(b=FAKE + 4), INVALID, "aligned"),
    (dict(r=FAKE + 8), INVALID, "aligned"),
    (dict(z=FAKE + 8), INVALID, "aligned"),
    (dict(y=FAKE + 2), INVALID, "aligned"),
    (dict(dt=E4M3, sx=FAKE + 2, sw=FAKE), INVALID, "aligned"),
    (dict(dt=E4M3, sx=FAKE, sw=FAKE + 4), INVALID, "aligned"),
    (dict(y=X), INVALID, "an output"),
    (dict(y=W), INVALID, "an output"),
    (dict(z=X), INVALID, "an output"),
    (dict(z=Y), INVALID, "an output"),
    (dict(z=FAKE, r=FAKE), INVALID, "an output"),
])
def test_linear_rejects(lib, kw, code, text):
    assert linear(lib, **kw) == code and text in msg(lib)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=E4M3), INVALID, "dtype"),
    (dict(act=5), INVALID, "activation"),
    (dict(T=-1), INVALID, "T must"),
    (dict(N=4), UNSUPPORTED, "multiple of 8"),
    (dict(dy=None), INVALID, "null"),
    (dict(z=None), INVALID, "null"),
    (dict(dz=FAKE + 4), INVALID, "aligned"),
    (dict(T=0, dy=None, z=None, dz=None), OK, ""),
])
def test_act_backward_rejects(lib, kw, code, text):
    a = dict(dy=FAKE, z=FAKE, dt=BF16, act=2, T=4, N=64, dz=FAKE)
    a.update(kw)
    assert lib.mem_act_backward(a["dy"], a["z"], a["dt"], a["act"], a["T"], a["N"], a["dz"], None) == code
    assert text in msg(lib)


def bwd(lib, dz=FAKE, x=X, w=W, dt=BF16, T=4, N=64, K=64, add=None, dx=DX, gw=FAKE, gb=FAKE, ws=FAKE, n=BIG):
    return lib.mem_linear_backward(dz, x, w, dt, T, N, K, add, dx, gw, gb, ws, n, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=E4M3), INVALID, "dtype"),
    (dict(N=12), UNSUPPORTED, "multiple of 8"),
    (dict(K=4), UNSUPPORTED, "multiple of 8"),
    (dict(T=-3), INVALID, "T must"),
    (dict(dz=None), INVALID, "null"),
    (dict(w=None), INVALID, "null"),
    (dict(x=None), INVALID, "null"),
    (dict(dx=FAKE + 8), INVALID, "aligned"),
    (dict(add=FAKE + 8), INVALID, "aligned"),
    (dict(gw=FAKE + 4), INVALID, "aligned"),
    (dict(gb=FAKE + 2), INVALID, "aligned"),
    (dict(ws=None), WORKSPACE, "workspace"),
    (dict(n=16), WORKSPACE, "workspace"),
    (dict(ws=FAKE + 64), INVALID, "256-byte"),
    (dict(dx=FAKE), INVALID, "dx_out"),
    (dict(dx=X), INVALID, "dx_out"),
    (dict(dx=W), INVALID, "dx_out"),
])
def test_linear_backward_rejects(lib, kw, code, text):
    assert bwd(lib, **kw) == code and text in msg(lib)


def test_noops_and_sizes(lib):
    assert linear(lib, T=0, x=None, y=None) == OK
    assert bwd(lib, T=0, dz=None) == OK
    assert bwd(lib, dx=None, gw=None, gb=None, ws=None, n=0, x=None, w=None) == OK
    assert lib.mem_linear_backward_workspace_size(-1, 64, 64, BF16) == 0
    small, large = (lib.mem_linear_backward_workspace_size(t, 1024, 1024, BF16) for t in (8, 16384))
    assert 1024 * 4 <= small < large


def test_binding_refuses_cpu_tensors():
    x, w = torch.zeros(4, 64), torch.zeros(32, 64)
    with pytest.raises(ValueError):
        pk.mem_linear(x, w)
    with pytest.raises(ValueError):
        pk.mem_act_backward(x, x, "silu")
    with pytest.raises(ValueError):
        pk.mem_linear_backward(torch.zeros(4, 32), x, w)
