"""Argument checks of layer norm, gated part and 8-bit blocks, on the host (fake pointers that
are never dereferenced; nothing is launched): refusals, overlapping buffers, random calls,
and what the binding checks."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk
from tests.test_abi_block_spans import PLACES, cases, expect

OK, INVALID, UNSUPPORTED, WORKSPACE, HIP = 0, -1, -2, -3, -4
F32, BF16, E4M3 = 0, 1, 2
A, B, C, D, E, F, G, H = (1 << e for e in range(32, 40))  # far apart
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("fake device pointers: host-only test")
    return pk.load()


def call(lib, fn, defaults, kw):
    a = {**defaults, **kw}
    return getattr(lib, fn)(*a.values(), None), lib.mem_last_error().decode()


NORM = dict(x=A, res=None, w=B, b=C, dt=BF16, T=4, D=64, eps=1e-5, s=None, y=D)
NORM_BWD = dict(dy=A, h=B, w=C, dt=BF16, T=4, D=64, eps=1e-5, ds=None, dx=D, gw=E, gb=F, ws=G, n=BIG)
GLU = dict(x=A, w=B, dt=BF16, sx=None, sw=None, b=None, T=4, N=64, K=64, act=2, z=None, y=C, ydt=BF16)
GLU_BWD = dict(dy=A, z=B, dt=BF16, act=2, T=4, N=64, dz=C)
QUANT = dict(x=A, dt=BF16, R=4, C=64, tile=0, q=B, s=C, qt=D, st=E)
BLOCKS = dict(x=A, w=B, sx=C, sw=D, tile=0, b=None, r=None, T=4, N=64, K=64, act=0, z=None, y=E, ydt=BF16, ws=None, n=0)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=E4M3), INVALID, "dtype"), (dict(dt=7), INVALID, "dtype"),
    (dict(T=-1), INVALID, "rows must be >= 0"), (dict(T=1 << 31), UNSUPPORTED, "2^31"),
    (dict(D=0), UNSUPPORTED, "multiple of 8"), (dict(D=12), UNSUPPORTED, "multiple of 8"),
    (dict(D=16392), UNSUPPORTED, "32 KiB"), (dict(dt=F32, D=8200), UNSUPPORTED, "32 KiB"),
    (dict(eps=-1.0), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"), (dict(eps=float("inf")), INVALID, "eps"),
    (dict(x=None), INVALID, "null"), (dict(y=None), INVALID, "null"),
    (dict(x=A + 8), INVALID, "aligned"), (dict(w=B + 2), INVALID, "aligned"), (dict(b=C + 4), INVALID, "aligned"),
    (dict(res=E + 4), INVALID, "aligned"), (dict(s=E + 8), INVALID, "aligned"),
    (dict(s=D), INVALID, "one buffer"), (dict(y=B), INVALID, "share"), (dict(y=C), INVALID, "share"), (dict(s=C), INVALID, "share"),
    (dict(T=0, x=None, y=None), OK, ""),
])
def test_layernorm_rejects(lib, kw, code, text):
    rc, msg = call(lib, "mem_layernorm", NORM, kw)
    assert rc == code and text in msg


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=E4M3), INVALID, "dtype"), (dict(T=-3), INVALID, "rows"), (dict(D=20), UNSUPPORTED, "multiple of 8"),
    (dict(eps=-0.5), INVALID, "eps"), (dict(dy=None), INVALID, "null"), (dict(h=None), INVALID, "null"),
    (dict(dx=None), INVALID, "null"), (dict(dx=D + 8), INVALID, "aligned"), (dict(gw=E + 2), INVALID, "aligned"),
    (dict(gb=F + 1), INVALID, "aligned"), (dict(ws=None), WORKSPACE, "workspace"), (dict(n=16), WORKSPACE, "workspace"),
    (dict(ws=G + 64), INVALID, "256-byte"), (dict(gw=F), INVALID, "share"), (dict(gw=A), INVALID, "share"),
    (dict(T=0, dy=None, h=None, dx=None), OK, ""),
])
def test_layernorm_backward_rejects(lib, kw, code, text):
    rc, msg = call(lib, "mem_layernorm_backward", NORM_BWD, kw)
    assert rc == code and text in msg


def test_layernorm_backward_workspace(lib):
    size = lib.mem_layernorm_backward_workspace_size
    assert size(-1, 64) == 0 and size(4, 0) == 0
    assert 0 < size(4, 64) <= size(4096, 64) == size(1 << 20, 64) and size(4096, 64) % 256 == 0
    # one gradient needs it, none does not
    for kw, need in ((dict(gw=None), True), (dict(gb=None), True), (dict(gw=None, gb=None), False)):
        rc, _ = call(lib, "mem_layernorm_backward", NORM_BWD, dict(kw, ws=None, n=0))
        assert rc == (WORKSPACE if need else HIP)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=7), INVALID, "dtype"), (dict(ydt=E4M3), INVALID, "y_dt"), (dict(dt=F32), INVALID, "y_dt"),
    (dict(act=4), INVALID, "activation"), (dict(act=-1), INVALID, "activation"),
    (dict(T=-1), INVALID, "T must"), (dict(T=1 << 31), UNSUPPORTED, "2^31"),
    (dict(N=12), UNSUPPORTED, "multiple of 8"), (dict(N=(1 << 19) + 8), UNSUPPORTED, "2^19"), (dict(K=20), UNSUPPORTED, "multiple of 8"),
    (dict(K=(1 << 20) + 16), UNSUPPORTED, "2^20"), (dict(T=(1 << 31) - 1, N=1 << 19), UNSUPPORTED, "tiles"),
    (dict(dt=E4M3, sx=D, sw=E, K=24), UNSUPPORTED, "multiple of 16"),
    (dict(sx=D), INVALID, "scales"), (dict(sw=D), INVALID, "scales"), (dict(dt=E4M3, sx=D), INVALID, "null"),
    (dict(x=None), INVALID, "null"), (dict(w=None), INVALID, "null"), (dict(y=None), INVALID, "null"),
    (dict(x=A + 8), INVALID, "aligned"), (dict(b=D + 8), INVALID, "aligned"), (dict(z=D + 8), INVALID, "aligned"),
    (dict(dt=E4M3, sx=D + 2, sw=E), INVALID, "aligned"), (dict(dt=E4M3, sx=D, sw=E + 8), INVALID, "aligned"),
    (dict(T=0, x=None, w=None, y=None), OK, ""),
])
def test_glu_rejects(lib, kw, code, text):
    rc, msg = call(lib, "mem_glu", GLU, kw)
    assert rc == code and text in msg


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=E4M3), INVALID, "dtype"), (dict(act=5), INVALID, "activation"), (dict(T=-1), INVALID, "T must"),
    (dict(T=1 << 31), UNSUPPORTED, "2^31"), (dict(N=4), UNSUPPORTED, "multiple of 8"), (dict(N=(1 << 19) + 8), UNSUPPORTED, "2^19"),
    (dict(dy=None), INVALID, "null"), (dict(z=None), INVALID, "null"), (dict(dz=None), INVALID, "null"),
    (dict(dz=C + 4), INVALID, "aligned"), (dict(dz=A), INVALID, "share"), (dict(dz=B + 16), INVALID, "share"),
    (dict(dz=B), HIP, ""), (dict(T=0, dy=None, z=None, dz=None), OK, ""),
])
def test_glu_backward_rejects(lib, kw, code, text):
    rc, msg = call(lib, "mem_glu_backward", GLU_BWD, kw)
    assert rc == code and text in msg


@pytest.mark.parametrize("kw,code,text", [
    (dict(dt=E4M3), INVALID, "dtype"), (dict(R=-1), INVALID, "R must"), (dict(R=1 << 31), UNSUPPORTED, "2^31"),
    (dict(C=0), UNSUPPORTED, "multiple of 16"), (dict(C=24), UNSUPPORTED, "multiple of 16"), (dict(C=(1 << 20) + 16), UNSUPPORTED, "2^20"),
    (dict(q=None), INVALID, "together"), (dict(s=None), INVALID, "together"), (dict(qt=None), INVALID, "together"),
    (dict(st=None), INVALID, "together"), (dict(x=None), INVALID, "null"), (dict(q=None, s=None, qt=None, st=None), INVALID, "null"),
    (dict(x=A + 8), INVALID, "aligned"), (dict(q=B + 8), INVALID, "aligned"), (dict(s=C + 2), INVALID, "aligned"),
    (dict(qt=D + 4), INVALID, "aligned"), (dict(st=E + 1), INVALID, "aligned"),
    (dict(q=None, s=None), HIP, ""), (dict(qt=None, st=None), HIP, ""), (dict(R=0, x=None), OK, ""),
])
def test_quantize_blocks_rejects(lib, kw, code, text):
    rc, msg = call(lib, "mem_quantize_blocks", QUANT, kw)
    assert rc == code and text in msg


@pytest.mark.parametrize("kw,code,text", [
    (dict(ydt=E4M3), INVALID, "y_dt"), (dict(act=9), INVALID, "activation"), (dict(T=-1), INVALID, "T must"),
    (dict(T=1 << 31), UNSUPPORTED, "2^31"), (dict(N=4), UNSUPPORTED, "multiple of 8"), (dict(K=24), UNSUPPORTED, "multiple of 16"),
    (dict(N=(1 << 20) + 8), UNSUPPORTED, "2^20"), (dict(T=(1 << 31) - 1, N=1 << 20), UNSUPPORTED, "tiles"),
    (dict(T=(1 << 30) - 127, N=8, K=16, ydt=F32), UNSUPPORTED, "128 x 128"), (dict(T=(1 << 30) - 128, N=8, K=16, ydt=F32), HIP, ""),
    (dict(x=None), INVALID, "null"), (dict(w=None), INVALID, "null"), (dict(sx=None), INVALID, "null"),
    (dict(sw=None), INVALID, "null"), (dict(y=None), INVALID, "null"), (dict(w=B + 4), INVALID, "aligned"),
    (dict(sx=C + 2), INVALID, "aligned"), (dict(sw=D + 4), INVALID, "aligned"), (dict(sw=D + 4, tile=1), HIP, ""),
    (dict(sw=D + 2, tile=1), INVALID, "aligned"), (dict(r=F + 8), INVALID, "aligned"), (dict(ws=F + 8), INVALID, "256-byte"),
    (dict(T=64, K=1 << 16, ydt=F32), WORKSPACE, "workspace"), (dict(T=64, K=1 << 16, ydt=F32, ws=F, n=100), WORKSPACE, "workspace"),
    (dict(T=64, K=1 << 16, ydt=F32, ws=F, n=BIG), HIP, ""), (dict(T=64, K=1 << 16), HIP, ""),
    (dict(T=0, x=None, w=None, y=None, sx=None, sw=None), INVALID, ""),
])
def test_linear_blocks_rejects(lib, kw, code, text):
    if kw.get("T") == 0:
        code = OK
    rc, msg = call(lib, "mem_linear_blocks", BLOCKS, kw)
    assert rc == code and text in msg


T = 6


@pytest.mark.parametrize("dt", [F32, BF16])
def test_layernorm_spans(lib, dt):
    e, d = 4 if dt == F32 else 2, 64
    rows = T * d * e
    sizes = dict(x=rows, res=rows, w=d * e, b=d * e, s=rows, y=rows)
    for a, bad in cases(sizes, ("s", "y"), [("s", "x"), ("s", "res"), ("y", "x"), ("y", "res")]):
        expect(lib, lib.mem_layernorm(a["x"], a["res"], a["w"], a["b"], dt, T, d, 1e-5, a["s"], a["y"], None), bad)
    sizes = dict(dy=rows, h=rows, ds=rows, w=d * e, dx=rows, gw=d * 4, gb=d * 4, ws=lib.mem_layernorm_backward_workspace_size(T, d))
    for a, bad in cases(sizes, ("dx", "gw", "gb", "ws"), [("dx", "dy"), ("dx", "h"), ("dx", "ds")]):
        if a["ws"] % 256 == 0:
            expect(lib, lib.mem_layernorm_backward(a["dy"], a["h"], a["w"], dt, T, d, 1e-5, a["ds"], a["dx"], a["gw"], a["gb"],
                                                    a["ws"], sizes["ws"], None), bad)


@pytest.mark.parametrize("dt,ydt", [(F32, F32), (BF16, BF16), (BF16, F32), (E4M3, BF16), (E4M3, F32)])
def test_glu_spans(lib, dt, ydt):
    N, K, n, e, ye = 32, 48, 64, {F32: 4, BF16: 2, E4M3: 1}[dt], 4 if ydt == F32 else 2
    sizes = dict(x=n * K * e, w=2 * N * K * e, sx=n * 4, sw=2 * N * 4, b=2 * N * ye, z=2 * n * N * ye, y=n * N * ye)
    if dt != E4M3:
        del sizes["sx"], sizes["sw"]
    for a, bad in cases(sizes, ("z", "y")):
        expect(lib, lib.mem_glu(a["x"], a["w"], dt, a.get("sx"), a.get("sw"), a["b"], n, N, K, 1, a["z"], a["y"], ydt, None), bad)
    if dt != E4M3 and dt == ydt:
        for a, bad in cases(dict(dy=n * N * e, z=2 * n * N * e, dz=2 * n * N * e), ("dz",), [("dz", "z")]):
            expect(lib, lib.mem_glu_backward(a["dy"], a["z"], dt, 2, n, N, a["dz"], None), bad)


@pytest.mark.parametrize("tile", [0, 1])
def test_quantize_blocks_spans(lib, tile):
    R, Ck = 256, 512
    nb = 2 * 4 * 4 if tile else None
    sizes = dict(x=R * Ck * 2, q=R * Ck, s=nb or 4 * R * 4, qt=R * Ck, st=nb or 2 * Ck * 4)
    for a, bad in cases(sizes, ("q", "s", "qt", "st")):
        if not any(a[k] % 16 for k in ("x", "q", "qt")):
            expect(lib, lib.mem_quantize_blocks(a["x"], BF16, R, Ck, tile, a["q"], a["s"], a["qt"], a["st"], None), bad)


@pytest.mark.parametrize("n,N,K,ydt,tile", [(64, 32, 256, BF16, 0), (64, 1024, 256, F32, 1), (64, 32, 65536, F32, 0)])
def test_linear_blocks_spans(lib, n, N, K, ydt, tile):
    ye, kb = 4 if ydt == F32 else 2, K // 128
    ws = lib.mem_linear_blocks_workspace_size(n, N, K, ydt)
    assert (ws > 0) == (K > 1000)
    sizes = dict(x=n * K, w=N * K, sx=kb * n * 4, sw=kb * (N // 128 if tile else N) * 4, b=N * ye, r=n * N * ye, z=n * N * ye, y=n * N * ye)
    if ws:
        sizes["ws"] = ws
    for a, bad in cases(sizes, [k for k in ("z", "y", "ws") if k in sizes], [("y", "r")]):
        if a.get("ws", 0) % 256 == 0:
            expect(lib, lib.mem_linear_blocks(a["x"], a["w"], a["sx"], a["sw"], tile, a["b"], a["r"], n, N, K, 1, a["z"], a["y"], ydt,
                                               a.get("ws"), ws, None), bad)


@pytest.mark.parametrize("seed", range(3))
def test_random_calls(lib, seed):
    rng = np.random.default_rng(seed)
    p = lambda: int(rng.choice([0, A, A, B, C, D, D + 8, E + 4, F + 1]))  # noqa: E731
    n = lambda: int(rng.choice([-8, 0, 1, 8, 16, 64, 128, 200, 1024, 16384, 16392, 1 << 19, 1 << 20, (1 << 20) + 16]))  # noqa: E731
    dt = lambda: int(rng.choice([0, 1, 1, 2, 7]))  # noqa: E731
    rows = lambda: int(rng.choice([-1, 0, 1, 333, 1 << 20, (1 << 31) - 1, 1 << 31, 1 << 40]))  # noqa: E731
    eps = lambda: float(rng.choice([0.0, 1e-5, -1.0, np.nan]))  # noqa: E731
    act = lambda: int(rng.integers(-1, 5))  # noqa: E731
    ws = lambda: int(rng.choice([0, 1000, BIG]))  # noqa: E731
    codes = {0, -1, -2, -3, -4}
    for _ in range(500):
        assert lib.mem_layernorm(p(), p(), p(), p(), dt(), rows(), n(), eps(), p(), p(), None) in codes
        assert lib.mem_layernorm_backward(p(), p(), p(), dt(), rows(), n(), eps(), p(), p(), p(), p(), p(), ws(), None) in codes
        assert lib.mem_glu(p(), p(), dt(), p(), p(), p(), rows(), n(), n(), act(), p(), p(), dt(), None) in codes
        assert lib.mem_glu_backward(p(), p(), dt(), act(), rows(), n(), p(), None) in codes
        assert lib.mem_quantize_blocks(p(), dt(), rows(), n(), act(), p(), p(), p(), p(), None) in codes
        assert lib.mem_linear_blocks(p(), p(), p(), p(), act(), p(), p(), rows(), n(), n(), act(), p(), p(), dt(), p(), ws(), None) in codes
    for r in (-1, 0, 1, 777, 1 << 20, (1 << 31) - 1):
        for c in (-8, 0, 8, 1032, 1 << 20):
            assert lib.mem_layernorm_backward_workspace_size(r, c) >= 0
            for d in (0, 1, 2, 9):
                assert lib.mem_linear_blocks_workspace_size(r, c, 1 << 20, d) >= 0


def test_binding_refuses_cpu_tensors():
    x, w, q = torch.zeros(4, 64), torch.zeros(32, 64), torch.zeros(4, 64).to(torch.float8_e4m3fn)
    for f in (lambda: pk.mem_layernorm(x), lambda: pk.mem_layernorm_backward(x, x), lambda: pk.mem_glu(x, w),
              lambda: pk.mem_glu_backward(x, torch.zeros(4, 128)), lambda: pk.mem_quantize_blocks(x),
              lambda: pk.mem_linear_blocks(q, q, x, x)):
        with pytest.raises(ValueError):
            f()


def test_names_are_public():
    for name in ("mem_layernorm", "mem_layernorm_backward", "mem_glu", "mem_glu_backward", "mem_quantize_blocks", "mem_linear_blocks"):
        assert name in pk.__all__ and isinstance(getattr(pk.load(), name), ctypes._CFuncPtr)
