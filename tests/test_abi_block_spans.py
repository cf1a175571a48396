"""Outputs that share any bytes with what the norm, projection and optimizer calls read or
write besides, not only those that start at the same place, are refused on the host (fake
pointers, nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2412_09764_amd as pk

OK, INVALID, HIP = 0, -1, -4
F32, BF16, E4M3 = 0, 1, 2
PLACES = [1 << e for e in range(32, 44)]  # far apart
T, D = 6, 64


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("fake device pointers: host-only test")
    return pk.load()


def expect(lib, rc, bad):
    """An accepted call ends in a HIP error on a host without a GPU."""
    assert rc == (INVALID if bad else HIP), lib.mem_last_error().decode()


def overlaps(sizes, writes, itself=()):
    """(kwargs, refused?) for buffers of these sizes in bytes: each pair with a write in it
    overlapping by 16 bytes at either end, inside one another, or starting at one place.
    itself: pairs that may be one buffer."""
    at = dict(zip(sizes, PLACES))
    yield at, False
    for a in writes:
        for b in sizes:
            if a == b:
                continue
            yield {**at, a: at[b]}, not ((a, b) in itself and sizes[a] == sizes[b])
            yield {**at, a: at[b] + sizes[b] - 16}, True
            yield {**at, b: at[a] + sizes[a] - 16}, True
            yield {**at, a: at[b] + sizes[b]}, False
            yield {**at, b: at[a] + sizes[a]}, False


def cases(sizes, writes, itself=()):
    return list(overlaps(sizes, writes, itself))


@pytest.mark.parametrize("dt,ydt", [(F32, F32), (BF16, BF16), (F32, E4M3), (BF16, E4M3)])
def test_norm(lib, dt, ydt):
    e = 4 if dt == F32 else 2
    rows = T * D * e
    sizes = dict(x=rows, res=rows, w=D * e, s=rows, y=T * D if ydt == E4M3 else rows)
    itself = [("s", "x"), ("s", "res")] + ([("y", "x"), ("y", "res")] if ydt != E4M3 else [])
    for a, bad in cases(sizes, ("s", "y"), itself):
        expect(lib, lib.mem_rmsnorm(a["x"], a["res"], a["w"], dt, T, D, 1e-5, a["s"], a["y"], ydt,
                                     1 << 50 if ydt == E4M3 else None, None), bad)
    if ydt == E4M3:
        a = dict(zip(sizes, PLACES))
        for b in sizes:
            for place in (a[b], a[b] + sizes[b] - 4, a[b] - T * 4 + 4):
                expect(lib, lib.mem_rmsnorm(a["x"], a["res"], a["w"], dt, T, D, 1e-5, a["s"], a["y"], ydt, place, None), True)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_norm_backward(lib, dt):
    e = 4 if dt == F32 else 2
    rows = T * D * e
    sizes = dict(dy=rows, h=rows, ds=rows, w=D * e, dx=rows, gw=D * 4, ws=lib.mem_rmsnorm_backward_workspace_size(T, D))
    assert sizes["ws"] % 256 == 0
    for a, bad in cases(sizes, ("dx", "gw", "ws"), [("dx", "dy"), ("dx", "h"), ("dx", "ds")]):
        if a["ws"] % 256:
            continue
        expect(lib, lib.mem_rmsnorm_backward(a["dy"], a["h"], a["w"], dt, T, D, 1e-5, a["ds"], a["dx"], a["gw"], a["ws"],
                                              sizes["ws"], None), bad)
    a = dict(zip(sizes, PLACES))
    # without a weight gradient the workspace is not used
    expect(lib, lib.mem_rmsnorm_backward(a["dy"], a["h"], a["w"], dt, T, D, 1e-5, a["ds"], a["dx"], None, a["h"], 1 << 20, None), False)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_quantize_rows(lib, dt):
    sizes = dict(x=T * D * (4 if dt == F32 else 2), q=T * D, s=T * 4)
    for a, bad in cases(sizes, ("q", "s")):
        if a["q"] % 16 or a["x"] % 16:
            continue
        expect(lib, lib.mem_quantize_rows(a["x"], dt, T, D, a["q"], a["s"], None), bad)


@pytest.mark.parametrize("dt,ydt", [(F32, F32), (BF16, BF16), (BF16, F32), (E4M3, BF16), (E4M3, F32)])
def test_linear(lib, dt, ydt):
    N, K, e, ye = 32, 48, {F32: 4, BF16: 2, E4M3: 1}[dt], 4 if ydt == F32 else 2
    n = 64  # tokens: the scales are a whole number of 16 bytes
    out = n * N * ye
    sizes = dict(x=n * K * e, w=N * K * e, sx=n * 4, sw=N * 4, b=N * ye, r=out, z=out, y=out)
    if dt != E4M3:
        del sizes["sx"], sizes["sw"]
    for a, bad in cases(sizes, ("z", "y"), [("y", "r")]):
        expect(lib, lib.mem_linear(a["x"], a["w"], dt, a.get("sx"), a.get("sw"), a["b"], a["r"], n, N, K, 1, a["z"],
                                    a["y"], ydt, None), bad)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_act_backward(lib, dt):
    n = T * D * (4 if dt == F32 else 2)
    for a, bad in cases(dict(dy=n, z=n, dz=n), ("dz",), [("dz", "dy"), ("dz", "z")]):
        expect(lib, lib.mem_act_backward(a["dy"], a["z"], dt, 2, T, D, a["dz"], None), bad)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("n", [64, 4096])  # one split of the tokens, and several
def test_linear_backward(lib, dt, n):
    N, K, e = 32, 48, 4 if dt == F32 else 2
    ws = lib.mem_linear_backward_workspace_size(n, N, K, dt)
    sizes = dict(dz=n * N * e, x=n * K * e, w=N * K * e, add=n * K * e, dx=n * K * e, gw=N * K * 4, gb=N * 4, ws=ws)
    for a, bad in cases(sizes, ("dx", "gw", "gb", "ws"), [("dx", "add")]):
        if a["ws"] % 256:
            continue
        expect(lib, lib.mem_linear_backward(a["dz"], a["x"], a["w"], dt, n, N, K, a["add"], a["dx"], a["gw"], a["gb"],
                                             a["ws"], ws, None), bad)
    a = dict(zip(sizes, PLACES))
    # dx alone uses no workspace
    expect(lib, lib.mem_linear_backward(a["dz"], a["x"], a["w"], dt, n, N, K, None, a["dx"], None, None, a["x"], ws, None), False)


def adamw(lib, tensors, **opts):
    ts = (pk._AdamwTensor * len(tensors))(*tensors)
    o = pk._AdamwOpts(1e-3, 0.9, 0.999, 1e-8, 0.1, 1, 0, **opts)
    return lib.mem_adamw(ctypes.addressof(ts), len(tensors), ctypes.addressof(o), None)


@pytest.mark.parametrize("gd", [F32, BF16])
@pytest.mark.parametrize("sd", [F32, E4M3])
def test_adamw(lib, gd, sd):
    n = 1024
    state, scale = (n, n // 128 * 4) if sd == E4M3 else (n * 4, 0)
    sizes = dict(param=n * 4, exp_avg=state, exp_avg_sq=state, grad=n * (4 if gd == F32 else 2), lr_dev=4, step_dev=8, grad_scale=4)
    if scale:
        sizes.update(exp_avg_scale=scale, exp_avg_sq_scale=scale)
    scalars = ("lr_dev", "step_dev", "grad_scale")
    far = pk._AdamwTensor(1 << 20, 1 << 21, 1 << 22, 1 << 23, None, None, 64, F32, F32, F32)
    for a, bad in cases(sizes, [w for w in sizes if w not in scalars and w != "grad"]):
        own = {k: v for k, v in a.items() if k not in scalars}
        if any(v % 16 for v in a.values()):
            continue
        t = pk._AdamwTensor(numel=n, param_dt=F32, grad_dt=gd, state_dt=sd, **own)
        expect(lib, adamw(lib, [far, t], **{k: a[k] for k in scalars}), bad)


def test_adamw_among_tensors(lib):
    """Gradients may be shared; one tensor's state over another's gradient may not."""
    make = lambda i, g: pk._AdamwTensor(PLACES[3 * i], g, PLACES[3 * i + 1], PLACES[3 * i + 2], None, None, 1000, F32, F32, F32)  # noqa: E731
    expect(lib, adamw(lib, [make(0, 1 << 50), make(1, 1 << 50), make(2, (1 << 50) + 400)]), False)
    for place in (PLACES[0], PLACES[1] + 3996, PLACES[2] - 3996):
        expect(lib, adamw(lib, [make(0, 1 << 50), make(1, place)]), True)
        expect(lib, adamw(lib, [make(1, place), make(2, 1 << 50), make(0, 1 << 50)]), True)
        assert "gradient" in lib.mem_last_error().decode()
    # a long gradient that begins in front of several short ones
    long = pk._AdamwTensor(1 << 55, 1 << 50, 1 << 56, 1 << 57, None, None, 1 << 20, F32, F32, F32)
    inside = pk._AdamwTensor((1 << 50) + (1 << 21), 1 << 51, 1 << 52, 1 << 53, None, None, 64, F32, F32, F32)
    expect(lib, adamw(lib, [long, make(0, (1 << 50) + 64), inside]), True)


def test_adamw_rows(lib):
    n, d, u = 64, 128, 32
    sizes = dict(param=n * d * 4, exp_avg=n * d, exp_avg_sq=n * d, exp_avg_scale=n * 4, exp_avg_sq_scale=n * 4,
                 grad=u * d * 4, rows=u * 8)
    for a, bad in cases(sizes, [w for w in sizes if w not in ("grad", "rows")]):
        t = pk._AdamwTensor(numel=n * d, param_dt=F32, grad_dt=F32, state_dt=E4M3, **{k: v for k, v in a.items() if k != "rows"})
        o = pk._AdamwOpts(1e-3, 0.9, 0.999, 1e-8, 0.1, 1, 0)
        expect(lib, lib.mem_adamw_rows(ctypes.addressof(t), n, d, a["rows"], u, ctypes.addressof(o), None), bad)
