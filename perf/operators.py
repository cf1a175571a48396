"""The operators around the product-key memory of a Memory+ block, as timed cases.

  norm      root-mean-square norm of the residual stream, with the residual's
            addition and an output in 8 bits with a scale per row; its backward
  linear    the block's projections: matrix product with bias, activation and
            residual in its epilogue; the backward of the product
  adamw     AdamW over many tensors at once, or over the touched rows of a value
            table, with states in 32 bits or in 8 bits with a scale per 128

`own` False computes them in elementary torch operations, `own` True through
paper_2412_09764_amd.  Sizes follow this library's workloads: value dims 64 to
2048, H * n up to 2048, 1 to 32768 tokens, tables of 4K to 1M rows.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
ESZ = {"f32": 4, "bf16": 2, "e4m3": 1}
E4M3_MAX = 448.0
BLOCK = 128  # elements that share one scale of an 8-bit state
M32 = 0xFFFFFFFF


# ------------------------------------------------------------------ cases ----
def _norm(name, T, D, dtype="bf16", res=True, quant=False, bwd=False):
    c = dict(op="norm", T=T, D=D, dtype=dtype, res=res, quant=quant, bwd=bwd)
    return c if name is None else dict(name=name, **c)


def _linear(name, do, T, N, K, dtype="bf16", act="none", bias=True, res=False):
    c = dict(op="linear", do=do, T=T, N=N, K=K, dtype=dtype, act=act, bias=bias, res=res)
    return c if name is None else dict(name=name, **c)


def _adamw(name, do, shapes, dtype="f32", bits=32, U=0, grad="f32", step=100):
    c = dict(op="adamw", do=do, shapes=shapes, dtype=dtype, bits=bits, U=U, grad=grad, step=step)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # one decoded token: the smallest call of all
        _norm("norm_t1", 1, 1024),
        # a ragged prompt normalised for 8-bit projections
        _norm("norm_fp8_t2000", 2000, 2048, quant=True),
        # the norm of a training step, forward and backward: 8 sequences x 4096 tokens
        _norm("norm_train_t32768", 32768, 2048, bwd=True),
        # one token's query projection (4 heads x 512) with its bias
        _linear("linear_t1", "forward", 1, 2048, 2048),
        # 8-bit gate projection of a ragged prompt with the activation fused
        _linear("linear_fp8_t2000", "forward", 2000, 2048, 2048, "e4m3", act="silu"),
        # the output projection of 32768 tokens onto the residual stream
        _linear("linear_t32768", "forward", 32768, 2048, 2048, bias=False, res=True),
        # the query projection's gradients at the 1M-key training workload
        _linear("linear_bwd_t16384", "backward", 16384, 2048, 1024),
        # a whole training step of an fp32 layer at odd sizes
        _linear("linear_f32_train_t777", "train", 777, 192, 200, "f32", act="gelu", res=True),
        # every small parameter of a layer: sub-keys, projections, sink keys, norms, biases
        _adamw("adamw_layer", "many", "4x2x1024x256,2048x1024,1024x1024,1024x1024,4x512,1024,2048,1024,777,1"),
        # a bf16 value table with a dense fp32 gradient: 256K rows x 2048, 8-bit states
        _adamw("adamw_table_8bit", "many", "262144x2048", "bf16", 8),
        # the touched rows of a 1M x 1024 table after 16384 tokens
        _adamw("adamw_rows_8bit", "rows", "1048576x1024", "bf16", 8, U=400001),
        # touched rows of the small fp32 configuration
        _adamw("adamw_rows_f32", "rows", "4096x64", "f32", 32, U=1601),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["norm", "norm", "linear", "linear", "linear", "adamw", "adamw"])
        if op == "norm":
            T = _log(rng, 1, 32768)
            D = rng.choice([64, 256, 1024, 2048, 8 * _log(rng, 8, 512)])
            dtype = rng.choice(["bf16", "bf16", "f32"])
            bwd = rng.random() < 0.4
            c = _norm(None, T, D, dtype, rng.random() < 0.6, not bwd and rng.random() < 0.4, bwd)
            if T * D * ESZ[dtype] > 32768 * 2048 * 2:
                continue
        elif op == "linear":
            do = rng.choice(["forward", "forward", "forward", "backward", "train"])
            dtype = rng.choice(["bf16", "bf16", "f32"] + (["e4m3", "e4m3"] if do == "forward" else []))
            if do == "train":
                dtype = "f32"
            T = _log(rng, 1, 32768)
            N = rng.choice([256, 512, 1024, 2048, 16 * _log(rng, 4, 256)])
            K = rng.choice([256, 512, 1024, 2048, 16 * _log(rng, 4, 256)])
            act = "none" if do == "backward" else rng.choice(["none", "relu", "silu", "gelu"])
            c = _linear(None, do, T, N, K, dtype, act, rng.random() < 0.6,
                        do != "backward" and rng.random() < 0.4)
            if T * N * K * (1 if do == "forward" else 2) > 32768 * 2048 * 2048:
                continue
            if dtype == "f32" and T * N * K > 4096 * 2048 * 2048:
                continue
        else:
            do = rng.choice(["many", "many", "rows"])
            dtype, bits = rng.choice([("f32", 32), ("f32", 8), ("bf16", 8), ("bf16", 32)])
            step = _log(rng, 1, 100000)
            if do == "many":
                sizes = [_log(rng, 1, 1 << 22) for _ in range(rng.randint(1, 40))]
                if rng.random() < 0.3:
                    sizes.append(_log(rng, 1 << 22, 1 << 27))
                c = _adamw(None, do, ",".join(map(str, sizes)), dtype, bits,
                           grad=rng.choice(["f32", "f32", "bf16"]), step=step)
            else:
                N = _log(rng, 64, 1 << 20)
                D = rng.choice([128, 256, 640, 1024, 2048]) if bits == 8 else 8 * _log(rng, 8, 256)
                if N * D > 1 << 29:
                    continue
                c = _adamw(None, do, "%dx%d" % (N, D), dtype, bits, U=_log(rng, 1, min(N, 400000)), step=step)
        return c


def _shapes(c):
    return [tuple(int(x) for x in s.split("x")) for s in c["shapes"].split(",")]


def _hyper(c):
    """What the optimizer's call is told: rates of a training run's middle."""
    return dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1, step=c["step"], seed=1234567 + c["step"])


# ----------------------------------------------------------------- inputs ----
def _e4m3_rows(x):
    """Rows in 8 bits and their scales, as a user's program holds quantised weights."""
    s = (x.abs().amax(-1) / E4M3_MAX).clamp_min(2.0 ** -126)
    return (x / s[:, None]).to(torch.float8_e4m3fn), s


def _e4m3_blocks(x):
    n = x.numel()
    pad = torch.zeros(-(-n // BLOCK) * BLOCK, device=x.device)
    pad[:n] = x.reshape(-1)
    q, s = _e4m3_rows(pad.view(-1, BLOCK))
    return q.view(-1)[:n].clone().view(x.shape), s


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))

    def randn(shape, std=1.0):
        return torch.empty(shape, device=dev).normal_(0.0, std, generator=g)

    st = {"case": dict(c)}
    if c["op"] == "norm":
        T, D, dt = c["T"], c["D"], DT[c["dtype"]]
        st["x"] = randn((T, D)).to(dt)
        st["res"] = randn((T, D), 2.0).to(dt) if c["res"] else None
        st["w"] = (1.0 + randn((D,), 0.1)).to(dt)
        if c["bwd"]:
            st["dy"] = randn((T, D)).to(dt)
            st["dsum"] = randn((T, D)).to(dt) if c["res"] else None
            st["gw"] = torch.zeros((D,), device=dev)
        return st
    if c["op"] == "linear":
        T, N, K, dt = c["T"], c["N"], c["K"], DT[c["dtype"]]
        x, w = randn((T, K)), randn((N, K), 1.0 / math.sqrt(K))
        ot = torch.bfloat16 if c["dtype"] == "e4m3" else dt
        if c["dtype"] == "e4m3":
            (st["x"], st["sx"]), (st["w"], st["sw"]) = _e4m3_rows(x), _e4m3_rows(w)
        else:
            st["x"], st["w"], st["sx"], st["sw"] = x.to(dt), w.to(dt), None, None
        if c["do"] != "backward":
            st["bias"] = randn((N,), 0.1).to(ot) if c["bias"] else None
            st["res"] = randn((T, N)).to(ot) if c["res"] else None
        if c["do"] != "forward":
            st["dy"] = randn((T, N)).to(dt)
            st["gW"] = torch.zeros((N, K), device=dev)
            st["gb"] = torch.zeros((N,), device=dev) if c["bias"] else None
        return st
    dt = DT[c["dtype"]]
    shapes = _shapes(c)
    for name in ("p", "g", "m", "v", "sm", "sv"):
        st[name] = []
    for s in shapes:
        st["p"].append(randn(s, 0.02).to(dt))
        m, v = randn(s, 3e-4), randn(s, 1e-3).square_().add_(1e-9)
        if c["bits"] == 8:  # the second state is held as its square root
            m, sm = _e4m3_blocks(m)
            v, sv = _e4m3_blocks(v.sqrt_())
            st["sm"].append(sm)
            st["sv"].append(sv)
        st["m"].append(m)
        st["v"].append(v)
        if c["do"] == "many":
            st["g"].append(randn(s, 1e-3).to(DT[c["grad"]]))
    if c["do"] == "rows":
        N, D = shapes[0]
        st["rows"] = torch.randperm(N, generator=g, device=dev)[:c["U"]].sort().values
        st["g"] = randn((c["U"], D), 1e-3)
    return st


# ------------------------------------------------------------ plain forms ----
def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _plain_norm(st):
    c = st["case"]
    dt = DT[c["dtype"]]
    x, w = st["x"].float(), st["w"].float()
    out = {}
    if c["res"]:  # the stream is stored in its type, and what is stored is normalised
        out["sum"] = (x + st["res"].float()).to(dt)
        x = out["sum"].float()
    rstd = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
    xh = x * rstd
    y = xh * w
    if c["quant"]:
        out["y"], out["scale"] = _e4m3_rows(y)
    else:
        out["y"] = y.to(dt)
    if c["bwd"]:
        dy = st["dy"].float()
        g = dy * w
        dx = rstd * (g - xh * (g * xh).mean(-1, keepdim=True))
        if c["res"]:
            dx = dx + st["dsum"].float()
        out["dx"] = dx.to(dt)
        out["grad_weight"] = st["gw"].add_((dy * xh).sum(0))
    return out


def _plain_linear(st):
    c = st["case"]
    x, w, out = st["x"].float(), st["w"].float(), {}
    ot = torch.bfloat16 if c["dtype"] == "e4m3" else DT[c["dtype"]]
    dz = st.get("dy")
    if c["do"] != "backward":
        z = x @ w.t()
        if c["dtype"] == "e4m3":
            z = z * st["sx"][:, None] * st["sw"]
        if c["bias"]:
            z = z + st["bias"].float()
        y = _act(z, c["act"])
        if c["res"]:
            y = y + st["res"].float()
        out["y"] = y.to(ot)
        if c["do"] == "train":
            out["z"] = z.to(ot)
            dz = out["dz"] = (dz.float() * _act_grad(out["z"].float(), c["act"])).to(ot)
    if c["do"] != "forward":
        dz = dz.float()
        out["dx"] = (dz @ w).to(ot)
        out["grad_w"] = st["gW"].add_(dz.t() @ x)
        if c["bias"]:
            out["grad_bias"] = st["gb"].add_(dz.sum(0))
    return out


def _mix32(x):
    """A 32-bit mix of a tensor of numbers below 2^32, or of one number."""
    x = (x ^ (x >> 16)) * 0x6A09E667 & M32
    x = (x ^ (x >> 15)) * 0xBB67AE85 & M32
    return x ^ (x >> 16)


def _key(seed, step, tensor):
    k = _mix32(_mix32(_mix32(seed & M32) + (seed >> 32 & M32) & M32) + (step & M32) & M32)
    return k + tensor * 0x9E3779B1 & M32


def _random_bits(at, key):
    """32 random bits for the elements at the given places of a tensor."""
    return _mix32(((at & M32) + key & M32) ^ ((at >> 32) * 0x3C6EF373 & M32)).to(torch.int32)


def _round_bf16(p, h):
    """p to bf16, up with the probability of what is cut off: 12 bits of h decide."""
    up = ((p.view(torch.int32) + (((h & 0xFFF) << 4) | 8)) & -65536).view(torch.float32)
    return torch.where(torch.isfinite(p), up, p).to(torch.bfloat16)


def _round_e4m3(x, more, nonzero):
    """x (blocks of 128) to 8 bits and a scale, up with the probability of what is cut off."""
    finite = torch.isfinite(x)
    s = torch.where(finite, x.abs(), 0).amax(-1) / E4M3_MAX
    s = torch.where(s < 2.0 ** -126, 0, s)
    a = (x * torch.where(s > 0, 1 / s, 0)[:, None]).abs()
    low = a < 2.0 ** -6
    b = torch.where(low, a + 2.0 ** -6, a)
    b = ((b.view(torch.int32) + more) & -(1 << 20)).view(torch.float32)
    b = torch.where(low, b - 2.0 ** -6, b).clamp_max(E4M3_MAX)
    if nonzero:  # a root of 0 below a first state that is not 0 would blow the update up
        b = torch.where((a > 0) & (b == 0), 2.0 ** -9, b)
    b = torch.where(finite, torch.copysign(b, x), float("nan"))
    return b.to(torch.float8_e4m3fn), s


def _blocks(x):
    n = x.numel()
    if n % BLOCK == 0:
        return x.reshape(-1, BLOCK)
    pad = torch.zeros(-(-n // BLOCK) * BLOCK, dtype=x.dtype, device=x.device)
    pad[:n] = x.reshape(-1)
    return pad.view(-1, BLOCK)


def _plain_step(p, g, m, v, sm, sv, at, key, c):
    """One tensor's new (p, m, v, sm, sv); `at`: the places of its elements."""
    h = _hyper(c)
    b1, b2 = h["betas"]
    t, lr = h["step"], h["lr"]
    shape, n = p.shape, p.numel()
    g, p0 = g.float().reshape(-1), p.float().reshape(-1)
    if c["bits"] == 8:
        m = (_blocks(m.float()) * sm[:, None]).reshape(-1)[:n]
        r = (_blocks(v.float()) * sv[:, None]).reshape(-1)[:n]
        v = r * r
    m, v = m.reshape(-1) * b1 + g * (1 - b1), v.reshape(-1) * b2 + (g * g) * (1 - b2)
    r = torch.sqrt(v)
    new = p0 * (1 - lr * h["weight_decay"]) - (m / (r * (1 / math.sqrt(1 - b2 ** t)) + h["eps"])) * (lr / (1 - b1 ** t))
    bits = _random_bits(at.reshape(-1), key) if c["bits"] == 8 or p.dtype == torch.bfloat16 else None
    new = (_round_bf16(new, bits) if p.dtype == torch.bfloat16 else new).view(shape)
    if c["bits"] == 8:
        bits = _blocks(bits)
        m, sm = _round_e4m3(_blocks(m), ((bits >> 24 & 0xFF) << 12) | (1 << 11), False)
        v, sv = _round_e4m3(_blocks(r), ((bits >> 12 & 0xFFF) << 8) | (1 << 7), True)
        m, v = m.view(-1)[:n], v.view(-1)[:n]
    return new, m.view(shape), v.view(shape), sm, sv


def _plain_adamw(st):
    c = st["case"]
    h = _hyper(c)
    if c["do"] == "rows":
        p, m, v, rows = st["p"][0], st["m"][0], st["v"][0], st["rows"]
        D = p.shape[1]
        at = rows[:, None] * D + torch.arange(D, device=p.device)
        sm = sv = None
        if c["bits"] == 8:
            sm, sv = (s.view(-1, D // BLOCK) for s in (st["sm"][0], st["sv"][0]))
        got = _plain_step(p[rows], st["g"], m.view(torch.uint8)[rows].view(m.dtype) if c["bits"] == 8 else m[rows],
                          v.view(torch.uint8)[rows].view(v.dtype) if c["bits"] == 8 else v[rows],
                          None if sm is None else sm[rows].view(-1), None if sv is None else sv[rows].view(-1),
                          at, _key(h["seed"], h["step"], 0), c)
        p[rows] = got[0]
        if c["bits"] == 8:
            m.view(torch.uint8)[rows] = got[1].view(torch.uint8)
            v.view(torch.uint8)[rows] = got[2].view(torch.uint8)
            sm[rows], sv[rows] = got[3].view(-1, D // BLOCK), got[4].view(-1, D // BLOCK)
        else:
            m[rows], v[rows] = got[1], got[2]
        return
    for i, p in enumerate(st["p"]):
        at = torch.arange(p.numel(), device=p.device)
        sm, sv = (st["sm"][i], st["sv"][i]) if c["bits"] == 8 else (None, None)
        got = _plain_step(p, st["g"][i], st["m"][i], st["v"][i], sm, sv, at, _key(h["seed"], h["step"], i), c)
        for name, x in zip(("p", "m", "v", "sm", "sv"), got):
            if x is not None:
                st[name][i].copy_(x)


# -------------------------------------------------- the framework's calls ----
def _own_norm(st):
    import paper_2412_09764_amd as pk
    c = st["case"]
    y, total, scale = pk.mem_rmsnorm(st["x"], st["w"], residual=st["res"], eps=1e-5, quantize=c["quant"])
    out = {"y": y}
    if c["res"]:
        out["sum"] = total
    if c["quant"]:
        out["scale"] = scale
    if c["bwd"]:
        out["dx"], out["grad_weight"] = pk.mem_rmsnorm_backward(
            st["dy"], total if c["res"] else st["x"], st["w"], eps=1e-5, dsum=st["dsum"], grad_weight=st["gw"])
    return out


def _own_linear(st):
    import paper_2412_09764_amd as pk
    c, out = st["case"], {}
    dz = st.get("dy")
    if c["do"] != "backward":
        y, z = pk.mem_linear(st["x"], st["w"], st["bias"], residual=st["res"], act=c["act"], x_scale=st["sx"],
                             w_scale=st["sw"], want_z=c["do"] == "train")
        out["y"] = y
        if c["do"] == "train":
            out["z"] = z
            dz = out["dz"] = pk.mem_act_backward(dz, z, c["act"])
    if c["do"] != "forward":
        dx, gW, gb = pk.mem_linear_backward(dz, st["x"], st["w"], grad_w=st["gW"], grad_bias=st["gb"],
                                            want_grad_bias=c["bias"])
        out["dx"], out["grad_w"] = dx, gW
        if c["bias"]:
            out["grad_bias"] = gb
    return out


def _own_adamw(st):
    import paper_2412_09764_amd as pk
    c = st["case"]
    if c["do"] == "rows":
        more = dict(exp_avg_scale=st["sm"][0], exp_avg_sq_scale=st["sv"][0]) if c["bits"] == 8 else {}
        pk.mem_adamw_rows(st["p"][0], st["rows"], st["g"], st["m"][0], st["v"][0], **more, **_hyper(c))
    else:
        more = dict(exp_avg_scales=st["sm"], exp_avg_sq_scales=st["sv"]) if c["bits"] == 8 else {}
        pk.mem_adamw(st["p"], st["g"], st["m"], st["v"], **more, **_hyper(c))


def run(state):
    op = state["case"]["op"]
    if op == "norm":
        return _own_norm(state) if own else _plain_norm(state)
    if op == "linear":
        return _own_linear(state) if own else _plain_linear(state)
    if own:
        _own_adamw(state)
    else:
        _plain_adamw(state)
    if state["case"]["do"] == "many" and len(state["p"]) > 12:
        # many small tensors: each kind whole, as one
        return {k: torch.cat([x.reshape(-1).view(torch.uint8) if x.element_size() == 1 else x.reshape(-1)
                              for x in state[k]]).view(state[k][0].dtype) for k in ("p", "m", "v", "sm", "sv") if state[k]}
    return {k: state[k] for k in ("p", "m", "v", "sm", "sv")}


# ------------------------------------------------------------------- work ----
def work(case):
    c = case
    e = ESZ[c["dtype"]]
    if c["op"] == "norm":
        T, D = c["T"], c["D"]
        b = T * D * (e * (3 if c["res"] else 1) + (1 if c["quant"] else e)) + D * e + (4 * T if c["quant"] else 0)
        f = 5.0 * T * D
        if c["bwd"]:  # dy, dsum, dx; grad_weight read and written
            b += T * D * e * (2 + c["res"]) + D * 8
            f += 10.0 * T * D
        return {"bytes": float(b), "flops": f}
    if c["op"] == "linear":
        T, N, K, do = c["T"], c["N"], c["K"], c["do"]
        o = 2 if c["dtype"] == "e4m3" else e
        b = (T + N) * K * e
        f = 0.0
        if c["dtype"] == "e4m3":
            b += 4 * (T + N)
        if do != "backward":
            b += T * N * o * (1 + c["res"]) + (N * o if c["bias"] else 0)
            f += 2.0 * T * N * K
        if do == "train":
            b += T * N * o * 2
        if do != "forward":
            b += T * N * e + T * K * e + N * K * 8 + (N * 8 if c["bias"] else 0)
            f += 4.0 * T * N * K
        return {"bytes": float(b), "flops": f}
    n = sum(math.prod(s) for s in _shapes(c))
    if c["do"] == "rows":
        n = c["U"] * _shapes(c)[0][1]
    states = 16.0 if c["bits"] == 32 else 4.0 + 16.0 / BLOCK
    b = n * (2 * e + (4 if c["do"] == "rows" else ESZ[c["grad"]]) + states) + 8 * c["U"]
    return {"bytes": float(b), "flops": 15.0 * n}


# ------------------------------------------------------------------ exact ----
def _exact_act(z, act):
    """The activation and its derivative."""
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


def exact(case, seed):
    c, st, out = case, prepare(case, seed), {}
    if c["op"] == "norm":
        dt = DT[c["dtype"]]
        h, w = st["x"].double(), st["w"].double()
        if c["res"]:
            out["sum"] = h + st["res"].double()
            h = out["sum"].to(dt).double()
        inv = torch.rsqrt(h.square().mean(-1) + 1e-5)[:, None]
        y = h * inv * w
        if c["quant"]:
            out["scale"] = y.abs().amax(-1) / E4M3_MAX
            out["y"] = (y / out["scale"][:, None]).float().to(torch.float8_e4m3fn).double()
        else:
            out["y"] = y
        if c["bwd"]:
            dy = st["dy"].double()
            D = c["D"]
            gh = dy * w
            dot = (gh * h).sum(-1, keepdim=True)
            dx = gh * inv - h * dot * inv ** 3 / D
            out["dx"] = dx + st["dsum"].double() if c["res"] else dx
            out["grad_weight"] = (dy * h * inv).sum(0)
        return out
    if c["op"] == "linear":
        x, w = st["x"].double(), st["w"].double()
        if c["dtype"] == "e4m3":
            x, w = x * st["sx"].double()[:, None], w * st["sw"].double()[:, None]
        dz = st["dy"].double() if c["do"] != "forward" else None
        if c["do"] != "backward":
            z = torch.mm(x, w.t())
            if c["bias"]:
                z += st["bias"].double()
            out["y"], d = _exact_act(z, c["act"])
            if c["res"]:
                out["y"] = out["y"] + st["res"].double()
            if c["do"] == "train":
                out["z"] = z
                dz = out["dz"] = dz * d
        if c["do"] != "forward":
            out["dx"] = torch.mm(dz, w)
            out["grad_w"] = torch.mm(dz.t(), x)
            if c["bias"]:
                out["grad_bias"] = dz.sum(0)
        return out
    h = _hyper(c)
    b1, b2 = h["betas"]
    ps, ms, vs = [], [], []
    for i, p in enumerate(st["p"]):
        rows = st["rows"] if c["do"] == "rows" else slice(None)
        whole, m, v = p.double(), st["m"][i], st["v"][i]
        if c["bits"] == 8:
            def values(code, s):
                n = code.numel()
                full = torch.zeros(s.numel() * BLOCK, dtype=torch.float64, device=code.device)
                full[:n] = code.reshape(-1).double()
                return (full.view(-1, BLOCK) * s.double()[:, None]).view(-1)[:n].view(code.shape)
            m, v = values(m, st["sm"][i]), values(v, st["sv"][i]).square()
        m, v = m.double(), v.double()
        g = st["g"].double() if c["do"] == "rows" else st["g"][i].double()
        m1 = b1 * m[rows] + (1 - b1) * g
        v1 = b2 * v[rows] + (1 - b2) * g * g
        mhat, vhat = m1 / (1 - b1 ** h["step"]), v1 / (1 - b2 ** h["step"])
        old = whole[rows]
        whole[rows] = old - h["lr"] * (mhat / (vhat.sqrt() + h["eps"]) + h["weight_decay"] * old)
        m[rows], v[rows] = m1, v1
        ps.append(whole)
        ms.append(m)
        vs.append(v)
    if c["bits"] == 8:  # which way a state is rounded is drawn: no value of its own in 64 bits
        ms, vs = [None] * len(ps), [None] * len(ps)
    none = [None] * len(ps)
    if c["do"] == "many" and len(ps) > 12:
        cat = lambda v: None if v[0] is None else torch.cat([x.reshape(-1) for x in v])  # noqa: E731
        return {"p": cat(ps), "m": cat(ms), "v": cat(vs), "sm": None, "sv": None}
    return {"p": ps, "m": ms, "v": vs, "sm": none, "sv": none}
