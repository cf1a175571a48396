"""More operators of the blocks around a product-key memory, as timed cases.

  layernorm  layer norm of the residual stream, with the residual's addition; its
             backward with the gradients of weight and bias
  glu        the gated feed-forward part of a block: gate and up projection, activation
             and product in one call; its backward
  blocks     matrix product in 8-bit floating point with a scale for each 128 elements
             along k: the rounding to blocks (rows, columns, or 128 x 128 tiles of a
             weight), the product with its epilogue, and the products of a training step

`own` False computes them in elementary torch operations, `own` True through
paper_2412_09764_amd.  Sizes follow this library's workloads: streams of 64 to 2048
wide, 1 to 32768 tokens, hidden parts up to four times as wide.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
ESZ = {"f32": 4, "bf16": 2, "e4m3": 1}
E4M3_MAX = 448.0
BLOCK = 128  # elements that share a scale
EPS = 1e-5


# ------------------------------------------------------------------ cases ----
def _case(name, **c):
    return c if name is None else dict(name=name, **c)


def _norm(name, T, D, dtype="bf16", res=True, affine=True, bwd=False, shift=0.5):
    return _case(name, op="layernorm", T=T, D=D, dtype=dtype, res=res, affine=affine, bwd=bwd, shift=shift)


def _glu(name, do, T, N, K, dtype="bf16", act="silu", bias=False):
    return _case(name, op="glu", do=do, T=T, N=N, K=K, dtype=dtype, act=act, bias=bias)


def _blocks(name, do, T, N, K, dtype="bf16", out="bf16", act="none", bias=False, res=False, tile=True):
    return _case(name, op="blocks", do=do, T=T, N=N, K=K, dtype=dtype, out=out, act=act, bias=bias, res=res, tile=tile)


def listed():
    return [
        # one decoded token on the residual stream
        _norm("layernorm_t1", 1, 1024),
        # a small fp32 layer's training step at odd sizes
        _norm("layernorm_f32_train_t777", 777, 200, "f32", res=False, bwd=True),
        # the norm of a training step, forward and backward: 8 sequences x 4096 tokens
        _norm("layernorm_train_t32768", 32768, 2048, bwd=True),
        # one decoded token's feed-forward part, four times as wide as the stream
        _glu("glu_t1", "forward", 1, 8192, 2048),
        # a ragged prompt in 8 bits with a scale per row (the row norm's and the weights')
        _glu("glu_fp8_t2000", "forward", 2000, 8192, 2048, "e4m3"),
        # a training step of a feed-forward part: 4 sequences x 4096 tokens, forward and all gradients,
        # the weight's added up in fp32 and handed on (to the sum over the other cards) in bf16
        _glu("glu_train_t16384", "train", 16384, 4096, 1024),
        # the same in fp32 at odd sizes, with biases
        _glu("glu_f32_train_t777", "train", 777, 328, 200, "f32", act="gelu", bias=True),
        # one token's projection in 8 bits: the token is rounded, the weight is held in tiles
        _blocks("blocks_t1", "forward", 1, 2048, 2048, bias=True),
        # a ragged prompt's projection with its activation
        _blocks("blocks_t2000", "forward", 2000, 4096, 2048, act="silu"),
        # an output projection of 32768 tokens onto the residual stream
        _blocks("blocks_t32768", "forward", 32768, 2048, 2048, res=True),
        # a projection's training step: activations, weight and gradient rounded both ways,
        # product, gradient of the input, gradient of the weight added in fp32
        _blocks("blocks_train_t16384", "train", 16384, 2048, 1024),
        # a master weight laid out in 8 bits for the forward and the backward product, after an optimizer step
        _blocks("blocks_weight_8192", "weight", 0, 8192, 2048, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["layernorm", "glu", "glu", "blocks", "blocks"])
        T = _log(rng, 1, 32768)
        N = rng.choice([256, 1024, 2048, 16 * _log(rng, 4, 512), 16 * _log(rng, 4, 512)])
        K = rng.choice([256, 1024, 2048, 16 * _log(rng, 4, 256), 16 * _log(rng, 4, 256)])
        if op == "layernorm":
            D = rng.choice([64, 256, 1024, 2048, 8 * _log(rng, 8, 512), 8 * _log(rng, 8, 512)])
            dtype = rng.choice(["bf16", "bf16", "f32"])
            c = _norm(None, T, D, dtype, rng.random() < 0.6, rng.random() < 0.8, rng.random() < 0.5,
                      rng.choice([0.0, 0.5, 3.0]))
            if T * D * ESZ[dtype] > 32768 * 2048 * 2:
                continue
        elif op == "glu":
            do = rng.choice(["forward", "forward", "train"])
            dtype = rng.choice(["bf16", "bf16", "f32"] + (["e4m3", "e4m3"] if do == "forward" else []))
            c = _glu(None, do, T, N, K, dtype, rng.choice(["silu", "silu", "gelu", "relu", "none"]),
                     rng.random() < 0.4)
            if 2 * T * N * K * (1 if do == "forward" else 3) > 3 * 16384 * 8192 * 1024:
                continue
            if dtype == "f32" and T * N * K > 4096 * 2048 * 2048:
                continue
        else:
            do = rng.choice(["forward", "forward", "forward", "train", "weight"])
            out = rng.choice(["bf16", "bf16", "f32"])
            dtype = rng.choice(["bf16", "bf16", "f32"])
            act = rng.choice(["none", "none", "relu", "silu", "gelu"]) if do == "forward" else "none"
            c = _blocks(None, do, 0 if do == "weight" else T, N, K, dtype, out if do == "forward" else "bf16", act,
                        rng.random() < 0.5, do == "forward" and rng.random() < 0.4, do != "forward" or rng.random() < 0.8)
            if T * N * K * (1 if do == "forward" else 3) > 32768 * 2048 * 2048:
                continue
        return c


# ----------------------------------------------------------------- inputs ----
def _e4m3_rows(x):
    """Rows in 8 bits with one scale each, as a user's program holds them."""
    s = (x.abs().amax(-1) / E4M3_MAX).clamp_min(2.0 ** -126)
    return (x / s[:, None]).to(torch.float8_e4m3fn), s


def _out_type(c):
    if c["op"] == "blocks":
        return DT[c["out"]]
    return torch.bfloat16 if c["dtype"] == "e4m3" else DT[c["dtype"]]


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))

    def randn(shape, std=1.0):
        return torch.empty(shape, device=dev).normal_(0.0, std, generator=g)

    st = {"case": dict(c)}
    if c["op"] == "layernorm":
        T, D, dt = c["T"], c["D"], DT[c["dtype"]]
        st["x"] = (randn((T, D)) + c["shift"]).to(dt)
        st["res"] = randn((T, D), 2.0).to(dt) if c["res"] else None
        st["w"] = (1.0 + randn((D,), 0.1)).to(dt) if c["affine"] else None
        st["b"] = randn((D,), 0.1).to(dt) if c["affine"] else None
        if c["bwd"]:
            st["dy"] = randn((T, D)).to(dt)
            st["dsum"] = randn((T, D)).to(dt) if c["res"] else None
            st["gw"] = randn((D,)) if c["affine"] else None
            st["gb"] = randn((D,)) if c["affine"] else None
        return st
    T, N, K, ot = c["T"], c["N"], c["K"], _out_type(c)
    if c["op"] == "glu":
        # rows 0 .. N-1 of the weight are the gate's, N .. 2N-1 the up projection's
        x, w = randn((T, K)), randn((2 * N, K), 1.0 / math.sqrt(K))
        st["sx"] = st["sw"] = None
        if c["dtype"] == "e4m3":
            (st["x"], st["sx"]), (st["w"], st["sw"]) = _e4m3_rows(x), _e4m3_rows(w)
        else:
            st["x"], st["w"] = x.to(DT[c["dtype"]]), w.to(DT[c["dtype"]])
        st["bias"] = randn((2 * N,), 0.1).to(ot) if c["bias"] else None
        if c["do"] == "train":
            st["dy"] = randn((T, N)).to(ot)
            st["gW"] = randn((2 * N, K))
            st["gb"] = randn((2 * N,)) if c["bias"] else None
        return st
    # activations of uneven size along k, as after a norm with a weight
    st["x"] = (randn((T, K)) * torch.exp(randn((K,), 0.5))).to(DT[c["dtype"]])
    w = randn((N, K), 1.0 / math.sqrt(K))
    if c["do"] == "forward":  # the weight is held in 8 bits
        st["w"], st["sw"] = _to_blocks(w, c["tile"])
        st["bias"] = randn((N,), 0.1).to(ot) if c["bias"] else None
        st["res"] = randn((T, N)).to(ot) if c["res"] else None
    else:
        st["w"] = w.to(DT[c["dtype"]])
        if c["do"] == "train":
            st["bias"] = randn((N,), 0.1).to(ot) if c["bias"] else None
            st["dy"] = randn((T, N)).to(DT[c["dtype"]])
            st["gW"] = randn((N, K))
    return st


# ------------------------------------------------------------ plain forms ----
def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(z * -math.sqrt(0.5))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * torch.special.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _plain_norm(st):
    c, out = st["case"], {}
    dt = DT[c["dtype"]]
    h = st["x"].float()
    if c["res"]:  # the stream is stored in its type, and what is stored is normalised
        out["sum"] = (h + st["res"].float()).to(dt)
        h = out["sum"].float()
    d = h - h.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS)
    xh = d * rstd
    y = xh
    if c["affine"]:
        y = xh * st["w"].float() + st["b"].float()
    out["y"] = y.to(dt)
    if c["bwd"]:
        dy = st["dy"].float()
        g = dy * st["w"].float() if c["affine"] else dy
        dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
        if c["res"]:
            dx = dx + st["dsum"].float()
        out["dx"] = dx.to(dt)
        if c["affine"]:
            out["grad_weight"] = st["gw"].add_((dy * xh).sum(0))
            out["grad_bias"] = st["gb"].add_(dy.sum(0))
    return out


def _plain_glu(st):
    c, out = st["case"], {}
    N, ot = c["N"], _out_type(c)
    x, w = st["x"].float(), st["w"].float()
    z = x @ w.t()
    if c["dtype"] == "e4m3":
        z = z * st["sx"][:, None] * st["sw"]
    if c["bias"]:
        z = z + st["bias"].float()
    out["y"] = (_act(z[:, :N], c["act"]) * z[:, N:]).to(ot)
    if c["do"] == "train":
        out["z"] = z.to(ot)
        gate, up, dy = out["z"][:, :N].float(), out["z"][:, N:].float(), st["dy"].float()
        out["dz"] = torch.cat([dy * up * _act_grad(gate, c["act"]), dy * _act(gate, c["act"])], 1).to(ot)
        dz = out["dz"].float()
        out["dx"] = (dz @ w).to(ot)
        out["grad_w"] = st["gW"].add_(dz.t() @ x).to(ot)
        if c["bias"]:
            out["grad_bias"] = st["gb"].add_(dz.sum(0)).to(ot)
    return out


def _pad(x, rows, cols):
    """x with zeros up to whole blocks of rows and columns."""
    r, k = x.shape
    R, C = -(-r // rows) * rows, -(-k // cols) * cols
    if (R, C) == (r, k):
        return x
    p = torch.zeros((R, C), dtype=x.dtype, device=x.device)
    p[:r, :k] = x
    return p


def _to_blocks(x, tile=False):
    """x [R, C] in 8 bits with a scale for each 128 along C, or each 128 x 128: the codes, and
    the scales [ceil(C / 128), R] or [ceil(C / 128), ceil(R / 128)].  In 64 bits: a quotient
    next to the border between two codes decides."""
    R, C = x.shape
    rows = BLOCK if tile else 1
    p = _pad(x.double(), rows, BLOCK).contiguous()
    p = p.view(p.shape[0] // rows, rows, p.shape[1] // BLOCK, BLOCK)
    top = p.abs().amax((1, 3), keepdim=True)
    low = top < E4M3_MAX * 2.0 ** -126  # the scale is 2^-126 there
    v = torch.where(low, p * 2.0 ** 126, p * E4M3_MAX / torch.where(low, 1.0, top))
    # to the nearest of 3 bits of mantissa, and of multiples of 2^-9, ties to even
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    q = (torch.round(v / step) * step).view(p.shape[0] * rows, -1)[:R, :C]
    s = (top[:, 0, :, 0].float() / E4M3_MAX).clamp_min(2.0 ** -126)
    return q.float().to(torch.float8_e4m3fn).contiguous(), s.t().contiguous()


def _from_blocks(q, s, tile):
    """The numbers that codes and scales stand for, in 32 bits."""
    s = s.t().repeat_interleave(BLOCK, 1)
    if tile:
        s = s.repeat_interleave(BLOCK, 0)
    return q.float() * s[:q.shape[0], :q.shape[1]]


def _both_ways(x, tile):
    """x in blocks along its rows' direction and, transposed, along its columns'; the
    transposed codes have their k (x's rows) padded to whole 16."""
    q, s = _to_blocks(x, tile)
    qt, st = _to_blocks(_pad(x.t(), 1, 16), tile)
    return q, s, qt, st


def _plain_blocks(st):
    c, out = st["case"], {}
    ot = _out_type(c)
    if c["do"] == "weight":
        out["q"], out["scale"], out["qt"], out["scale_t"] = _both_ways(st["w"], True)
        return out
    if c["do"] == "forward":
        z = _from_blocks(*_to_blocks(st["x"]), False) @ _from_blocks(st["w"], st["sw"], c["tile"]).t()
        if c["bias"]:
            z = z + st["bias"].float()
        z = _act(z, c["act"])
        if c["res"]:
            z = z + st["res"].float()
        out["y"] = z.to(ot)
        return out
    xq, xs, xqt, xst = _both_ways(st["x"], False)
    wq, ws, wqt, wst = _both_ways(st["w"], True)
    dq, ds, dqt, dst = _both_ways(st["dy"], False)
    z = _from_blocks(xq, xs, False) @ _from_blocks(wq, ws, True).t()
    if c["bias"]:
        z = z + st["bias"].float()
    out["y"] = z.to(ot)
    K, N = c["K"], c["N"]
    out["dx"] = (_from_blocks(dq, ds, False) @ _from_blocks(wqt, wst, True)[:, :N].t()).to(ot)
    out["grad_w"] = st["gW"].add_(_from_blocks(dqt, dst, False) @ _from_blocks(xqt, xst, False).t())
    return out


# -------------------------------------------------- the framework's calls ----
def _own_norm(st):
    import paper_2412_09764_amd as pk
    c = st["case"]
    y, total = pk.mem_layernorm(st["x"], st["w"], st["b"], residual=st["res"], eps=EPS)
    out = {"y": y}
    if c["res"]:
        out["sum"] = total
    if c["bwd"]:
        dx, gw, gb = pk.mem_layernorm_backward(
            st["dy"], total if c["res"] else st["x"], st["w"], eps=EPS, dsum=st["dsum"], grad_weight=st["gw"],
            grad_bias=st["gb"], want_grad_weight=c["affine"], want_grad_bias=c["affine"])
        out["dx"] = dx
        if c["affine"]:
            out["grad_weight"], out["grad_bias"] = gw, gb
    return out


def _own_glu(st):
    import paper_2412_09764_amd as pk
    c, train = st["case"], st["case"]["do"] == "train"
    y, z = pk.mem_glu(st["x"], st["w"], st["bias"], act=c["act"], x_scale=st["sx"], w_scale=st["sw"], want_z=train)
    out = {"y": y}
    if train:
        out["z"] = z
        out["dz"] = pk.mem_glu_backward(st["dy"], z, c["act"])
        out["dx"], gW, gb = pk.mem_linear_backward(
            out["dz"], st["x"], st["w"], grad_w=st["gW"], grad_bias=st["gb"], want_grad_bias=c["bias"])
        out["grad_w"] = gW.to(z.dtype)
        if c["bias"]:
            out["grad_bias"] = gb.to(z.dtype)
    return out


def _own_blocks(st):
    import paper_2412_09764_amd as pk
    c, out = st["case"], {}
    ot = _out_type(c)
    if c["do"] == "weight":
        out["q"], out["scale"], out["qt"], out["scale_t"] = pk.mem_quantize_blocks(st["w"], tile=True, want_cols=True)
        return out
    if c["do"] == "forward":
        q, s, _, _ = pk.mem_quantize_blocks(st["x"])
        out["y"], _ = pk.mem_linear_blocks(q, st["w"], s, st["sw"], st["bias"], residual=st["res"], act=c["act"],
                                           out_dtype=ot)
        return out
    xq, xs, xqt, xst = pk.mem_quantize_blocks(st["x"], want_cols=True)
    wq, ws, wqt, wst = pk.mem_quantize_blocks(st["w"], tile=True, want_cols=True)
    dq, ds, dqt, dst = pk.mem_quantize_blocks(st["dy"], want_cols=True)
    out["y"], _ = pk.mem_linear_blocks(xq, wq, xs, ws, st["bias"], out_dtype=ot)
    out["dx"], _ = pk.mem_linear_blocks(dq, wqt, ds, wst, out_dtype=ot)
    out["grad_w"], _ = pk.mem_linear_blocks(dqt, xqt, dst, xst, residual=st["gW"], y_out=st["gW"],
                                            out_dtype=torch.float32)
    return out


def run(state):
    op = state["case"]["op"]
    if op == "layernorm":
        return _own_norm(state) if own else _plain_norm(state)
    if op == "glu":
        return _own_glu(state) if own else _plain_glu(state)
    return _own_blocks(state) if own else _plain_blocks(state)


# ------------------------------------------------------------------- work ----
def work(case):
    c = case
    e = ESZ[c["dtype"]]
    if c["op"] == "layernorm":
        T, D = c["T"], c["D"]
        b = T * D * e * (4 if c["res"] else 2) + (2 * D * e if c["affine"] else 0)
        f = 8.0 * T * D
        if c["bwd"]:  # dy, dsum, dx; the gradients read and written
            b += T * D * e * (2 + c["res"]) + (16 * D if c["affine"] else 0)
            f += 16.0 * T * D
        return {"bytes": float(b), "flops": f}
    T, N, K = c["T"], c["N"], c["K"]
    o = 4 if _out_type(c) is torch.float32 else 2
    if c["op"] == "glu":
        b = (T + 2 * N) * K * e + T * N * o + (2 * N * o if c["bias"] else 0)
        if c["dtype"] == "e4m3":
            b += 4 * (T + 2 * N)
        f = 4.0 * T * N * K
        if c["do"] == "train":  # z, dz and dx written, dy read, the gradients read and written
            b += T * N * o * 5 + T * K * o + 2 * N * K * (8 + o % 4) + (2 * N * (8 + o % 4) if c["bias"] else 0)
            f *= 3
        return {"bytes": float(b), "flops": f}
    kb, nb, tb = -(-K // BLOCK), -(-N // BLOCK), -(-T // BLOCK)
    if c["do"] == "weight":
        return {"bytes": float(N * K * (e + 2) + 8 * kb * nb), "flops": 4.0 * N * K}
    if c["do"] == "forward":
        b = T * K * e + N * K + 4 * kb * (nb if c["tile"] else N) + T * N * o * (1 + c["res"]) + (N * o if c["bias"] else 0)
        return {"bytes": float(b), "flops": 2.0 * T * N * K}
    b = (T * K + N * K + T * N) * e + T * (N + K) * o + N * K * 8 + (N * o if c["bias"] else 0)
    return {"bytes": float(b), "flops": 6.0 * T * N * K}


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


def _exact_blocks(x, rows):
    """(codes, scale of each element, scales) of x in blocks of `rows` x 128, in 64 bits, by
    a search among the 8-bit numbers."""
    R, C = x.shape
    dev = x.device
    nums = torch.arange(127, device=dev, dtype=torch.uint8).view(torch.float8_e4m3fn).double()  # 0 .. 448
    rb, cb = -(-R // rows), -(-C // BLOCK)
    x = x.double()
    a = torch.zeros((rb * rows, cb * BLOCK), dtype=torch.float64, device=dev)
    a[:R, :C] = x.abs()
    top = a.view(rb, rows, cb, BLOCK).amax(3).amax(1)
    scale = (top / 448).clamp(min=2.0 ** -126)
    each = scale.repeat_interleave(rows, 0)[:R].repeat_interleave(BLOCK, 1)[:, :C]
    big = top.repeat_interleave(rows, 0)[:R].repeat_interleave(BLOCK, 1)[:, :C]
    v = torch.where(each > 2.0 ** -126, x.abs() * 448 / big.clamp(min=2.0 ** -149), x.abs() / each)
    del a, big
    mid = (nums[1:] + nums[:-1]) / 2
    hi = torch.searchsorted(mid, v, right=True)  # a value on the border counts as above it here
    tie = (hi > 0) & (v == mid[(hi - 1).clamp(min=0)])
    hi = torch.where(tie & (hi % 2 == 1), hi - 1, hi)  # the even code of the two
    return torch.sign(x) * nums[hi], each, scale.t()


def exact(case, seed):
    c, st, out = case, prepare(case, seed), {}
    if c["op"] == "layernorm":
        dt, D = DT[c["dtype"]], c["D"]
        h = st["x"].double()
        if c["res"]:
            out["sum"] = h + st["res"].double()
            h = out["sum"].to(dt).double()
        var, mean = torch.var_mean(h, -1, correction=0, keepdim=True)
        inv = torch.rsqrt(var + EPS)
        xh = (h - mean) * inv
        out["y"] = torch.addcmul(st["b"].double(), xh, st["w"].double()) if c["affine"] else xh
        if c["bwd"]:
            dy = st["dy"].double()
            g = dy * st["w"].double() if c["affine"] else dy
            dx = (D * g - g.sum(-1, keepdim=True) - xh * (g * xh).sum(-1, keepdim=True)) * (inv / D)
            out["dx"] = dx + st["dsum"].double() if c["res"] else dx
            if c["affine"]:
                out["grad_weight"] = st["gw"].double() + (dy * xh).sum(0)
                out["grad_bias"] = st["gb"].double() + dy.sum(0)
        return out
    N, K = c["N"], c["K"]
    if c["op"] == "glu":
        x, w = st["x"].double(), st["w"].double()
        if c["dtype"] == "e4m3":
            x, w = x * st["sx"].double()[:, None], w * st["sw"].double()[:, None]
        gate, up = torch.mm(x, w[:N].t()), torch.mm(x, w[N:].t())
        if c["bias"]:
            gate += st["bias"][:N].double()
            up += st["bias"][N:].double()
        out["y"] = _exact_act(gate, c["act"])[0] * up
        if c["do"] == "train":  # z and dz are stored in their type, and what is stored goes on
            dy, ot = st["dy"].double(), _out_type(c)
            out["z"] = torch.cat([gate, up], 1)
            gate, up = gate.to(ot).double(), up.to(ot).double()
            a, d = _exact_act(gate, c["act"])
            dg, du = dy * up * d, dy * a
            out["dz"] = torch.cat([dg, du], 1)
            dg, du = dg.to(ot).double(), du.to(ot).double()
            out["dx"] = torch.mm(dg, w[:N]) + torch.mm(du, w[N:])
            out["grad_w"] = st["gW"].double() + torch.cat([torch.mm(dg.t(), x), torch.mm(du.t(), x)])
            if c["bias"]:
                out["grad_bias"] = st["gb"].double() + torch.cat([dg.sum(0), du.sum(0)])
        return out
    if c["do"] == "weight":
        q, _, s = _exact_blocks(st["w"], BLOCK)
        out["q"], out["scale"] = q, s
        qt = torch.zeros((K, -(-N // 16) * 16), dtype=torch.float64, device=q.device)
        qt[:, :N] = q.t()
        out["qt"], out["scale_t"] = qt, s.t()
        return out

    def values(x, rows):
        q, each, _ = _exact_blocks(x, rows)
        return q * each

    def held(q, s):  # the weight's codes and scales
        each = s.double().t().repeat_interleave(BLOCK, 1)
        if c["tile"]:
            each = each.repeat_interleave(BLOCK, 0)
        return q.double() * each[:N, :K]

    if c["do"] == "forward":
        z = torch.mm(values(st["x"], 1), held(st["w"], st["sw"]).t())
        if c["bias"]:
            z += st["bias"].double()
        out["y"] = _exact_act(z, c["act"])[0]
        if c["res"]:
            out["y"] = out["y"] + st["res"].double()
        return out
    w = values(st["w"], BLOCK)
    out["y"] = torch.mm(values(st["x"], 1), w.t())
    if c["bias"]:
        out["y"] += st["bias"].double()
    out["dx"] = torch.mm(values(st["dy"], 1), w)
    out["grad_w"] = st["gW"].double() + torch.mm(values(st["dy"].t(), 1), values(st["x"].t(), 1).t())
    return out
