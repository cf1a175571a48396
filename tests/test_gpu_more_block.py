"""Layer norm, gated part and products in 8-bit blocks together, as a block's feed-forward half
uses them: a training step against fp64 autograd, the same step on a side stream, captured
and replayed, two captured steps at once, the 8-bit forward and step; then sizes whose
offsets pass 32 bits and more work than one launch holds."""
import pytest
import torch

import paper_2412_09764_amd as pk
from tests.test_gpu_blocks import spread

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


class Half:
    """layernorm(x + res) -> gated part -> output projection added to the stream."""

    def __init__(self, T, D, N, dt, seed=0, act="silu"):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).to(dt).to(DEV)  # noqa: E731
        self.T, self.D, self.N, self.dt, self.act = T, D, N, dt, act
        self.x, self.res, self.dout = r(T, D) + 1, r(T, D), r(T, D)
        self.p = dict(w=1 + r(D, std=0.1), b=r(D, std=0.1), wi=r(2 * N, D, std=D ** -0.5), bi=r(2 * N, std=0.1),
                      wo=r(D, N, std=N ** -0.5))

    def buffers(self):
        T, D, N, dt = self.T, self.D, self.N, self.dt
        e = lambda *s, d=dt: torch.zeros(s, dtype=d, device=DEV)  # noqa: E731
        o = dict(h=e(T, D), xn=e(T, D), z=e(T, 2 * N), y=e(T, N), out=e(T, D), dy=e(T, N), dz=e(T, 2 * N), dxn=e(T, D), dx=e(T, D))
        o["grad"] = {k: e(*v.shape, d=F32) for k, v in self.p.items()}
        L, c = pk.load(), 1 if dt == BF16 else 0
        o["ws"] = {k: torch.empty(max(int(n), 256), dtype=torch.uint8, device=DEV) for k, n in dict(
            norm=L.mem_layernorm_backward_workspace_size(T, D), wi=L.mem_linear_backward_workspace_size(T, 2 * N, D, c),
            wo=L.mem_linear_backward_workspace_size(T, D, N, c)).items()}
        return o

    def step(self, o, stream=None):
        p, g, ws, s = self.p, o["grad"], o["ws"], dict(stream=stream)
        pk.mem_layernorm(self.x, p["w"], p["b"], self.res, sum_out=o["h"], y_out=o["xn"], **s)
        pk.mem_glu(o["xn"], p["wi"], p["bi"], act=self.act, y_out=o["y"], z_out=o["z"], **s)
        pk.mem_linear(o["y"], p["wo"], residual=o["h"], y_out=o["out"], **s)
        pk.mem_linear_backward(self.dout, o["y"], p["wo"], dx=o["dy"], grad_w=g["wo"], want_grad_bias=False, workspace=ws["wo"], **s)
        pk.mem_glu_backward(o["dy"], o["z"], self.act, dz_out=o["dz"], **s)
        pk.mem_linear_backward(o["dz"], o["xn"], p["wi"], dx=o["dxn"], grad_w=g["wi"], grad_bias=g["bi"], workspace=ws["wi"], **s)
        pk.mem_layernorm_backward(o["dxn"], o["h"], p["w"], dsum=self.dout, dx=o["dx"], grad_weight=g["w"], grad_bias=g["b"],
                                  workspace=ws["norm"], **s)

    def reference(self):
        p = {k: t.detach().cpu().double().requires_grad_() for k, t in self.p.items()}
        x, res = (t.cpu().double().requires_grad_() for t in (self.x, self.res))
        h = x + res
        xn = torch.nn.functional.layer_norm(h, (self.D,), p["w"], p["b"], 1e-5)
        z = xn @ p["wi"].t() + p["bi"]
        f = torch.nn.functional.silu if self.act == "silu" else torch.nn.functional.gelu
        out = (f(z[:, :self.N]) * z[:, self.N:]) @ p["wo"].t() + h
        (out * self.dout.cpu().double()).sum().backward()
        return out.detach(), {**{k: t.grad for k, t in p.items()}, "x": x.grad, "res": res.grad}


def flat(o):
    return [t for k, t in o.items() if k not in ("grad", "ws")] + list(o["grad"].values())


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_training_step(gpu_lib, act):
    """fp32: each number is a chain of at most five sums of up to 272 terms, under 2^10 roundings
    of 2^-24 of the largest."""
    b = Half(T=200, D=136, N=264, dt=F32, act=act)
    o = b.buffers()
    b.step(o)
    out, grads = b.reference()
    close = lambda a, w: float((a.cpu().double() - w).abs().max()) <= 2.0 ** -14 * float(w.abs().max())  # noqa: E731
    assert close(o["out"], out) and torch.equal(grads["x"], grads["res"]) and close(o["dx"], grads["x"])
    for k in b.p:
        assert close(o["grad"][k], grads[k]), k
    # the gradients accumulate: a second step doubles them to within their last bit
    once = {k: v.clone() for k, v in o["grad"].items()}
    b.step(o)
    for k in b.p:
        assert torch.allclose(o["grad"][k], 2 * once[k], rtol=2.0 ** -20, atol=float(once[k].abs().max()) * 2.0 ** -20)


@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
def test_side_stream(gpu_lib, dt):
    b = Half(T=304, D=256, N=520, dt=dt)
    ref, got = b.buffers(), b.buffers()
    b.step(ref)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.step(got, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for x, y in zip(flat(ref), flat(got)):
        assert torch.equal(x, y)
    # outputs and workspaces that the calls allocate belong to that stream
    with torch.cuda.stream(s):
        x, wi, z, dz = b.x.clone(), b.p["wi"].clone(), ref["z"].clone(), ref["dy"].clone()
        long = torch.randn(64, 65536, device=DEV).to(E4M3)
        sc = torch.ones(512, 64, device=DEV)
    s.synchronize()

    def calls(**kw):
        q = pk.mem_quantize_blocks(x, want_cols=True, **kw)
        return (*pk.mem_layernorm(x, residual=x, **kw), *pk.mem_layernorm_backward(x, x, **kw), *pk.mem_glu(x, wi, want_z=True, **kw),
                pk.mem_glu_backward(dz, z, **kw), *(t.view(torch.uint8) if t.dtype == E4M3 else t for t in q),
                *pk.mem_linear_blocks(q[0], q[0], q[1], q[1], want_z=True, **kw),
                pk.mem_linear_blocks(long, long, sc, sc, out_dtype=F32, **kw)[0])
    want, have = calls(), calls(stream=s)
    junk = [torch.full((1 << 20,), 7.0, device=DEV) for _ in range(8)]
    s.synchronize()
    for a, c in zip(want, have):
        assert torch.equal(a, c)
    del junk


@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
def test_captured_step(gpu_lib, dt):
    """Captured once and replayed, eager steps and synchronisations between the replays: bit for
    bit the eager run."""
    halves = [Half(T=777, D=256, N=328, dt=dt, seed=3) for _ in range(2)]
    outs = [b.buffers() for b in halves]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            halves[1].step(outs[1], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for t in flat(outs[1]):
        t.zero_()
    for k in range(4):
        for b in halves:  # other inputs for every replay
            b.x.add_(0.25)
        halves[0].step(outs[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(flat(outs[0]), flat(outs[1])):
            assert torch.equal(x, y), k


def blocks_step(o, x, w, dy, stream=None):
    """A projection's training step in 8 bits into the buffers o."""
    s = dict(stream=stream)
    xq, xs, xqt, xst = pk.mem_quantize_blocks(x, q_out=o["xq"], scale_out=o["xs"], qt_out=o["xqt"], scale_t_out=o["xst"], **s)
    wq, ws, wqt, wst = pk.mem_quantize_blocks(w, tile=True, q_out=o["wq"], scale_out=o["ws"], qt_out=o["wqt"], scale_t_out=o["wst"], **s)
    dq, ds, dqt, dst = pk.mem_quantize_blocks(dy, q_out=o["dq"], scale_out=o["ds"], qt_out=o["dqt"], scale_t_out=o["dst"], **s)
    pk.mem_linear_blocks(xq, wq, xs, ws, y_out=o["y"], **s)
    pk.mem_linear_blocks(dq, wqt, ds, wst, y_out=o["dx"], **s)
    pk.mem_linear_blocks(dqt, xqt, dst, xst, residual=o["gw"], y_out=o["gw"], out_dtype=F32, workspace=o["space"], **s)


def blocks_buffers(T, N, K):
    c = lambda n: -(-n // 128)  # noqa: E731
    e = lambda *s, d=F32: torch.zeros(s, device=DEV).to(d)  # noqa: E731
    T16 = -(-T // 16) * 16
    nb = pk.load().mem_linear_blocks_workspace_size(N, K, T16, 0)
    return dict(xq=e(T, K, d=E4M3), xs=e(c(K), T), xqt=e(K, T16, d=E4M3), xst=e(c(T), K), wq=e(N, K, d=E4M3), ws=e(c(K), c(N)),
                wqt=e(K, N, d=E4M3), wst=e(c(N), c(K)), dq=e(T, N, d=E4M3), ds=e(c(N), T), dqt=e(N, T16, d=E4M3), dst=e(c(T), N),
                y=e(T, N, d=BF16), dx=e(T, K, d=BF16), gw=e(N, K), space=torch.empty(max(nb, 256), dtype=torch.uint8, device=DEV)), nb


def same(a, b):
    return all(torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)) for k in a if k != "space")


def test_two_captured_steps_at_once(gpu_lib):
    """Two graphs with buffers and workspaces of their own, replayed on two streams at the same
    time; the weight's gradient is split over k and uses its workspace."""
    T, N, K = 16001, 256, 144
    g = torch.Generator(device=DEV).manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).to(BF16)  # noqa: E731
    ins = [(r(T, K), r(N, K), r(T, N)) for _ in range(2)]
    want, got = [blocks_buffers(T, N, K)[0] for _ in ins], [blocks_buffers(T, N, K) for _ in ins]
    assert all(nb > 0 for _, nb in got)
    got = [o for o, _ in got]
    graphs, streams = [], [torch.cuda.Stream() for _ in ins]
    for i, s in enumerate(streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                blocks_step(got[i], *ins[i], stream=s)
            graphs.append(graph)
    torch.cuda.synchronize()
    for o in got:
        o["gw"].zero_()
    for _ in range(3):
        for o, i in zip(want, ins):
            blocks_step(o, *i)
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(want, got))


def test_forward_in_8_bit_blocks(gpu_lib):
    """layernorm -> rows in blocks -> product with bias and activation, against the fp64 product
    of the numbers that the codes stand for; few tokens give the same as many but for what the
    8-bit instruction cuts off."""
    T, D, N = 333, 1040, 520
    g = torch.Generator(device=DEV).manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).to(BF16)  # noqa: E731
    x, res, w, bias = r(T, D), r(T, D), r(N, D) / 32, r(N)
    wq, sw, _, _ = pk.mem_quantize_blocks(w, tile=True)
    y, _ = pk.mem_layernorm(x, residual=res)
    q, s, _, _ = pk.mem_quantize_blocks(y)
    out, _ = pk.mem_linear_blocks(q, wq, s, sw, bias, act="silu")
    a, b = q.double() * spread(s.double(), 1, T, D), wq.double() * spread(sw.double(), 128, N, D)
    assert float((a - y.double()).abs().max()) <= 2.0 ** -4 * float(y.abs().max())  # half a step of a code
    z = a @ b.t().contiguous() + bias.double()
    want, size = z * torch.sigmoid(z), a.abs() @ b.abs().t().contiguous()
    tol = 1.13 * (2.0 ** -10 * size + 2.0 ** -16 * size) + 2.0 ** -12 * (z.abs() + want.abs())
    assert torch.all((out.double() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol))
    few, _ = pk.mem_linear_blocks(q[:8].contiguous(), wq, s[:, :8].contiguous(), sw, bias, act="silu")
    assert torch.all((few.double() - want[:8]).abs() <= tol[:8] + 2.0 ** -8 * (want[:8].abs() + tol[:8]))


def test_offsets_past_32_bits_products(gpu_lib):
    """y of more than 2^32 elements: the last rows are those of a small call."""
    K, N = 32, 32768
    g = torch.Generator(device=DEV).manual_seed(2)
    for T in (140001,):
        x = torch.randn((T, K), generator=g, device=DEV).to(BF16)
        w = torch.randn((2 * N, K), generator=g, device=DEV).to(BF16)
        y, _ = pk.mem_glu(x, w)
        assert y.numel() > 1 << 32
        for at in (0, 70000, T - 300):
            assert torch.equal(y[at:at + 300], pk.mem_glu(x[at:at + 300].contiguous(), w)[0])
        del y
        q, s, _, _ = pk.mem_quantize_blocks(x)
        wq, ws, _, _ = pk.mem_quantize_blocks(w[:N].contiguous(), tile=True)
        y, _ = pk.mem_linear_blocks(q, wq, s, ws)
        for at in (0, 70000, T - 300):
            part, _ = pk.mem_linear_blocks(q[at:at + 300].contiguous(), wq, s[:, at:at + 300].contiguous(), ws)
            assert torch.equal(y[at:at + 300], part)
        del y


def test_offsets_past_32_bits_rows(gpu_lib):
    R, C = (1 << 21) + 77, 2064
    x = torch.empty((R, C), dtype=BF16, device=DEV)
    for i in range(0, R, 1 << 18):  # in pieces: the draw is in fp32
        x[i:i + (1 << 18)].normal_(generator=torch.Generator(device=DEV).manual_seed(i))
    q, s, qt, st = pk.mem_quantize_blocks(x, want_cols=True)
    for at in (0, (1 << 20) + 128 * 5, R - 77):
        n = min(256, R - at)
        a, b, c, d = pk.mem_quantize_blocks(x[at:at + n].contiguous(), want_cols=True)
        assert torch.equal(q[at:at + n].view(torch.uint8), a.view(torch.uint8)) and torch.equal(s[:, at:at + n], b)
        if at % 128 == 0 or at == R - 77:
            blk = -(-n // 128)
            if at % 128 == 0:
                assert torch.equal(st[at // 128:at // 128 + blk], d)
                assert torch.equal(qt[:, at:at + n].view(torch.uint8), c[:, :n].view(torch.uint8))
    assert not qt[:, R:].view(torch.uint8).any()
    one, two, _, _ = pk.mem_quantize_blocks(x)
    assert torch.equal(one.view(torch.uint8), q.view(torch.uint8)) and torch.equal(two, s)


def test_more_squares_than_workgroups(gpu_lib):
    """More than 2^20 squares of 128 x 128, and groups of 16 rows, are walked by the workgroups."""
    R, C = (1 << 27) + 200, 16
    x = torch.ones((R, C), dtype=BF16, device=DEV)
    x[:, 3] = 0.5
    x[R - 1] = 4.0
    q, s, qt, st = pk.mem_quantize_blocks(x, want_cols=True)
    assert torch.equal(s[0, :R - 1].min(), s[0, :R - 1].max()) and float(s[0, R - 1]) == float(s[0, 0]) * 4
    b = q.view(torch.uint8)
    assert bool((b[:R - 1] == b[0]).all()) and bool((b[R - 1] == b[0, 0]).all()) and float(q[0, 3]) == 224
    assert bool((qt[3, :R - 1 - (R - 1) % 128].view(torch.uint8) == qt[0, 0].view(torch.uint8)).all())
    assert torch.equal(st[:-1], st[:1].expand(len(st) - 1, C)) and float(st[-1, 0]) == float(s[0, R - 1])
    del qt, st, q
    one, two, _, _ = pk.mem_quantize_blocks(x)
    assert torch.equal(two, s) and torch.equal(one.view(torch.uint8), b)


def test_strided_operands_are_refused(gpu_lib):
    x = torch.randn(64, 256, device=DEV).to(BF16)
    t = x.t()
    w = torch.randn(64, 256, device=DEV).to(BF16)
    for f in (lambda: pk.mem_layernorm(t), lambda: pk.mem_glu(x[:, ::2], w), lambda: pk.mem_quantize_blocks(x[:, :128]),
              lambda: pk.mem_glu_backward(x[:, :64], x[:, :128])):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(pk.PkmemError):  # an address that is no multiple of 16 bytes
        pk.mem_layernorm(torch.zeros(65, device=DEV, dtype=BF16)[1:].view(1, 64))
    with pytest.raises(ValueError):  # scales of another number of blocks
        q, s, _, _ = pk.mem_quantize_blocks(x)
        pk.mem_linear_blocks(q, q, s, s[:1].contiguous())
    with pytest.raises(ValueError):
        pk.mem_glu(x, torch.randn(65, 256, device=DEV).to(BF16))
