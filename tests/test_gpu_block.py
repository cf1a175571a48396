"""The norm, the projections and the optimizer together with the memory, as a
Memory+ block uses them: a whole training step against fp64 autograd, the 8-bit
forward, the same step on a side stream and replayed from a graph."""
import numpy as np
import pytest
import torch

import paper_2412_09764_amd as pk
from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu

DEV = "cuda"
HYPER = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)


class Block:
    """norm(x + res) -> query projection -> search -> value bag, gated by a second
    projection -> output projection added to the stream."""

    def __init__(self, T, D, S, H, n, k, dt, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).to(dt).to(DEV)  # noqa: E731
        self.T, self.D, self.S, self.H, self.n, self.k, self.dt = T, D, S, H, n, k, dt
        self.x, self.res, self.dout = r(T, D), r(T, D), r(T, D)
        self.p = dict(norm=1 + r(D, std=0.1), wq=r(H * n, D, std=D ** -0.5), bq=r(H * n, std=0.1),
                      keys=r(H, 2, S, n // 2, std=n ** -0.5), w1=r(D, D, std=D ** -0.5),
                      w2=r(D, D, std=D ** -0.5), values=r(S * S, D, std=0.1))

    def outputs(self):
        """Every buffer of a step, so that it can be captured."""
        T, D, H, n, k, dt = self.T, self.D, self.H, self.n, self.k, self.dt
        e = lambda *s, d=torch.float32: torch.zeros(s, dtype=d, device=DEV)  # noqa: E731
        o = dict(h=e(T, D, d=dt), xn=e(T, D, d=dt), q=e(T, H * n, d=dt), gate=e(T, D, d=dt), idx=e(T, H, k, d=torch.int64),
                 w=e(T, H, k), mem=e(T, D, d=dt), y=e(T, D, d=dt), out=e(T, D, d=dt), dmem=e(T, D, d=dt), dy=e(T, D, d=dt),
                 dgate=e(T, D), gz=e(T, H, k), gq=e(T, H, n), dxn=e(T, D, d=dt), dx=e(T, D, d=dt), dgc=e(T, D, d=dt),
                 gqc=e(T, H * n, d=dt))
        o["grad"] = {name: e(*p.shape) for name, p in self.p.items()}
        L = pk.load()
        dtc = 1 if dt == torch.bfloat16 else 0
        nb = dict(search=pk.mem_search_workspace_size(T, H, self.S, k),
                  bag=pk.mem_bag_backward_workspace_size(T, H, k, self.S ** 2, D, "sorted"),
                  keys=L.mem_search_backward_workspace_size(T, H, self.S, k),
                  norm=L.mem_rmsnorm_backward_workspace_size(T, D),
                  lq=L.mem_linear_backward_workspace_size(T, H * n, D, dtc), ld=L.mem_linear_backward_workspace_size(T, D, D, dtc))
        o["ws"] = {name: torch.empty(max(int(b), 256), dtype=torch.uint8, device=DEV) for name, b in nb.items()}
        return o

    def step(self, o, stream=None):
        """Forward and backward; gradients accumulate into o["grad"]."""
        p, g, ws, s = self.p, o["grad"], o["ws"], dict(stream=stream)
        T, H, n = self.T, self.H, self.n
        pk.mem_rmsnorm(self.x, p["norm"], self.res, sum_out=o["h"], y_out=o["xn"], **s)
        pk.mem_linear(o["xn"], p["wq"], p["bq"], y_out=o["q"], **s)
        pk.mem_linear(o["xn"], p["w1"], y_out=o["gate"], **s)
        pk.mem_search(o["q"].view(T, H, n), p["keys"], self.k, idx_out=o["idx"], w_out=o["w"], want_score=False,
                      workspace=ws["search"], **s)
        pk.mem_bag_forward_gated(p["values"], o["idx"].view(T, -1), o["w"].view(T, -1), o["gate"], out=o["mem"], y_out=o["y"], **s)
        pk.mem_linear(o["mem"], p["w2"], residual=o["h"], y_out=o["out"], **s)
        pk.mem_linear_backward(self.dout, o["mem"], p["w2"], dx=o["dmem"], grad_w=g["w2"], want_grad_bias=False, workspace=ws["ld"], **s)
        pk.mem_gate_backward(o["dmem"], o["gate"], o["y"], dy_out=o["dy"], grad_gate=o["dgate"], **s)
        pk.mem_bag_backward(o["dy"], p["values"], o["idx"], o["w"], grad_values=g["values"], want_grad_w=False,
                            grad_scores=o["gz"], mode="sorted", workspace=ws["bag"], **s)
        pk.mem_search_backward(o["q"].view(T, H, n), p["keys"], o["idx"], o["gz"], grad_q=o["gq"], grad_subkeys=g["keys"],
                               workspace=ws["keys"], **s)
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            o["dgc"].copy_(o["dgate"])
            o["gqc"].copy_(o["gq"].view(T, H * n))
        pk.mem_linear_backward(o["dgc"], o["xn"], p["w1"], dx=o["dxn"], grad_w=g["w1"], want_grad_bias=False, workspace=ws["ld"], **s)
        pk.mem_linear_backward(o["gqc"], o["xn"], p["wq"], dx_add=o["dxn"], dx=o["dxn"], grad_w=g["wq"], grad_bias=g["bq"],
                               workspace=ws["lq"], **s)
        pk.mem_rmsnorm_backward(o["dxn"], o["h"], p["norm"], dsum=self.dout, dx=o["dx"], grad_weight=g["norm"],
                                workspace=ws["norm"], **s)

    def reference(self, idx):
        """Output and gradients in 64 bits, for a given selection."""
        p = {name: t.detach().cpu().double().requires_grad_() for name, t in self.p.items()}
        x, res = (t.cpu().double().requires_grad_() for t in (self.x, self.res))
        T, H, d = self.T, self.H, self.n // 2
        h = x + res
        xn = h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-5) * p["norm"]
        q = (xn @ p["wq"].t() + p["bq"]).view(T, H, 2 * d)
        i1, i2 = idx // self.S, idx % self.S
        hh = torch.arange(H)[None, :, None]
        z = (q[:, :, None, :d] * p["keys"][hh, 0, i1]).sum(-1) + (q[:, :, None, d:] * p["keys"][hh, 1, i2]).sum(-1)
        y = (torch.softmax(z, -1)[..., None] * p["values"][idx]).sum((1, 2))
        gate = xn @ p["w1"].t()
        out = (y * gate * torch.sigmoid(gate)) @ p["w2"].t() + h
        (out * self.dout.cpu().double()).sum().backward()
        return out.detach(), {**{name: t.grad for name, t in p.items()}, "x": x.grad, "res": res.grad}


def test_training_step(gpu_lib):
    """fp32: every gradient within 2^-14 of its largest entry (each is a chain of at most six
    products of up to 96 terms, under 2^10 roundings of 2^-24), then the optimizer's step on
    all parameters, the values as touched rows."""
    b = Block(T=96, D=64, S=16, H=2, n=32, k=4, dt=torch.float32)
    o = b.outputs()
    b.step(o)
    out, grads = b.reference(o["idx"].cpu())
    close = lambda a, w: float((a.cpu().double() - w).abs().max()) <= 2.0 ** -14 * float(w.abs().max())  # noqa: E731
    assert close(o["out"], out)
    assert torch.equal(grads["x"], grads["res"]) and close(o["dx"], grads["x"])
    for name in b.p:
        assert close(o["grad"][name], grads[name]), name
    rows, grad_rows, _, _ = pk.mem_bag_backward_sparse(o["dy"], b.p["values"], o["idx"], o["w"])
    assert torch.equal(grad_rows, o["grad"]["values"][rows])
    before = {name: t.cpu().double().numpy() for name, t in b.p.items()}
    names = [name for name in b.p if name != "values"]
    st = {name: pk.mem_adamw_state(b.p[name]) for name in b.p}
    pk.mem_adamw([b.p[m] for m in names], [o["grad"][m] for m in names], [st[m][0] for m in names], [st[m][1] for m in names],
                 step=1, **HYPER)
    pk.mem_adamw_rows(b.p["values"], rows, grad_rows, st["values"][0], st["values"][1], step=1, **HYPER)
    for name in b.p:
        g = o["grad"][name].cpu().double().numpy()
        zero = np.zeros_like(g)
        want, _, _ = bo.adamw(before[name], g, zero, zero, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"], 1)
        if name == "values":  # rows that no token chose stay
            rest = np.ones(len(g), bool)
            rest[rows.cpu().numpy()] = False
            want[rest] = before[name][rest]
        # 4 u of the parameter and 32 u of an update of at most lr
        err = np.abs(b.p[name].cpu().double().numpy() - want)
        assert np.all(err <= 2.0 ** -24 * (4 * np.abs(before[name]) + 32 * HYPER["lr"])), name


def test_forward_in_8_bits(gpu_lib):
    """The norm's codes and scales go into the 8-bit product as they are; against the fp64
    product of the values they stand for."""
    T, D, N = 333, 1024, 520
    g = torch.Generator(device=DEV).manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).bfloat16()  # noqa: E731
    x, res, w, bias = r(T, D), r(T, D), r(N, D) / 32, r(N)
    wq, sw = pk.mem_quantize_rows(w)
    xq, _, sx = pk.mem_rmsnorm(x, None, res, quantize=True)
    y, _ = pk.mem_linear(xq, wq, bias, act="silu", x_scale=sx, w_scale=sw)
    a, b = xq.double() * sx.double()[:, None], wq.double() * sw.double()[:, None]
    z = a @ b.t().contiguous() + bias.double()
    want = z * torch.sigmoid(z)
    tol = 1.1 * (D + 4) * 2.0 ** -24 * (a.abs() @ b.abs().t().contiguous() + bias.double().abs()) + \
        2.0 ** -12 * (z.abs() + want.abs()) + 2.0 ** -8 * want.abs()
    assert torch.all((y.double() - want).abs() <= tol)


def _flat(o):
    return [t for name, t in o.items() if name not in ("grad", "ws")] + list(o["grad"].values())


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_side_stream(gpu_lib, dt):
    b = Block(T=200, D=128, S=32, H=2, n=64, k=8, dt=dt)
    ref, got = b.outputs(), b.outputs()
    b.step(ref)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.step(got, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for x, y in zip(_flat(ref), _flat(got)):
        assert torch.equal(x, y)
    # outputs and workspaces that the calls allocate belong to that stream
    with torch.cuda.stream(s):
        x, w, dz = b.x.clone(), b.p["w1"].clone(), b.dout.clone()
    s.synchronize()
    want = pk.mem_linear_backward(dz, x, w), pk.mem_rmsnorm_backward(dz, x), pk.mem_linear(x, w, act="gelu", want_z=True)
    have = (pk.mem_linear_backward(dz, x, w, stream=s), pk.mem_rmsnorm_backward(dz, x, stream=s),
            pk.mem_linear(x, w, act="gelu", want_z=True, stream=s))
    junk = [torch.full((1 << 20,), 7.0, device=DEV) for _ in range(8)]
    s.synchronize()
    for a, c in zip(want, have):
        for x, y in zip(a, c):
            assert torch.equal(x, y)
    del junk


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_captured_block(gpu_lib, dt):
    """Forward, backward and optimizer captured once and replayed, eager steps and
    synchronisations between the replays: bit for bit the eager run."""
    blocks = [Block(T=300, D=128, S=32, H=2, n=64, k=8, dt=dt, seed=3) for _ in range(2)]
    outs = [b.outputs() for b in blocks]
    state = [{name: pk.mem_adamw_state(p, 8 if name == "values" else 32) for name, p in b.p.items()} for b in blocks]
    ts = [torch.zeros(1, dtype=torch.int64, device=DEV) for _ in blocks]

    def step(i, stream):
        b, o, st = blocks[i], outs[i], state[i]
        with torch.cuda.stream(stream):
            ts[i].add_(1)
            for g in o["grad"].values():
                g.zero_()
        b.step(o, stream=stream)
        names = list(b.p)
        pk.mem_adamw([b.p[m] for m in names], [o["grad"][m] for m in names], [st[m][0] for m in names],
                     [st[m][1] for m in names], step=ts[i], seed=5, exp_avg_scales=[st[m][2] for m in names],
                     exp_avg_sq_scales=[st[m][3] for m in names], stream=stream, **HYPER)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(1, side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for k in range(4):
        step(0, torch.cuda.current_stream())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(_flat(outs[0]), _flat(outs[1])):
            assert torch.equal(x, y), k
        for name in blocks[0].p:
            assert torch.equal(blocks[0].p[name], blocks[1].p[name]), (k, name)
            for x, y in zip(state[0][name], state[1][name]):
                assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (k, name)
