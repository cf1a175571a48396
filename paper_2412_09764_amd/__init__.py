"""Product-key memory hot path on MI355X: thin binding of libpkmem.so.

The library (include/pkmem.h) implements the product-key search of Sec. 3.1.1
of "Memory Layers at Scale" (arXiv 2412.09764) followed by the softmax of
Sec. 3, Eq. (1), and the weighted EmbeddingBag forward and backward of
Sec. 3.1.4, with the norm, projections and optimizer of the block around them, as
hand-written HIP kernels for gfx950.

This module only marshals arguments: it checks tensor placement and dtype,
allocates outputs and workspaces with torch on the current device (on the
`stream` argument when one is given, else on the current stream), passes raw
pointers and that HIP stream through the C ABI, and turns a non-zero status
into PkmemError.  Every step of the computation runs in the library;
there is no fallback: without the built library every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct

import torch  # noqa: F401  (first: the library binds to the HIP runtime torch loads)

__all__ = [
    "PkmemError", "load", "lib_path", "mem_search", "mem_search_noalloc", "mem_search_backward",
    "mem_search_qnorm", "NOALLOC_SCRATCH_BYTES",
    "mem_search_backward_qnorm", "mem_search_extra", "mem_search_sink",
    "mem_search_backward_sink", "mem_bag_forward",
    "mem_bag_forward_gated", "mem_gate_backward",
    "mem_bag_backward",
    "mem_bag_backward_sparse", "mem_search_workspace_size", "mem_bag_backward_workspace_size",
    "BWD_MODES", "F32", "BF16", "mem_timer_start", "mem_timer_stop", "mem_timer_read",
    "E4M3", "mem_rmsnorm", "mem_rmsnorm_backward", "mem_quantize_rows",
    "mem_linear", "mem_act_backward", "mem_linear_backward", "ACTIVATIONS",
    "mem_layernorm", "mem_layernorm_backward", "mem_glu", "mem_glu_backward",
    "mem_quantize_blocks", "mem_linear_blocks", "SCALE_BLOCK",
    "mem_adamw", "mem_adamw_rows", "mem_adamw_state", "ADAMW_STATE_BLOCK",
]

F32, BF16, E4M3 = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
ADAMW_STATE_BLOCK = 128  # elements that share the scales of 8-bit optimizer states
SCALE_BLOCK = 128  # elements along k (rows and columns of a tile) that share a scale
NOALLOC_SCRATCH_BYTES = 128 << 20  # PKMEM_NOALLOC_SCRATCH_BYTES
BWD_MODES = {"auto": 0, "atomic": 1, "sorted": 2}
_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None


class PkmemError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"pkmem status {code}: {msg}")
        self.code = code


def lib_path() -> str:
    return os.environ.get("PKMEM_LIB", os.path.join(_HERE, "libpkmem.so"))


def load() -> ctypes.CDLL:
    """Load libpkmem.so (raises if it has not been built)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2412_09764_amd.build`")
    L = ctypes.CDLL(path)
    P, I64, I32, SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
    L.mem_search_workspace_size.argtypes = [I64, I32, I32, I32]
    L.mem_search_workspace_size.restype = SZ
    L.mem_search.argtypes = [P, I32, P, I32, I64, I32, I32, I32, I32, P, P, P, P, P, SZ, P]
    L.mem_search.restype = I32
    L.mem_search_noalloc.argtypes = [P, I32, P, I32, I64, I32, I32, I32, I32, P, P, P, P, P]
    L.mem_search_noalloc.restype = I32
    L.mem_search_backward_workspace_size.argtypes = [I64, I32, I32, I32]
    L.mem_search_backward_workspace_size.restype = SZ
    L.mem_search_backward.argtypes = [P, I32, P, I32, I64, I32, I32, I32, I32, P, P, P, P, P, SZ, P]
    L.mem_search_backward.restype = I32
    F32 = ctypes.c_float
    L.mem_search_qnorm.argtypes = [P, I32, P, I32, I64, I32, I32, I32, I32, F32, P, P, P, P, P, P,
                                   P, SZ, P]
    L.mem_search_qnorm.restype = I32
    L.mem_search_backward_qnorm.argtypes = [P, I32, P, I32, I64, I32, I32, I32, I32, F32, P, P, P,
                                            P, P, SZ, P]
    L.mem_search_backward_qnorm.restype = I32
    L.mem_search_extra.argtypes = [P, I32, P, I32, I64, I32, I32, I32, I32, I32, P, P, P, P, P, P, SZ,
                                   P]
    L.mem_search_extra.restype = I32
    L.mem_search_sink.argtypes = [P, I32, P, I32, I64, I32, I32, I32, I32, I32, P, P, I64, P, P, P,
                                  P, P, SZ, P]
    L.mem_search_sink.restype = I32
    L.mem_search_backward_sink_workspace_size.argtypes = [I64, I32, I32, I32, I32]
    L.mem_search_backward_sink_workspace_size.restype = SZ
    L.mem_search_backward_sink.argtypes = [P, I32, P, I32, I64, I32, I32, I32, I32, P, P, P, P, P, P,
                                           P, SZ, P]
    L.mem_search_backward_sink.restype = I32
    L.mem_bag_forward.argtypes = [P, I32, I64, I32, P, P, I64, I32, P, P]
    L.mem_bag_forward.restype = I32
    L.mem_bag_forward_gated.argtypes = [P, I32, I64, I32, P, P, I64, I32, P, P, P, P]
    L.mem_bag_forward_gated.restype = I32
    L.mem_gate_backward.argtypes = [P, P, P, I32, I64, I32, P, P, P]
    L.mem_gate_backward.restype = I32
    L.mem_bag_backward_workspace_size.argtypes = [I64, I32, I32, I64, I32, I32]
    L.mem_bag_backward_workspace_size.restype = SZ
    L.mem_bag_backward.argtypes = [P, P, I32, I64, I32, P, P, I64, I32, I32, P, P, P, I32, P, SZ, P]
    L.mem_bag_backward.restype = I32
    L.mem_bag_backward_sparse.argtypes = [P, P, I32, I64, I32, P, P, I64, I32, I32, P, P, I64, P,
                                          P, P, P, SZ, P]
    L.mem_bag_backward_sparse.restype = I32
    L.mem_rmsnorm.argtypes = [P, P, P, I32, I64, I32, F32, P, P, I32, P, P]
    L.mem_rmsnorm.restype = I32
    L.mem_rmsnorm_backward_workspace_size.argtypes = [I64, I32]
    L.mem_rmsnorm_backward_workspace_size.restype = SZ
    L.mem_rmsnorm_backward.argtypes = [P, P, P, I32, I64, I32, F32, P, P, P, P, SZ, P]
    L.mem_rmsnorm_backward.restype = I32
    L.mem_quantize_rows.argtypes = [P, I32, I64, I32, P, P, P]
    L.mem_quantize_rows.restype = I32
    L.mem_linear.argtypes = [P, P, I32, P, P, P, P, I64, I32, I32, I32, P, P, I32, P]
    L.mem_linear.restype = I32
    L.mem_act_backward.argtypes = [P, P, I32, I32, I64, I32, P, P]
    L.mem_act_backward.restype = I32
    L.mem_linear_backward_workspace_size.argtypes = [I64, I32, I32, I32]
    L.mem_linear_backward_workspace_size.restype = SZ
    L.mem_linear_backward.argtypes = [P, P, P, I32, I64, I32, I32, P, P, P, P, P, SZ, P]
    L.mem_linear_backward.restype = I32
    L.mem_layernorm.argtypes = [P, P, P, P, I32, I64, I32, F32, P, P, P]
    L.mem_layernorm.restype = I32
    L.mem_layernorm_backward_workspace_size.argtypes = [I64, I32]
    L.mem_layernorm_backward_workspace_size.restype = SZ
    L.mem_layernorm_backward.argtypes = [P, P, P, I32, I64, I32, F32, P, P, P, P, P, SZ, P]
    L.mem_layernorm_backward.restype = I32
    L.mem_glu.argtypes = [P, P, I32, P, P, P, I64, I32, I32, I32, P, P, I32, P]
    L.mem_glu.restype = I32
    L.mem_glu_backward.argtypes = [P, P, I32, I32, I64, I32, P, P]
    L.mem_glu_backward.restype = I32
    L.mem_quantize_blocks.argtypes = [P, I32, I64, I32, I32, P, P, P, P, P]
    L.mem_quantize_blocks.restype = I32
    L.mem_linear_blocks_workspace_size.argtypes = [I64, I32, I32, I32]
    L.mem_linear_blocks_workspace_size.restype = SZ
    L.mem_linear_blocks.argtypes = [P, P, P, P, I32, P, P, I64, I32, I32, I32, P, P, I32, P, SZ, P]
    L.mem_linear_blocks.restype = I32
    L.mem_adamw.argtypes = [P, I32, P, P]
    L.mem_adamw.restype = I32
    L.mem_adamw_rows.argtypes = [P, I64, I32, P, I64, P, P]
    L.mem_adamw_rows.restype = I32
    L.mem_last_error.argtypes = []
    L.mem_last_error.restype = ctypes.c_char_p
    L.mem_version.argtypes = []
    L.mem_version.restype = I32
    L.mem_timer_start.argtypes = [ctypes.c_char_p]
    L.mem_timer_start.restype = I32
    L.mem_timer_stop.argtypes = []
    L.mem_timer_stop.restype = I32
    L.mem_timer_read.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int), I32]
    L.mem_timer_read.restype = I32
    _LIB = L
    return L


def _check(rc: int) -> None:
    if rc != 0:
        raise PkmemError(rc, load().mem_last_error().decode(errors="replace"))


def _dt(t: torch.Tensor) -> int:
    dt = t.dtype
    if dt is torch.float32:
        return F32
    if dt is torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype} (float32 or bfloat16)")


def _dev(*ts: torch.Tensor) -> None:
    for t in ts:
        if t is not None:
            if not t.is_cuda:
                raise ValueError("tensors must be on the GPU")
            if not t.is_contiguous():
                raise ValueError("tensors must be contiguous")


def _ptr(t):
    return None if t is None else t.data_ptr()


# A small call is bound by the host (a decode step of three kernels takes 17 us),
# and torch's stream object alone takes 4 us a call, so the handle is asked for
# directly (torch has no public call for the handle alone), and the stream
# context is entered only where a stream is given.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(_current_device())


def _launches_on_stream(fn):
    """Runs fn with its `stream` argument (if given) as torch's current stream:
    outputs, workspaces and zero-filled accumulators allocated by the wrapper
    then belong to the stream the library launches on, and the fills are
    ordered before the launch on that stream."""
    @functools.wraps(fn)
    def wrapper(*args, **kw):
        stream = kw.get("stream")
        if stream is None:
            return fn(*args, **kw)
        with torch.cuda.stream(stream):
            return fn(*args, **kw)
    return wrapper


def _workspace(nbytes: int, device, ws):
    if ws is not None:
        if ws.numel() * ws.element_size() < nbytes:
            raise ValueError(f"workspace too small: {nbytes} bytes needed")
        return ws
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)


def mem_timer_start(*kernels: str) -> None:
    """Record HIP events around every launch of the named kernels (pkmem.h)."""
    _check(load().mem_timer_start(",".join(kernels).encode()))


def mem_timer_stop() -> None:
    _check(load().mem_timer_stop())


def mem_timer_read(cap: int = 1 << 16) -> list:
    """[(kernel_position, ms)] of the launches recorded since the last read."""
    ms = (ctypes.c_float * cap)()
    which = (ctypes.c_int * cap)()
    n = load().mem_timer_read(ms, which, cap)
    if n < 0:
        _check(n)
    return [(int(which[i]), float(ms[i])) for i in range(min(n, cap))]


def mem_search_workspace_size(T: int, H: int, S: int, k: int) -> int:
    return int(load().mem_search_workspace_size(T, H, S, k))


def mem_bag_backward_workspace_size(T: int, H: int, k: int, N: int, D: int, mode="auto") -> int:
    m = BWD_MODES[mode] if isinstance(mode, str) else int(mode)
    return int(load().mem_bag_backward_workspace_size(T, H, k, N, D, m))


@_launches_on_stream
def mem_search(q: torch.Tensor, subkeys: torch.Tensor, k: int, *, idx_out=None, w_out=None,
               score_out=None, half_idx_out=None, want_score: bool = True,
               want_half: bool = False, workspace=None, stream=None):
    """Product-key search + softmax.  q [T, H, n], subkeys [H, 2, S, n/2].

    Returns (idx int64 [T,H,k], w fp32 [T,H,k], score fp32 [T,H,k] or None,
    half_idx int32 [T,H,2,k] or None).
    """
    return _search(q, subkeys, k, None, idx_out, w_out, score_out, half_idx_out, want_score,
                   want_half, None, None, workspace, stream)[:4]


@_launches_on_stream
def mem_search_noalloc(q: torch.Tensor, subkeys: torch.Tensor, k: int, *, idx_out=None,
                       w_out=None, score_out=None, half_idx_out=None, want_score: bool = True,
                       want_half: bool = False, stream=None):
    """mem_search with its workspace in the library's static device scratch
    array (no workspace argument; the C call allocates nothing).  Outputs not
    given are allocated here with torch; pass them all to allocate nothing.
    Requires mem_search_workspace_size(T, H, S, k) <= NOALLOC_SCRATCH_BYTES."""
    L = load()
    _dev(q, subkeys)
    T, H, n = q.shape
    S = subkeys.shape[2]
    dev = q.device
    if idx_out is None:
        idx_out = torch.empty((T, H, k), dtype=torch.int64, device=dev)
    if w_out is None:
        w_out = torch.empty((T, H, k), dtype=torch.float32, device=dev)
    if score_out is None and want_score:
        score_out = torch.empty((T, H, k), dtype=torch.float32, device=dev)
    if half_idx_out is None and want_half:
        half_idx_out = torch.empty((T, H, 2, k), dtype=torch.int32, device=dev)
    _dev(idx_out, w_out, score_out, half_idx_out)
    _check(L.mem_search_noalloc(_ptr(q), _dt(q), _ptr(subkeys), _dt(subkeys), T, H, n, S, k,
                                _ptr(idx_out), _ptr(w_out), _ptr(score_out), _ptr(half_idx_out),
                                _stream(stream)))
    return idx_out, w_out, score_out, half_idx_out


@_launches_on_stream
def mem_search_qnorm(q: torch.Tensor, subkeys: torch.Tensor, k: int, eps: float = 1e-5, *,
                     idx_out=None, w_out=None, score_out=None, half_idx_out=None,
                     want_score: bool = True, want_half: bool = False, qhat_out=None,
                     stats_out=None, want_qhat: bool = False, want_stats: bool = False,
                     workspace=None, stream=None):
    """mem_search of the LayerNorm-normalised queries (no affine, eps), the
    normalisation fused into the scoring.  Returns (idx, w, score, half_idx,
    qhat [T,H,n] in q's dtype or None, stats fp32 [T,H,2] (mean, rstd) or None)."""
    T, H, n = q.shape
    if qhat_out is None and want_qhat:
        qhat_out = torch.empty((T, H, n), dtype=q.dtype, device=q.device)
    if stats_out is None and want_stats:
        stats_out = torch.empty((T, H, 2), dtype=torch.float32, device=q.device)
    return _search(q, subkeys, k, float(eps), idx_out, w_out, score_out, half_idx_out, want_score,
                   want_half, qhat_out, stats_out, workspace, stream)


@_launches_on_stream
def mem_search_extra(q: torch.Tensor, subkeys: torch.Tensor, k: int, extra_idx: torch.Tensor, *,
                     idx_out=None, w_out=None, score_out=None, half_idx_out=None,
                     want_score: bool = True, want_half: bool = False, workspace=None,
                     stream=None):
    """mem_search plus r extra key-value pairs per (token, head): extra_idx
    [T, H, r] int64 composed indices, scored as full keys, in slots k..k+r-1;
    softmax over all k + r.  Returns (idx, w, score, half_idx) with k + r slots."""
    return _search_extra(q, subkeys, k, extra_idx, None, 0, idx_out, w_out, score_out,
                         half_idx_out, want_score, want_half, workspace, stream)


@_launches_on_stream
def mem_search_sink(q: torch.Tensor, subkeys: torch.Tensor, k: int, sink_keys: torch.Tensor,
                    sink_row0: int, extra_idx=None, *, idx_out=None, w_out=None, score_out=None,
                    half_idx_out=None, want_score: bool = True, want_half: bool = False,
                    workspace=None, stream=None):
    """mem_search_extra (extra_idx [T, H, r] or None) plus one fixed key-value
    pair per head in the last slot: key sink_keys [H, n] (subkeys' dtype),
    scored q . sink_keys[h]; index sink_row0 + h (>= S*S, the value-table row of
    head h's sink value).  Returns (idx, w, score, half_idx) with k + r + 1 slots."""
    if extra_idx is None:
        T, H, _ = q.shape
        extra_idx = torch.empty((T, H, 0), dtype=torch.int64, device=q.device)
    return _search_extra(q, subkeys, k, extra_idx, sink_keys, int(sink_row0), idx_out, w_out,
                         score_out, half_idx_out, want_score, want_half, workspace, stream)


def _search_extra(q, subkeys, k, extra_idx, sink_keys, sink_row0, idx_out, w_out, score_out,
                  half_idx_out, want_score, want_half, workspace, stream):
    L = load()
    _dev(q, subkeys, extra_idx, sink_keys)
    T, H, n = q.shape
    S = subkeys.shape[2]
    r = extra_idx.shape[2] if extra_idx.dim() == 3 else 0
    if extra_idx.dtype != torch.int64:
        raise ValueError("extra_idx must be int64")
    if sink_keys is not None and (sink_keys.shape != (H, n) or sink_keys.dtype != subkeys.dtype):
        raise ValueError("sink_keys must be [H, n] in the sub-keys' dtype")
    dev = q.device
    kk = k + r + (1 if sink_keys is not None else 0)
    if idx_out is None:
        idx_out = torch.empty((T, H, kk), dtype=torch.int64, device=dev)
    if w_out is None:
        w_out = torch.empty((T, H, kk), dtype=torch.float32, device=dev)
    if score_out is None and want_score:
        score_out = torch.empty((T, H, kk), dtype=torch.float32, device=dev)
    if half_idx_out is None and want_half:
        half_idx_out = torch.empty((T, H, 2, k), dtype=torch.int32, device=dev)
    _dev(idx_out, w_out, score_out, half_idx_out)
    ws = _workspace(mem_search_workspace_size(T, H, S, k), dev, workspace)
    outs = (_ptr(idx_out), _ptr(w_out), _ptr(score_out), _ptr(half_idx_out), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(stream))
    if sink_keys is None:
        _check(L.mem_search_extra(_ptr(q), _dt(q), _ptr(subkeys), _dt(subkeys), T, H, n, S, k, r,
                                  _ptr(extra_idx), *outs))
    else:
        _check(L.mem_search_sink(_ptr(q), _dt(q), _ptr(subkeys), _dt(subkeys), T, H, n, S, k, r,
                                 _ptr(extra_idx), _ptr(sink_keys), sink_row0, *outs))
    return idx_out, w_out, score_out, half_idx_out


def _search(q, subkeys, k, eps, idx_out, w_out, score_out, half_idx_out, want_score, want_half,
            qhat_out, stats_out, workspace, stream):
    L = load()
    _dev(q, subkeys)
    T, H, n = q.shape
    S = subkeys.shape[2]
    dev = q.device
    if idx_out is None:
        idx_out = torch.empty((T, H, k), dtype=torch.int64, device=dev)
    if w_out is None:
        w_out = torch.empty((T, H, k), dtype=torch.float32, device=dev)
    if score_out is None and want_score:
        score_out = torch.empty((T, H, k), dtype=torch.float32, device=dev)
    if half_idx_out is None and want_half:
        half_idx_out = torch.empty((T, H, 2, k), dtype=torch.int32, device=dev)
    _dev(idx_out, w_out, score_out, half_idx_out)
    nbytes = mem_search_workspace_size(T, H, S, k)
    ws = _workspace(nbytes, dev, workspace)
    if eps is None:
        _check(L.mem_search(_ptr(q), _dt(q), _ptr(subkeys), _dt(subkeys), T, H, n, S, k,
                            _ptr(idx_out), _ptr(w_out), _ptr(score_out), _ptr(half_idx_out),
                            _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))
    else:
        _dev(qhat_out, stats_out)
        _check(L.mem_search_qnorm(_ptr(q), _dt(q), _ptr(subkeys), _dt(subkeys), T, H, n, S, k, eps,
                                  _ptr(idx_out), _ptr(w_out), _ptr(score_out), _ptr(half_idx_out),
                                  _ptr(qhat_out), _ptr(stats_out), _ptr(ws),
                                  ws.numel() * ws.element_size(), _stream(stream)))
    return idx_out, w_out, score_out, half_idx_out, qhat_out, stats_out


@_launches_on_stream
def mem_search_backward(q: torch.Tensor, subkeys: torch.Tensor, idx: torch.Tensor,
                        grad_scores: torch.Tensor, *, grad_q=None, grad_subkeys=None,
                        want_grad_q: bool = True, want_grad_subkeys: bool = True, workspace=None,
                        stream=None):
    """Gradients of the selected scores into q ([T,H,n], written) and the
    sub-keys ([H,2,S,n/2], ACCUMULATED; a zero table is allocated if none is
    given).  Returns (grad_q, grad_subkeys)."""
    return _search_backward(q, subkeys, idx, grad_scores, None, grad_q, grad_subkeys, want_grad_q,
                            want_grad_subkeys, workspace, stream)


@_launches_on_stream
def mem_search_backward_qnorm(q: torch.Tensor, subkeys: torch.Tensor, idx: torch.Tensor,
                              grad_scores: torch.Tensor, eps: float = 1e-5, *, grad_q=None,
                              grad_subkeys=None, want_grad_q: bool = True,
                              want_grad_subkeys: bool = True, workspace=None, stream=None):
    """mem_search_backward through the query normalisation of
    mem_search_qnorm (same q and eps): grad_q with respect to the raw
    queries, grad_subkeys accumulated from the normalised ones."""
    return _search_backward(q, subkeys, idx, grad_scores, float(eps), grad_q, grad_subkeys,
                            want_grad_q, want_grad_subkeys, workspace, stream)


@_launches_on_stream
def mem_search_backward_sink(q: torch.Tensor, subkeys: torch.Tensor, idx: torch.Tensor,
                             grad_scores: torch.Tensor, sink_keys: torch.Tensor, *, grad_q=None,
                             grad_subkeys=None, grad_sink=None, want_grad_q: bool = True,
                             want_grad_subkeys: bool = True, want_grad_sink: bool = True,
                             workspace=None, stream=None):
    """Search backward of mem_search_sink: idx and grad_scores [T, H, k + 1]
    (last slot the sink's).  grad_q written; grad_subkeys and grad_sink
    ([H, n] fp32) ACCUMULATED (zero tables allocated if none are given).
    Returns (grad_q, grad_subkeys, grad_sink)."""
    L = load()
    _dev(q, subkeys, idx, grad_scores, sink_keys)
    T, H, n = q.shape
    S = subkeys.shape[2]
    k = idx.shape[2] - 1
    if grad_q is None and want_grad_q:
        grad_q = torch.empty((T, H, n), dtype=torch.float32, device=q.device)
    if grad_subkeys is None and want_grad_subkeys:
        grad_subkeys = torch.zeros(subkeys.shape, dtype=torch.float32, device=q.device)
    if grad_sink is None and want_grad_sink:
        grad_sink = torch.zeros((H, n), dtype=torch.float32, device=q.device)
    _dev(grad_q, grad_subkeys, grad_sink)
    nbytes = int(L.mem_search_backward_sink_workspace_size(T, H, n, S, k))
    ws = _workspace(nbytes, q.device, workspace)
    _check(L.mem_search_backward_sink(_ptr(q), _dt(q), _ptr(subkeys), _dt(subkeys), T, H, n, S, k,
                                      _ptr(idx), _ptr(grad_scores), _ptr(sink_keys), _ptr(grad_q),
                                      _ptr(grad_subkeys), _ptr(grad_sink), _ptr(ws),
                                      ws.numel() * ws.element_size(), _stream(stream)))
    return grad_q, grad_subkeys, grad_sink


def _search_backward(q, subkeys, idx, grad_scores, eps, grad_q, grad_subkeys, want_grad_q,
                     want_grad_subkeys, workspace, stream):
    L = load()
    _dev(q, subkeys, idx, grad_scores)
    T, H, n = q.shape
    S = subkeys.shape[2]
    k = idx.shape[2]
    if grad_q is None and want_grad_q:
        grad_q = torch.empty((T, H, n), dtype=torch.float32, device=q.device)
    if grad_subkeys is None and want_grad_subkeys:
        grad_subkeys = torch.zeros(subkeys.shape, dtype=torch.float32, device=q.device)
    _dev(grad_q, grad_subkeys)
    nbytes = int(L.mem_search_backward_workspace_size(T, H, S, k))
    ws = _workspace(nbytes, q.device, workspace)
    args = (_ptr(idx), _ptr(grad_scores), _ptr(grad_q), _ptr(grad_subkeys), _ptr(ws),
            ws.numel() * ws.element_size(), _stream(stream))
    if eps is None:
        _check(L.mem_search_backward(_ptr(q), _dt(q), _ptr(subkeys), _dt(subkeys), T, H, n, S, k,
                                     *args))
    else:
        _check(L.mem_search_backward_qnorm(_ptr(q), _dt(q), _ptr(subkeys), _dt(subkeys), T, H, n,
                                           S, k, eps, *args))
    return grad_q, grad_subkeys


@_launches_on_stream
def mem_bag_forward(values: torch.Tensor, idx: torch.Tensor, w: torch.Tensor, *, y_out=None,
                    stream=None):
    """y[t] = sum_j w[t, j] values[idx[t, j]]; idx, w of shape [T, ...] (bag = rest)."""
    L = load()
    _dev(values, idx, w)
    N, D = values.shape
    T = idx.shape[0]
    bag = idx.numel() // T if T else (idx[0].numel() if idx.dim() > 1 else 1)
    if idx.dtype != torch.int64 or w.dtype != torch.float32:
        raise TypeError("idx must be int64 and w float32")
    if y_out is None:
        y_out = torch.empty((T, D), dtype=values.dtype, device=values.device)
    _dev(y_out)
    _check(L.mem_bag_forward(_ptr(values), _dt(values), N, D, _ptr(idx), _ptr(w), T, bag,
                             _ptr(y_out), _stream(stream)))
    return y_out


@_launches_on_stream
def mem_bag_forward_gated(values: torch.Tensor, idx: torch.Tensor, w: torch.Tensor,
                          gate: torch.Tensor, *, want_y=True, out=None, y_out=None, stream=None):
    """Memory+ epilogue: out = bag * silu(gate), gate [T, D] in the value dtype.
    Returns (out, y) with y the un-gated bag (None unless want_y)."""
    L = load()
    _dev(values, idx, w, gate)
    N, D = values.shape
    T = idx.shape[0]
    bag = idx.numel() // T if T else (idx[0].numel() if idx.dim() > 1 else 1)
    if idx.dtype != torch.int64 or w.dtype != torch.float32:
        raise TypeError("idx must be int64 and w float32")
    if gate.dtype != values.dtype or tuple(gate.shape) != (T, D) or not gate.is_contiguous():
        raise ValueError("gate must be a contiguous [T, D] tensor of the value dtype")
    if out is None:
        out = torch.empty((T, D), dtype=values.dtype, device=values.device)
    if y_out is None and want_y:
        y_out = torch.empty((T, D), dtype=values.dtype, device=values.device)
    _dev(out, y_out)
    _check(L.mem_bag_forward_gated(_ptr(values), _dt(values), N, D, _ptr(idx), _ptr(w), T, bag,
                                   _ptr(gate), _ptr(y_out), _ptr(out), _stream(stream)))
    return out, y_out


@_launches_on_stream
def mem_gate_backward(d_out: torch.Tensor, gate: torch.Tensor, y: torch.Tensor, *, dy_out=None,
                      grad_gate=None, stream=None):
    """Backward of out = y * silu(gate): returns (dy [value dtype], grad_gate fp32)."""
    L = load()
    _dev(d_out, gate, y)
    T, D = d_out.shape
    for t_ in (gate, y):
        if t_.dtype != d_out.dtype or tuple(t_.shape) != (T, D) or not t_.is_contiguous():
            raise ValueError("gate and y must be contiguous [T, D] tensors of d_out's dtype")
    if dy_out is None:
        dy_out = torch.empty((T, D), dtype=d_out.dtype, device=d_out.device)
    if grad_gate is None:
        grad_gate = torch.empty((T, D), dtype=torch.float32, device=d_out.device)
    _dev(dy_out, grad_gate)
    _check(L.mem_gate_backward(_ptr(d_out), _ptr(gate), _ptr(y), _dt(d_out), T, D, _ptr(dy_out),
                               _ptr(grad_gate), _stream(stream)))
    return dy_out, grad_gate


@_launches_on_stream
def mem_bag_backward(dy: torch.Tensor, values: torch.Tensor, idx: torch.Tensor, w: torch.Tensor,
                     *, grad_values=None, grad_w=None, grad_scores=None, want_grad_values=True,
                     want_grad_w=True, want_grad_scores=True, mode="auto", workspace=None,
                     stream=None):
    """EmbeddingBag + softmax backward.  idx, w [T, H, k].  grad_values is
    ACCUMULATED into (a zero table is allocated if none is given)."""
    Lb = load()
    _dev(dy, values, idx, w)
    N, D = values.shape
    T, H, k = idx.shape
    dev = values.device
    if grad_values is None and want_grad_values:
        grad_values = torch.zeros((N, D), dtype=torch.float32, device=dev)
    if grad_w is None and want_grad_w:
        grad_w = torch.empty((T, H, k), dtype=torch.float32, device=dev)
    if grad_scores is None and want_grad_scores:
        grad_scores = torch.empty((T, H, k), dtype=torch.float32, device=dev)
    _dev(grad_values, grad_w, grad_scores)
    m = BWD_MODES[mode] if isinstance(mode, str) else int(mode)
    nbytes = int(Lb.mem_bag_backward_workspace_size(T, H, k, N, D, m))
    ws = _workspace(nbytes, dev, workspace)
    _check(Lb.mem_bag_backward(_ptr(dy), _ptr(values), _dt(values), N, D, _ptr(idx), _ptr(w), T,
                               H, k, _ptr(grad_values), _ptr(grad_w), _ptr(grad_scores), m,
                               _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))
    return grad_values, grad_w, grad_scores


@_launches_on_stream
def mem_bag_backward_sparse(dy: torch.Tensor, values: torch.Tensor, idx: torch.Tensor,
                            w: torch.Tensor, *, want_grad_w=True, want_grad_scores=True,
                            workspace=None, stream=None):
    """Backward with the value gradient as touched rows only.

    Returns (rows int64 [U], grad_rows fp32 [U, D], grad_w, grad_scores); waits
    for the stream to learn U.
    """
    Lb = load()
    _dev(dy, values, idx, w)
    N, D = values.shape
    T, H, k = idx.shape
    dev = values.device
    cap = max(1, min(T * H * k, N))
    rows = torch.empty((cap,), dtype=torch.int64, device=dev)
    grad_rows = torch.empty((cap, D), dtype=torch.float32, device=dev)
    grad_w = torch.empty((T, H, k), dtype=torch.float32, device=dev) if want_grad_w else None
    grad_scores = torch.empty((T, H, k), dtype=torch.float32, device=dev) if want_grad_scores else None
    nbytes = int(Lb.mem_bag_backward_workspace_size(T, H, k, N, D, BWD_MODES["sorted"]))
    ws = _workspace(nbytes, dev, workspace)
    U = ctypes.c_int64(0)
    _check(Lb.mem_bag_backward_sparse(_ptr(dy), _ptr(values), _dt(values), N, D, _ptr(idx),
                                      _ptr(w), T, H, k, _ptr(rows), _ptr(grad_rows), cap,
                                      ctypes.addressof(U), _ptr(grad_w), _ptr(grad_scores),
                                      _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))
    u = int(U.value)
    return rows[:u], grad_rows[:u], grad_w, grad_scores


# ------------------------------------------------ norm, projections, optimizer
def _here(*ts) -> None:
    """The tensors lie, dense, on the device the call launches on."""
    dev = -2  # of no tensor
    for t in ts:
        if t is not None:
            d = t.get_device()
            if d != dev:
                if d < 0:
                    raise ValueError("tensors must be on the GPU")
                if dev >= 0:
                    raise ValueError("tensors must be on one device")
                if d != _current_device():
                    raise ValueError("tensors must be on the current device")
                dev = d
            if not t.is_contiguous():
                raise ValueError("tensors must be contiguous")


def _like(t, shape, dtype, what: str) -> None:
    if t is not None and (t.shape != shape or t.dtype is not dtype):
        raise ValueError(f"{what} must be a {dtype} tensor of shape {tuple(shape)}")


@_launches_on_stream
def mem_rmsnorm(x: torch.Tensor, weight=None, residual=None, eps: float = 1e-5, *,
                quantize: bool = False, sum_out=None, y_out=None, scale_out=None,
                want_sum: bool = True, stream=None):
    """Root-mean-square norm of h = x + residual ([T, D]; residual may be None).

    Returns (y, h, scale): y in x's dtype and scale None, or with quantize y in
    float8_e4m3fn with scale fp32 [T] (the norm is about y * scale[:, None]); h None
    without a residual or with want_sum False unless sum_out is given (it may be x or
    residual)."""
    _here(x, weight, residual, sum_out, y_out, scale_out)
    shape, xdt = x.shape, x.dtype
    T, D = shape
    dt = ydt = _dt(x)
    wp = rp = hp = sp = None
    if weight is not None:
        _like(weight, (D,), xdt, "weight")
        wp = weight.data_ptr()
    if residual is not None:
        _like(residual, shape, xdt, "residual")
        rp = residual.data_ptr()
        if sum_out is None and want_sum:
            sum_out = torch.empty_like(x)
    if sum_out is not None:
        _like(sum_out, shape, xdt, "sum_out")
        hp = sum_out.data_ptr()
    if not quantize:
        if scale_out is not None:
            raise ValueError("scale_out is for quantize")
    else:
        xdt, ydt = torch.float8_e4m3fn, E4M3
        if scale_out is None:
            scale_out = torch.empty((T,), dtype=torch.float32, device=x.device)
        else:
            _like(scale_out, (T,), torch.float32, "scale_out")
        sp = scale_out.data_ptr()
    if y_out is None:
        y_out = torch.empty_like(x, dtype=xdt) if quantize else torch.empty_like(x)
    else:
        _like(y_out, shape, xdt, "y_out")
    _check((_LIB or load()).mem_rmsnorm(x.data_ptr(), rp, wp, dt, T, D, eps, hp, y_out.data_ptr(), ydt,
                                        sp, _stream(stream)))
    return y_out, sum_out, scale_out


@_launches_on_stream
def mem_rmsnorm_backward(dy: torch.Tensor, h: torch.Tensor, weight=None, eps: float = 1e-5, *,
                         dsum=None, dx=None, grad_weight=None, want_grad_weight: bool = True,
                         workspace=None, stream=None):
    """Backward of mem_rmsnorm: dy the gradient of y, h what was normalised (its sum,
    or x without a residual), dsum what reaches h along the stream (or None).
    Returns (dx [T, D] in dy's dtype, the gradient of x and residual alike; grad_weight
    fp32 [D], ACCUMULATED: zeros are allocated if none is given)."""
    L = load()
    _here(dy, h, weight, dsum, dx, grad_weight, workspace)
    T, D = dy.shape
    _like(h, (T, D), dy.dtype, "h")
    _like(weight, (D,), dy.dtype, "weight")
    _like(dsum, (T, D), dy.dtype, "dsum")
    if dx is None:
        dx = torch.empty_like(dy)
    _like(dx, (T, D), dy.dtype, "dx")
    if grad_weight is None and want_grad_weight:
        grad_weight = torch.zeros((D,), dtype=torch.float32, device=dy.device)
    _like(grad_weight, (D,), torch.float32, "grad_weight")
    ws = None
    if grad_weight is not None:
        ws = _workspace(int(L.mem_rmsnorm_backward_workspace_size(T, D)), dy.device, workspace)
    _check(L.mem_rmsnorm_backward(_ptr(dy), _ptr(h), _ptr(weight), _dt(dy), T, D, float(eps),
                                  _ptr(dsum), _ptr(dx), _ptr(grad_weight), _ptr(ws),
                                  0 if ws is None else ws.numel() * ws.element_size(),
                                  _stream(stream)))
    return dx, grad_weight


@_launches_on_stream
def mem_quantize_rows(x: torch.Tensor, *, q_out=None, scale_out=None, stream=None):
    """Rows of x [R, C] in 8 bits: (q float8_e4m3fn [R, C], scale fp32 [R]), x about
    q * scale[:, None]."""
    L = load()
    _here(x, q_out, scale_out)
    R, C = x.shape
    dt = _dt(x)
    if q_out is None:
        q_out = torch.empty((R, C), dtype=torch.float8_e4m3fn, device=x.device)
    _like(q_out, (R, C), torch.float8_e4m3fn, "q_out")
    if scale_out is None:
        scale_out = torch.empty((R,), dtype=torch.float32, device=x.device)
    _like(scale_out, (R,), torch.float32, "scale_out")
    _check(L.mem_quantize_rows(_ptr(x), dt, R, C, _ptr(q_out), _ptr(scale_out), _stream(stream)))
    return q_out, scale_out


def _act(act) -> int:
    return ACTIVATIONS[act] if isinstance(act, str) else int(act)


@_launches_on_stream
def mem_linear(x: torch.Tensor, w: torch.Tensor, bias=None, *, residual=None, act="none",
               x_scale=None, w_scale=None, out_dtype=None, y_out=None, z_out=None,
               want_z: bool = False, stream=None):
    """act(x w^T + bias) + residual: x [T, K], w [N, K], bias [N], residual [T, N].

    act: a name of ACTIVATIONS.  float8_e4m3fn operands come with x_scale [T] and
    w_scale [N] (mem_rmsnorm(quantize=True), mem_quantize_rows).  out_dtype: float32 or
    bfloat16 (default: x's, bfloat16 for 8 bits), the dtype of bias and residual too.
    Returns (y, z) with z = x w^T + bias before the activation, None unless want_z.
    y_out may be residual."""
    _here(x, w, bias, residual, x_scale, w_scale, y_out, z_out)
    T, K = x.shape
    N, xdt = w.shape[0], x.dtype
    _like(w, (N, K), xdt, "w")
    sx = sw = bp = rp = zp = None
    if xdt is torch.float8_e4m3fn:
        dt = E4M3
        if x_scale is None or w_scale is None:
            raise ValueError("float8_e4m3fn operands need x_scale and w_scale")
        _like(x_scale, (T,), torch.float32, "x_scale")
        _like(w_scale, (N,), torch.float32, "w_scale")
        sx, sw = x_scale.data_ptr(), w_scale.data_ptr()
    else:
        dt = _dt(x)
        sx, sw = _ptr(x_scale), _ptr(w_scale)  # refused by the call where given
    if out_dtype is None:
        out_dtype = torch.bfloat16 if dt == E4M3 else xdt
    shape = (T, N)
    if y_out is None:
        y_out = x.new_empty(shape, dtype=out_dtype)
    else:
        _like(y_out, shape, out_dtype, "y_out")
    if z_out is not None:
        _like(z_out, shape, out_dtype, "z_out")
        zp = z_out.data_ptr()
    elif want_z:
        z_out = x.new_empty(shape, dtype=out_dtype)
        zp = z_out.data_ptr()
    if bias is not None:
        _like(bias, (N,), out_dtype, "bias")
        bp = bias.data_ptr()
    if residual is not None:
        _like(residual, shape, out_dtype, "residual")
        rp = residual.data_ptr()
    _check((_LIB or load()).mem_linear(x.data_ptr(), w.data_ptr(), dt, sx, sw, bp, rp, T, N, K,
                                       _act(act), zp,
                                       y_out.data_ptr(), _dt(y_out), _stream(stream)))
    return y_out, z_out


@_launches_on_stream
def mem_act_backward(dy: torch.Tensor, z: torch.Tensor, act, *, dz_out=None, stream=None):
    """dz = dy * act'(z), [T, N]: what mem_linear_backward takes after mem_linear with an
    activation.  dz_out may be dy or z."""
    L = load()
    _here(dy, z, dz_out)
    T, N = dy.shape
    _like(z, (T, N), dy.dtype, "z")
    if dz_out is None:
        dz_out = torch.empty_like(dy)
    _like(dz_out, (T, N), dy.dtype, "dz_out")
    _check(L.mem_act_backward(_ptr(dy), _ptr(z), _dt(dy), _act(act), T, N, _ptr(dz_out),
                              _stream(stream)))
    return dz_out


@_launches_on_stream
def mem_linear_backward(dz: torch.Tensor, x: torch.Tensor, w: torch.Tensor, *, dx_add=None,
                        dx=None, grad_w=None, grad_bias=None, want_dx: bool = True,
                        want_grad_w: bool = True, want_grad_bias: bool = True, workspace=None,
                        stream=None):
    """Gradients of x w^T + bias from dz [T, N]: (dx = dz w + dx_add [T, K] in dz's dtype,
    grad_w fp32 [N, K] and grad_bias fp32 [N], both ACCUMULATED; zeros are allocated if
    none are given).  dx may be dx_add."""
    L = load()
    _here(dz, x, w, dx_add, dx, grad_w, grad_bias, workspace)
    T, N = dz.shape
    K = x.shape[1]
    _like(x, (T, K), dz.dtype, "x")
    _like(w, (N, K), dz.dtype, "w")
    _like(dx_add, (T, K), dz.dtype, "dx_add")
    dev = dz.device
    if dx is None and want_dx:
        dx = torch.empty((T, K), dtype=dz.dtype, device=dev)
    if grad_w is None and want_grad_w:
        grad_w = torch.zeros((N, K), dtype=torch.float32, device=dev)
    if grad_bias is None and want_grad_bias:
        grad_bias = torch.zeros((N,), dtype=torch.float32, device=dev)
    _like(dx, (T, K), dz.dtype, "dx")
    _like(grad_w, (N, K), torch.float32, "grad_w")
    _like(grad_bias, (N,), torch.float32, "grad_bias")
    dt = _dt(dz)
    nbytes = 0
    if grad_w is not None or grad_bias is not None:
        nbytes = int(L.mem_linear_backward_workspace_size(T, N, K, dt))
    ws = _workspace(nbytes, dev, workspace) if nbytes else None
    _check(L.mem_linear_backward(_ptr(dz), _ptr(x), _ptr(w), dt, T, N, K, _ptr(dx_add), _ptr(dx),
                                 _ptr(grad_w), _ptr(grad_bias), _ptr(ws),
                                 0 if ws is None else ws.numel() * ws.element_size(),
                                 _stream(stream)))
    return dx, grad_w, grad_bias


@_launches_on_stream
def mem_layernorm(x: torch.Tensor, weight=None, bias=None, residual=None, eps: float = 1e-5, *,
                  sum_out=None, y_out=None, want_sum: bool = True, stream=None):
    """Layer norm of h = x + residual ([T, D]; residual may be None).

    Returns (y, h), both in x's dtype; h None without a residual or with want_sum False
    unless sum_out is given (it may be x or residual)."""
    _here(x, weight, bias, residual, sum_out, y_out)
    shape, xdt = x.shape, x.dtype
    T, D = shape
    dt = _dt(x)
    wp = bp = rp = hp = None
    if weight is not None:
        _like(weight, (D,), xdt, "weight")
        wp = weight.data_ptr()
    if bias is not None:
        _like(bias, (D,), xdt, "bias")
        bp = bias.data_ptr()
    if residual is not None:
        _like(residual, shape, xdt, "residual")
        rp = residual.data_ptr()
        if sum_out is None and want_sum:
            sum_out = torch.empty_like(x)
    if sum_out is not None:
        _like(sum_out, shape, xdt, "sum_out")
        hp = sum_out.data_ptr()
    if y_out is None:
        y_out = torch.empty_like(x)
    else:
        _like(y_out, shape, xdt, "y_out")
    _check((_LIB or load()).mem_layernorm(x.data_ptr(), rp, wp, bp, dt, T, D, eps, hp, y_out.data_ptr(),
                                          _stream(stream)))
    return y_out, sum_out


@_launches_on_stream
def mem_layernorm_backward(dy: torch.Tensor, h: torch.Tensor, weight=None, eps: float = 1e-5, *,
                           dsum=None, dx=None, grad_weight=None, grad_bias=None,
                           want_grad_weight: bool = True, want_grad_bias: bool = True,
                           workspace=None, stream=None):
    """Backward of mem_layernorm: dy the gradient of y, h what was normalised (its sum, or x
    without a residual), dsum what reaches h along the stream (or None).  Returns (dx [T, D]
    in dy's dtype, the gradient of x and residual alike; grad_weight and grad_bias fp32 [D],
    ACCUMULATED: zeros are allocated if none is given)."""
    L = load()
    _here(dy, h, weight, dsum, dx, grad_weight, grad_bias, workspace)
    T, D = dy.shape
    dt = _dt(dy)
    _like(h, (T, D), dy.dtype, "h")
    _like(weight, (D,), dy.dtype, "weight")
    _like(dsum, (T, D), dy.dtype, "dsum")
    if dx is None:
        dx = torch.empty_like(dy)
    _like(dx, (T, D), dy.dtype, "dx")
    if grad_weight is None and want_grad_weight:
        grad_weight = torch.zeros((D,), dtype=torch.float32, device=dy.device)
    if grad_bias is None and want_grad_bias:
        grad_bias = torch.zeros((D,), dtype=torch.float32, device=dy.device)
    _like(grad_weight, (D,), torch.float32, "grad_weight")
    _like(grad_bias, (D,), torch.float32, "grad_bias")
    ws = None
    if grad_weight is not None or grad_bias is not None:
        ws = _workspace(int(L.mem_layernorm_backward_workspace_size(T, D)), dy.device, workspace)
    _check(L.mem_layernorm_backward(_ptr(dy), _ptr(h), _ptr(weight), dt, T, D, float(eps), _ptr(dsum),
                                    _ptr(dx), _ptr(grad_weight), _ptr(grad_bias), _ptr(ws),
                                    0 if ws is None else ws.numel() * ws.element_size(),
                                    _stream(stream)))
    return dx, grad_weight, grad_bias


@_launches_on_stream
def mem_glu(x: torch.Tensor, w: torch.Tensor, bias=None, *, act="silu", x_scale=None, w_scale=None,
            out_dtype=None, y_out=None, z_out=None, want_z: bool = False, stream=None):
    """The gated feed-forward part: with z = x w^T + bias, act(z[:, :N]) * z[:, N:].

    x [T, K]; w [2 N, K] (the gate's N rows, then the up projection's), bias [2 N]; act, 8-bit
    operands with x_scale [T] and w_scale [2 N], and out_dtype as for mem_linear.  bfloat16
    results of many 8-bit rows (more than 256 tiles of 128 x 128 of z) cut products 13 bits
    below the largest of 8 along K: ask for float32 where sums cancel.
    Returns (y [T, N], z [T, 2 N], None unless want_z)."""
    _here(x, w, bias, x_scale, w_scale, y_out, z_out)
    T, K = x.shape
    N2, xdt = w.shape[0], x.dtype
    _like(w, (N2, K), xdt, "w")
    if N2 % 2:
        raise ValueError("w must have a gate's and as many of an up projection's rows")
    sx = sw = bp = zp = None
    if xdt is torch.float8_e4m3fn:
        dt = E4M3
        if x_scale is None or w_scale is None:
            raise ValueError("float8_e4m3fn operands need x_scale and w_scale")
        _like(x_scale, (T,), torch.float32, "x_scale")
        _like(w_scale, (N2,), torch.float32, "w_scale")
    else:
        dt = _dt(x)
    sx, sw = _ptr(x_scale), _ptr(w_scale)  # refused by the call beside other operands
    if out_dtype is None:
        out_dtype = torch.bfloat16 if dt == E4M3 else xdt
    if y_out is None:
        y_out = x.new_empty((T, N2 // 2), dtype=out_dtype)
    else:
        _like(y_out, (T, N2 // 2), out_dtype, "y_out")
    if z_out is None and want_z:
        z_out = x.new_empty((T, N2), dtype=out_dtype)
    if z_out is not None:
        _like(z_out, (T, N2), out_dtype, "z_out")
        zp = z_out.data_ptr()
    if bias is not None:
        _like(bias, (N2,), out_dtype, "bias")
        bp = bias.data_ptr()
    _check((_LIB or load()).mem_glu(x.data_ptr(), w.data_ptr(), dt, sx, sw, bp, T, N2 // 2, K, _act(act),
                                    zp, y_out.data_ptr(), _dt(y_out), _stream(stream)))
    return y_out, z_out


@_launches_on_stream
def mem_glu_backward(dy: torch.Tensor, z: torch.Tensor, act="silu", *, dz_out=None, stream=None):
    """dz [T, 2 N] of mem_glu from dy [T, N] and its z [T, 2 N]; dz_out may be z.  Then
    mem_linear_backward(dz, x, w) gives the gradients of x, w and bias."""
    L = load()
    _here(dy, z, dz_out)
    T, N = dy.shape
    dt = _dt(dy)
    _like(z, (T, 2 * N), dy.dtype, "z")
    if dz_out is None:
        dz_out = torch.empty_like(z)
    _like(dz_out, (T, 2 * N), dy.dtype, "dz_out")
    _check(L.mem_glu_backward(_ptr(dy), _ptr(z), dt, _act(act), T, N, _ptr(dz_out), _stream(stream)))
    return dz_out


@_launches_on_stream
def mem_quantize_blocks(x: torch.Tensor, *, tile: bool = False, want_rows: bool = True,
                        want_cols: bool = False, q_out=None, scale_out=None, qt_out=None,
                        scale_t_out=None, stream=None):
    """x [R, C] in 8 bits with a scale for each 128 elements of a row (tile: each 128 x 128).

    Returns (q, scale, qt, scale_t), what is not wanted None: q float8_e4m3fn [R, C] with scale
    fp32 [ceil(C/128), R] (tile: [ceil(C/128), ceil(R/128)]), and the same of x's columns:
    qt [C, R rounded up to 16] (zeros past R) with scale_t [ceil(R/128), C] (tile:
    [ceil(R/128), ceil(C/128)]).  They are operands of mem_linear_blocks."""
    _here(x, q_out, scale_out, qt_out, scale_t_out)
    R, C = x.shape
    dt = _dt(x)
    rb, cb = -(-R // SCALE_BLOCK), -(-C // SCALE_BLOCK)
    qp = sp = qtp = stp = None
    if want_rows or q_out is not None or scale_out is not None:
        shape, sshape = (R, C), (cb, rb if tile else R)
        if q_out is None:
            q_out = x.new_empty(shape, dtype=torch.float8_e4m3fn)
        else:
            _like(q_out, shape, torch.float8_e4m3fn, "q_out")
        if scale_out is None:
            scale_out = x.new_empty(sshape, dtype=torch.float32)
        else:
            _like(scale_out, sshape, torch.float32, "scale_out")
        qp, sp = q_out.data_ptr(), scale_out.data_ptr()
    if want_cols or qt_out is not None or scale_t_out is not None:
        shape, sshape = (C, -(-R // 16) * 16), (rb, cb if tile else C)
        if qt_out is None:
            qt_out = x.new_empty(shape, dtype=torch.float8_e4m3fn)
        else:
            _like(qt_out, shape, torch.float8_e4m3fn, "qt_out")
        if scale_t_out is None:
            scale_t_out = x.new_empty(sshape, dtype=torch.float32)
        else:
            _like(scale_t_out, sshape, torch.float32, "scale_t_out")
        qtp, stp = qt_out.data_ptr(), scale_t_out.data_ptr()
    if R:  # empty tensors have no address
        _check((_LIB or load()).mem_quantize_blocks(x.data_ptr(), dt, R, C, bool(tile), qp, sp, qtp, stp,
                                                    _stream(stream)))
    return q_out, scale_out, qt_out, scale_t_out


@_launches_on_stream
def mem_linear_blocks(x: torch.Tensor, w: torch.Tensor, x_scale: torch.Tensor, w_scale: torch.Tensor,
                      bias=None, *, residual=None, act="none", out_dtype=None, y_out=None, z_out=None,
                      want_z: bool = False, workspace=None, stream=None):
    """act(x w^T + bias) + residual for float8_e4m3fn operands x [T, K] and w [N, K] with a scale
    for each 128 along K: x_scale [ceil(K/128), T], w_scale [ceil(K/128), N] or, for
    128 x 128 tiles, [ceil(K/128), ceil(N/128)] (mem_quantize_blocks).

    out_dtype: float32 or bfloat16 (the default), the dtype of bias and residual too; in
    float32, and for up to 8 rows, products are exact, else they are cut 13 bits below the
    largest of 8 along K: ask for float32 where sums cancel.  y_out may be residual.  Returns (y, z) with z = x w^T + bias
    before the activation, None unless want_z."""
    _here(x, w, x_scale, w_scale, bias, residual, y_out, z_out, workspace)
    T, K = x.shape
    N = w.shape[0]
    if x.dtype is not torch.float8_e4m3fn:
        raise TypeError(f"unsupported dtype {x.dtype} (float8_e4m3fn)")
    _like(w, (N, K), torch.float8_e4m3fn, "w")
    kb, nb = -(-K // SCALE_BLOCK), -(-N // SCALE_BLOCK)
    _like(x_scale, (kb, T), torch.float32, "x_scale")
    tiled = tuple(w_scale.shape) == (kb, nb)
    _like(w_scale, (kb, nb if tiled else N), torch.float32, "w_scale")
    if out_dtype is None:
        out_dtype = torch.bfloat16
    shape = (T, N)
    zp = bp = rp = None
    if y_out is None:
        y_out = x.new_empty(shape, dtype=out_dtype)
    else:
        _like(y_out, shape, out_dtype, "y_out")
    if z_out is None and want_z:
        z_out = x.new_empty(shape, dtype=out_dtype)
    if z_out is not None:
        _like(z_out, shape, out_dtype, "z_out")
        zp = z_out.data_ptr()
    if bias is not None:
        _like(bias, (N,), out_dtype, "bias")
        bp = bias.data_ptr()
    if residual is not None:
        _like(residual, shape, out_dtype, "residual")
        rp = residual.data_ptr()
    L, ydt = _LIB or load(), _dt(y_out)
    wsp = nbytes = 0
    if ydt == F32:
        nbytes = L.mem_linear_blocks_workspace_size(T, N, K, ydt)
        if nbytes:
            ws = _workspace(nbytes, x.device, workspace)
            wsp, nbytes = ws.data_ptr(), ws.numel() * ws.element_size()
    _check(L.mem_linear_blocks(x.data_ptr(), w.data_ptr(), x_scale.data_ptr(), w_scale.data_ptr(), tiled, bp, rp,
                               T, N, K, _act(act), zp, y_out.data_ptr(), ydt, wsp, nbytes, _stream(stream)))
    return y_out, z_out


class _AdamwTensor(ctypes.Structure):  # pkmem_adamw_tensor
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "exp_avg", "exp_avg_sq",
                                               "exp_avg_scale", "exp_avg_sq_scale")]
    _fields_ += [("numel", ctypes.c_int64)]
    _fields_ += [(n, ctypes.c_int) for n in ("param_dt", "grad_dt", "state_dt")]


_ADAMW_PACK = struct.Struct("6Pq3i4x")  # the same, several times faster to fill


class _AdamwOpts(ctypes.Structure):  # pkmem_adamw_opts
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")]
    _fields_ += [("step", ctypes.c_int64), ("seed", ctypes.c_uint64)]
    _fields_ += [(n, ctypes.c_void_p) for n in ("lr_dev", "step_dev", "grad_scale")]


def mem_adamw_state(param: torch.Tensor, bits: int = 32):
    """Zero states of mem_adamw for one parameter: (exp_avg, exp_avg_sq, exp_avg_scale,
    exp_avg_sq_scale), fp32 with scales None, or with bits = 8 float8_e4m3fn (the second
    one the square root) with an fp32 scale per 128 elements."""
    if bits == 32:
        return (*(torch.zeros(param.shape, dtype=torch.float32, device=param.device)
                  for _ in range(2)), None, None)
    if bits != 8:
        raise ValueError("states have 32 or 8 bits")
    codes = [torch.zeros(param.shape, dtype=torch.uint8, device=param.device).view(torch.float8_e4m3fn)
             for _ in range(2)]
    blocks = -(-param.numel() // ADAMW_STATE_BLOCK)
    return (*codes, *(torch.zeros((blocks,), dtype=torch.float32, device=param.device)
                      for _ in range(2)))


_DT = {torch.float32: F32, torch.bfloat16: BF16}
_ADAMW_STATES = {torch.float32: F32, torch.float8_e4m3fn: E4M3}


def _adamw_tensor(p, g, m, v, sm, sv, gshape) -> tuple:
    """The checked fields of one _AdamwTensor."""
    _here(p, g, m, v, sm, sv)
    shape, sdt = p.shape, m.dtype
    if m.shape != shape or v.shape != shape or g.shape != gshape:
        raise ValueError("states must have the parameter's shape, gradients their own")
    if v.dtype is not sdt or sdt not in _ADAMW_STATES:
        raise TypeError("states must both be float32 or both float8_e4m3fn")
    if p.dtype not in _DT or g.dtype not in _DT:
        raise TypeError("parameters and gradients must be float32 or bfloat16")
    n = p.numel()
    if sdt is torch.float32:
        if sm is not None or sv is not None:
            raise ValueError("scales belong to float8_e4m3fn states")
        sm = sv = 0
    else:
        blocks = -(-n // ADAMW_STATE_BLOCK)
        for s in (sm, sv):
            if s is None or s.dtype is not torch.float32 or s.numel() != blocks:
                raise ValueError(f"float8_e4m3fn states need fp32 scales, one per {ADAMW_STATE_BLOCK} elements")
        sm, sv = sm.data_ptr(), sv.data_ptr()
    return (p.data_ptr(), g.data_ptr(), m.data_ptr(), v.data_ptr(), sm, sv, n, _DT[p.dtype],
            _DT[g.dtype], _ADAMW_STATES[sdt])


def _adamw_opts(lr, betas, eps, weight_decay, step, seed, grad_scale) -> _AdamwOpts:
    fixed_lr, fixed_step, lr_dev, step_dev, scale = lr, step, None, None, None
    if isinstance(lr, torch.Tensor):
        _like(lr.reshape(-1), (1,), torch.float32, "lr")
        _here(lr)
        fixed_lr, lr_dev = 0.0, lr.data_ptr()
    if isinstance(step, torch.Tensor):
        _like(step.reshape(-1), (1,), torch.int64, "step")
        _here(step)
        fixed_step, step_dev = 0, step.data_ptr()
    if grad_scale is not None:
        _like(grad_scale.reshape(-1), (1,), torch.float32, "grad_scale")
        _here(grad_scale)
        scale = grad_scale.data_ptr()
    return _AdamwOpts(fixed_lr, betas[0], betas[1], eps, weight_decay, int(fixed_step),
                      int(seed) & 0xFFFFFFFFFFFFFFFF, lr_dev, step_dev, scale)


@_launches_on_stream
def mem_adamw(params, grads, exp_avgs, exp_avg_sqs, *, lr, step, betas=(0.9, 0.999),
              eps: float = 1e-8, weight_decay: float = 0.01, exp_avg_scales=None,
              exp_avg_sq_scales=None, grad_scale=None, seed: int = 0, stream=None) -> None:
    """One AdamW step on lists of tensors, in place (states: mem_adamw_state).

    lr: a number or an fp32 device scalar; step: 1, 2, ... or an int64 device scalar;
    grad_scale: an fp32 device scalar that multiplies the gradients (0 or not finite: the
    step changes nothing).  exp_avg_scales, exp_avg_sq_scales: lists of the 8-bit states'
    scales (None entries for 32-bit ones).  seed: of the rounding of bf16 parameters and
    8-bit states; the step number is mixed in."""
    L = load()
    n = len(params)
    none = [None] * n
    sms = none if exp_avg_scales is None else exp_avg_scales
    svs = none if exp_avg_sq_scales is None else exp_avg_sq_scales
    if not len(grads) == len(exp_avgs) == len(exp_avg_sqs) == len(sms) == len(svs) == n:
        raise ValueError("lists of different lengths")
    size = _ADAMW_PACK.size
    ts = ctypes.create_string_buffer(max(n, 1) * size)
    for i, (p, g, m, v, sm, sv) in enumerate(zip(params, grads, exp_avgs, exp_avg_sqs, sms, svs)):
        _ADAMW_PACK.pack_into(ts, i * size, *_adamw_tensor(p, g, m, v, sm, sv, p.shape))
    o = _adamw_opts(lr, betas, eps, weight_decay, step, seed, grad_scale)
    _check(L.mem_adamw(ctypes.addressof(ts), n, ctypes.addressof(o), _stream(stream)))


@_launches_on_stream
def mem_adamw_rows(param: torch.Tensor, rows: torch.Tensor, grad_rows: torch.Tensor,
                   exp_avg: torch.Tensor, exp_avg_sq: torch.Tensor, *, lr, step,
                   betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                   exp_avg_scale=None, exp_avg_sq_scale=None, grad_scale=None, seed: int = 0,
                   stream=None) -> None:
    """One AdamW step, in place, on the rows of param [N, D] that rows (int64 [U],
    ascending) names, with their gradients grad_rows fp32 [U, D]: what
    mem_bag_backward_sparse returns.  The other rows keep value and states.  Arguments
    as mem_adamw's."""
    L = load()
    N, D = param.shape
    U = rows.numel()
    _here(param, rows)
    _like(rows, (U,), torch.int64, "rows")
    if grad_rows.dtype is not torch.float32:
        raise TypeError("gradients of rows must be float32")
    t = _AdamwTensor(*_adamw_tensor(param, grad_rows, exp_avg, exp_avg_sq, exp_avg_scale,
                                    exp_avg_sq_scale, (U, D)))
    o = _adamw_opts(lr, betas, eps, weight_decay, step, seed, grad_scale)
    _check(L.mem_adamw_rows(ctypes.addressof(t), N, D, _ptr(rows), U, ctypes.addressof(o),
                            _stream(stream)))
