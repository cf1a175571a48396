"""Plain fp64 oracle of what stands around the memory in a block: the
root-mean-square norm, rows in 8 bits, the projections and AdamW.

TEST INFRASTRUCTURE ONLY: NumPy float64, one primitive per step, no code
shared with the HIP library.  Roundings that belong to a definition (e4m3
codes, states in 8 bits, bf16 parameters) are computed on the grid itself.
"""
from __future__ import annotations

import math

import numpy as np

E4M3_MAX = 448.0
BLOCK = 128


# --------------------------------------------------------------- e4m3 codes ----
def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes (4 bits of exponent, bias 7; the two
    codes of all ones are NaN, there is no infinity)."""
    v = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        x = (m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = math.nan if (e, m) == (15, 7) else (-x if s else x)
    return v


_POS = e4m3_values()[:127]  # ascending: 0 .. 448


def to_e4m3(x: np.ndarray) -> np.ndarray:
    """Values on the e4m3 grid nearest to x (|x| <= 464), ties to the even code."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_POS, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POS[lo], _POS[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return np.copysign(_POS[np.where(up, hi, lo)], x)


def quantize_rows(y: np.ndarray):
    """(values on the grid, scales) of rows: scale = max(max|y| / 448, 2^-126)."""
    s = np.maximum(np.abs(y).max(-1) / E4M3_MAX, 2.0 ** -126)
    return to_e4m3(y / s[:, None]), s


# --------------------------------------------------------------------- norm ----
def rmsnorm(h, w, eps):
    ss = (h * h).mean(-1, keepdims=True) + eps
    rstd = np.where(ss == 0, 0.0, 1 / np.sqrt(np.where(ss == 0, 1.0, ss)))
    return h * rstd * w


def rmsnorm_backward(dy, h, w, eps, dsum=None):
    """(dx, grad_weight) of sum(dy * rmsnorm(h)), plus dsum into dx."""
    ss = (h * h).mean(-1, keepdims=True) + eps
    rstd = np.where(ss == 0, 0.0, 1 / np.sqrt(np.where(ss == 0, 1.0, ss)))
    xh, g = h * rstd, dy * w
    dx = rstd * (g - xh * (g * xh).mean(-1, keepdims=True))
    return (dx if dsum is None else dx + dsum), (dy * xh).sum(0)


def _layer_stats(h, eps):
    d = h - h.mean(-1, keepdims=True)
    var = (d * d).mean(-1, keepdims=True) + eps
    return d, np.where(var == 0, 0.0, 1 / np.sqrt(np.where(var == 0, 1.0, var)))


def layernorm(h, w, b, eps):
    d, rstd = _layer_stats(h, eps)
    return d * rstd * w + b


def layernorm_backward(dy, h, w, eps, dsum=None):
    """(dx, grad_weight, grad_bias) of sum(dy * layernorm(h)), plus dsum into dx."""
    d, rstd = _layer_stats(h, eps)
    xh, g = d * rstd, dy * w
    dx = rstd * (g - g.mean(-1, keepdims=True) - xh * (g * xh).mean(-1, keepdims=True))
    return (dx if dsum is None else dx + dsum), (dy * xh).sum(0), dy.sum(0)


# -------------------------------------------------------------- projections ----
_erf = np.vectorize(math.erf, otypes=[float])


def act(z, name):
    if name == "relu":
        return np.where(z > 0, z, 0.0)
    if name == "silu":
        return z / (1 + np.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + _erf(z / math.sqrt(2)))
    return z


def act_grad(z, name):
    if name == "relu":
        return (z > 0).astype(float)
    if name == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return np.ones_like(z)


def linear(x, w, bias=None, res=None, name="none"):
    """(y, z): z = x w^T + bias, y = act(z) + res."""
    z = x @ w.T
    if bias is not None:
        z = z + bias
    y = act(z, name)
    return (y if res is None else y + res), z


def linear_backward(dz, x, w, add=None):
    """(dx, grad_w, grad_bias)."""
    dx = dz @ w
    return (dx if add is None else dx + add), dz.T @ x, dz.sum(0)


def glu(x, w, b, name):
    """(act(gate) * up, z) with z = x w^T + b, its first half the gate."""
    z = x @ w.T + b
    n = z.shape[1] // 2
    return act(z[:, :n], name) * z[:, n:], z


def glu_backward(dy, z, name):
    n = z.shape[1] // 2
    gate, up = z[:, :n], z[:, n:]
    return np.concatenate([dy * up * act_grad(gate, name), dy * act(gate, name)], 1)


# ------------------------------------------------------------ 8 bits in blocks ----
def quantize_blocks(x, rows):
    """(values on the grid, scale of each element, scales [column block, row block]) of x in
    blocks of `rows` x 128: scale = max(max|x| / 448, 2^-126)."""
    R, C = x.shape
    q, each = np.empty_like(x), np.empty_like(x)
    s = np.empty((-(-C // BLOCK), -(-R // rows)))
    for j in range(s.shape[0]):
        for i in range(s.shape[1]):
            at = np.s_[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK]
            big = np.abs(x[at]).max()
            low = big < E4M3_MAX * 2.0 ** -126
            s[j, i] = 2.0 ** -126 if low else big / E4M3_MAX
            each[at] = s[j, i]
            # 448 x / max: exact where it lies on a border
            q[at] = to_e4m3(x[at] * 2.0 ** 126 if low else x[at] * E4M3_MAX / big)
    return q, each, s


# -------------------------------------------------------------------- AdamW ----
def adamw(p, g, m, v, lr, betas, eps, wd, t):
    """(p, m, v) after step t, unrounded."""
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    mh, vh = m / (1 - b1 ** t), v / (1 - b2 ** t)
    return p - lr * wd * p - lr * mh / (np.sqrt(vh) + eps), m, v


def _mix(x):
    x = np.asarray(x, np.uint64)
    M = np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667)) & M
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85)) & M
    return x ^ (x >> np.uint64(16))


def random_bits(at, seed, step, tensor=0):
    """The 32 bits that decide the roundings of the elements at places `at`."""
    M = 0xFFFFFFFF
    k = int(_mix(seed & M))
    k = int(_mix((k + (seed >> 32)) & M))
    k = int(_mix((k + step) & M))
    k = (k + tensor * 0x9E3779B1) & M
    at = np.asarray(at, np.uint64)
    hi = ((at >> np.uint64(32)) * np.uint64(0x3C6EF373)) & np.uint64(M)
    return _mix((((at & np.uint64(M)) + np.uint64(k)) & np.uint64(M)) ^ hi).astype(np.int64)


def bf16_up(p, bits):
    """(lower neighbour in magnitude, upper, up?, distance of the decision from its
    border in units of the cut-off part) of rounding fp64 p to bf16 by 12 random bits."""
    a = np.abs(p)
    e = np.floor(np.log2(np.where(a > 0, a, 1.0)))
    step = 2.0 ** (np.maximum(e, -126) - 7)
    lo = np.floor(a / step) * step
    frac = (a - lo) / step
    u = ((bits & 0xFFF) + 0.5) / 4096
    return np.copysign(lo, p), np.copysign(lo + step, p), frac + u >= 1, np.abs(frac + u - 1)


def state_up(x, bits, width, nonzero):
    """Blocks of 128 on the e4m3 grid by random bits (`width` of them): (scales, value
    if rounded down, value if rounded up, up?, distance of the decision from its border)."""
    n = x.size
    pad = np.zeros(-(-n // BLOCK) * BLOCK)
    pad[:n] = x.reshape(-1)
    s = np.abs(pad).reshape(-1, BLOCK).max(-1) / E4M3_MAX
    s = np.where(s < 2.0 ** -126, 0.0, s)
    full = np.repeat(s, BLOCK)[:n]
    a = np.where(full > 0, np.abs(x.reshape(-1)) / np.where(full > 0, full, 1), 0.0)
    e = np.maximum(np.floor(np.log2(np.where(a > 0, a, 1e-30))), -6)
    step = 2.0 ** (e - 3)
    lo = np.floor(a / step) * step
    frac = (a - lo) / step
    u = (bits.reshape(-1) + 0.5) / 2 ** width
    hi = np.minimum(lo + step, E4M3_MAX)
    if nonzero:
        lo = np.where((a > 0) & (lo == 0), 2.0 ** -9, lo)
    sign = np.where(x.reshape(-1) < 0, -1.0, 1.0)
    return s, sign * lo, sign * hi, frac + u >= 1, np.abs(frac + u - 1)
