"""Slow fp64 reference of what stands between the matrix products of a decoder layer.

NumPy, element by element where that is clearer; written from the definitions in include/qg_layer.h and sharing no code
with the library.  Test infrastructure only.
"""
from __future__ import annotations

import numpy as np

BLOCK = 64
FLOOR = 2.0 ** -40
QMAX = {"i8": 127.0, "e4m3": 448.0}


def scale_of(values: np.ndarray, kv: str = "i8") -> float:
    """The 8-bit scale of all of `values`."""
    a = np.max(np.abs(values)) if values.size else 0.0
    if not np.isfinite(a):
        return float("nan")
    return max(float(a) / QMAX[kv], FLOOR)


def norm(x, residual, w, eps):
    """(h, y): sum and norm, fp64 rows."""
    h = np.asarray(x, np.float64)
    if residual is not None:
        h = h + np.asarray(residual, np.float64)
    with np.errstate(all="ignore"):
        y = h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps) * np.asarray(w, np.float64)
    return h, y


def gate(g, u):
    g, u = np.asarray(g, np.float64), np.asarray(u, np.float64)
    with np.errstate(all="ignore"):
        return g / (1.0 + np.exp(-g)) * u


# ---- 8-bit numbers ---------------------------------------------------------------------------

def table(kv: str) -> np.ndarray:
    """The number that each of the 256 bytes stands for."""
    out = np.empty(256)
    for u in range(256):
        if kv == "i8":
            out[u] = u - 128
            continue
        e, m, sign = (u >> 3) & 15, u & 7, -1.0 if u >> 7 else 1.0
        if e == 15 and m == 7:
            out[u] = np.nan
        else:
            out[u] = sign * (m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return out


def half_step(x: np.ndarray, kv: str) -> np.ndarray:
    """How far the nearest 8-bit number may be from x (in units of the scale, |x| <= QMAX)."""
    if kv == "i8":
        return np.full_like(np.asarray(x, np.float64), 0.5)
    return np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10)


# ---- the cache's layout ------------------------------------------------------------------------

def key_byte(token: int, d: int, D: int) -> int:
    t, i = divmod(token, 16)
    c, rest = divmod(d, 64)
    b, e = divmod(rest, 16)
    return (((t * (D // 64) + c) * 4 + b) * 16 + i) * 16 + e


def value_byte(token: int, d: int, D: int) -> int:
    f, i = divmod(d, 16)
    t, rest = divmod(token, 16)
    b, r = divmod(rest, 4)
    return ((f * 4 + b) * 16 + i) * 16 + 4 * t + r


def order(name: str, D: int) -> np.ndarray:
    """[64, D] byte places of a block."""
    at = key_byte if name == "k" else value_byte
    return np.array([[at(j, d, D) for d in range(D)] for j in range(BLOCK)])


def block_values(codes: np.ndarray, scale: np.ndarray, name: str, kv: str, D: int) -> np.ndarray:
    """bytes [heads, 64 D], scale [heads] -> values [64, heads, D]."""
    x = table(kv)[codes[:, order(name, D)]]
    return np.transpose(x * np.asarray(scale, np.float64)[:, None, None], (1, 0, 2))


def sequence_values(codes, scale, blocks, length, name, kv, D):
    """Values [length, heads, D] and whether each token's block is there."""
    heads = codes.shape[1]
    out, there = np.zeros((length, heads, D)), np.zeros(length, bool)
    for i in range(-(-length // BLOCK)):
        lo, hi = i * BLOCK, min(length, i * BLOCK + BLOCK)
        if i < len(blocks) and 0 <= blocks[i] < codes.shape[0]:
            out[lo:hi] = block_values(codes[blocks[i]], scale[blocks[i]], name, kv, D)[:hi - lo]
            there[lo:hi] = True
    return out, there


# ---- rotation, attention -------------------------------------------------------------------------

def rotate(x, cos, sin, pos, neighbours):
    """x [rows, heads, D], tables [positions, rot/2], pos [rows]."""
    x = np.asarray(x, np.float64).copy()
    if cos is None:
        return x
    half = cos.shape[1]
    for r, p in enumerate(pos):
        p = min(int(p), cos.shape[0] - 1)
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
            u, v = x[r, :, a].copy(), x[r, :, b].copy()
            c, s = float(cos[p, i]), float(sin[p, i])
            x[r, :, a], x[r, :, b] = u * c - v * s, v * c + u * s
    return x


def attention(q, k, v, there, before, scale, causal, window):
    """q [rows, q_heads, D], k, v [length, kv_heads, D]: (out, error terms).

    The second result is, per output, sum_t p_t |v_t| and the largest sum_d |q_d k_td| of a seen token: what rounding errors of the
    probabilities and of the scores are measured by."""
    rows, Hq, D = q.shape
    length, H = k.shape[:2]
    G = Hq // H
    out, weight, reach = np.zeros((rows, Hq, D)), np.zeros((rows, Hq, D)), np.zeros((rows, Hq, 1))
    t = np.arange(length)
    for j in range(rows):
        pos = before + j
        see = there.copy()
        if causal:
            see &= t <= pos
        if window:
            see &= t > pos - window
        if not see.any():
            continue
        for h in range(Hq):
            kk, vv = k[see, h // G], v[see, h // G]
            with np.errstate(invalid="ignore"):
                s = scale * (kk @ q[j, h])
                p = np.exp(s - np.max(s))
                p /= np.sum(p)
                out[j, h], weight[j, h] = p @ vv, p @ np.abs(vv)
                reach[j, h] = scale * np.max(np.abs(kk) @ np.abs(q[j, h]))
    return out, weight, reach
