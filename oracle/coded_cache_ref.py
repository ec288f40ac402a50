"""The cache held in 8 bits and attention with a window, in 64 bits, from their definitions (no GPU, no kernels of the package).

Blocks of 64 tokens of a KV head.  int8: scale = amax / 127 to 32 bits and then to 16 significant ones, code = nearest integer to x / scale;
e4m3: scale = the smallest power of two with amax <= 448 scale, code = x / scale in 4 exponent and 3 fraction bits; ties to even in both."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 64
INT8, E4M3 = 0, 1
TINY = 2.0 ** -100


def half_even(x):
    return np.rint(np.asarray(x, np.float64))


def scale_of(x, fmt):
    """Scale of a block x (any shape); NaN if it holds one, or an infinity."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return math.nan
    amax = float(np.abs(x).max())
    if amax < TINY:
        return 0.0
    if fmt == INT8:
        m, e = math.frexp(float(np.float32(np.float32(amax) / np.float32(127))))
        s = float(half_even(m * 65536.0))
        if 127.0 * math.ldexp(s / 65536.0, e) > float(np.finfo(np.float32).max):       # (down, where the largest code would read as infinity)
            s -= 1.0
        return math.ldexp(s / 65536.0, e)
    e = math.frexp(amax)[1] - 10
    while amax > math.ldexp(448.0, e):
        e += 1
    return math.ldexp(1.0, e)


def e4m3(x):
    """x (|x| <= 448) rounded to e4m3."""
    x = np.asarray(x, np.float64)
    step = np.ldexp(1.0, np.maximum(np.frexp(x)[1] - 1, -6) - 3)
    return half_even(x / step) * step


def held(x, fmt):
    """Rows x [n, d] of a KV head as the cache holds them."""
    x = np.asarray(x, np.float64)
    out = x.copy()
    for p in range(x.shape[0] // BLOCK):
        rows = slice(p * BLOCK, (p + 1) * BLOCK)
        s = scale_of(x[rows], fmt)
        if s == 0.0:
            out[rows] = 0.0
        elif s != s:
            out[rows] = math.nan
        else:
            out[rows] = (half_even(x[rows] / s) if fmt == INT8 else e4m3(x[rows] / s)) * s
    return out


def seen(n, m, sinks, window):
    """[m, n]: what the last m of n tokens attend."""
    p, t = np.arange(n - m, n)[:, None], np.arange(n)
    return (t <= p) & ((t < sinks) | (t > p - window))


def attend(q, K, V, sinks, window):
    """q [m, Hq, d], K, V [Hkv, n, d] -> out [m, Hq, d], lse [m, Hq], and for each the largest sum |q_c k_c| / sqrt(d) over the keys seen.
    Tokens that a query does not see have no part, whatever they are."""
    m, Hq, d = q.shape
    Hkv, n, _ = K.shape
    see = seen(n, m, sinks, window)
    out, lse = np.zeros((m, Hq, d)), np.zeros((m, Hq))
    for i in range(m):
        t = np.nonzero(see[i])[0]
        for h in range(Hkv):
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            with np.errstate(all="ignore"):
                s = q[i, heads] @ K[h, t].T / math.sqrt(d)
                top = s.max(1, keepdims=True)
                w = np.exp(s - np.where(np.isfinite(top), top, 0.0))
                total = w.sum(1, keepdims=True)
                out[i, heads] = (w @ V[h, t]) / total
                lse[i, heads] = (top + np.log(total))[:, 0]
    return out, lse
