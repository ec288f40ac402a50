"""Plain definitions, in 64 bits, of the operators beside the top-k decode: rotary appends, dense and block-sparse attention of one new
token, accumulated attention weight, eviction.  NumPy, one sequence at a time; nothing here is shared with the library."""
from __future__ import annotations

import numpy as np

PAGE = 64


def rms_rotate(x, weight, eps, positions, inv_freq, interleaved):
    """x [n, heads, d], weight [d] or None, positions [n], inv_freq [r / 2] -> [n, heads, d], not rounded."""
    y = np.asarray(x, dtype=np.float64).copy()
    if weight is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + float(eps)) * np.asarray(weight, dtype=np.float64)
    r = 2 * len(inv_freq)
    t = np.asarray(positions, dtype=np.float64)[:, None, None] * np.asarray(inv_freq, dtype=np.float64)
    first, second = (np.s_[..., 0:r:2], np.s_[..., 1:r:2]) if interleaved else (np.s_[..., :r // 2], np.s_[..., r // 2:r])
    a, b = y[first].copy(), y[second].copy()
    y[first], y[second] = a * np.cos(t) - b * np.sin(t), b * np.cos(t) + a * np.sin(t)
    return y


def attend(q, K, V, positions=None):
    """q [Hq, d], K, V [Hkv, N, d] float64, positions: per KV head the tokens attended (None: all)
    -> out [Hq, d], lse [Hq], mass [Hkv, N] (weight of each key, summed over the group's heads)."""
    Hq, d = q.shape
    Hkv, N, _ = K.shape
    G = Hq // Hkv
    out, lse, mass = np.empty((Hq, d)), np.empty(Hq), np.zeros((Hkv, N))
    for h in range(Hq):
        at = np.arange(N) if positions is None else np.asarray(positions[h // G])
        s = (K[h // G][at] @ q[h]) / np.sqrt(d)
        e = np.exp(s - s.max())
        out[h], lse[h] = (e / e.sum()) @ V[h // G][at], s.max() + np.log(e.sum())
        mass[h // G, at] += e / e.sum()
    return out, lse, mass


def page_scores(q, K):
    """[Hkv, P]: per page the largest over the group's heads of sum_c max(q_c lo_c, q_c hi_c)."""
    Hkv, N, d = K.shape
    q = q.reshape(Hkv, -1, d)
    pages = [K[:, p:p + PAGE] for p in range(0, N, PAGE)]
    lo, hi = np.stack([p.min(1) for p in pages], 1), np.stack([p.max(1) for p in pages], 1)
    return np.maximum(q[:, :, None] * lo[:, None], q[:, :, None] * hi[:, None]).sum(-1).max(1)


def pick_blocks(q, K, n_blocks):
    """Per KV head the ascending pages attended: the newest and the best of the others, ties to the lower page."""
    picked = []
    for row in page_scores(q, K):
        older = sorted(range(len(row) - 1), key=lambda p: (-row[p], p))[:n_blocks - 1]
        picked.append(sorted(older + [len(row) - 1]))
    return picked


def block_tokens(pages, N):
    return [np.concatenate([np.arange(p * PAGE, min(N, (p + 1) * PAGE)) for p in head]) for head in pages]


def add_mass(mass, idx, vals, lse, d, G):
    """mass [Hkv, cap] float64 plus the weights of idx, vals [Hq, k] (idx < 0: nothing), lse [Hq]."""
    out = mass.copy()
    for h in range(idx.shape[0]):
        use = idx[h] >= 0
        np.add.at(out[h // G], idx[h][use], np.exp(vals[h][use].astype(np.float64) / np.sqrt(d) - lse[h]))
    return out


def survivors(mass, N, budget, recent):
    """mass [Hkv, >= N] -> per KV head the ascending positions that stay."""
    if N <= budget:
        return [np.arange(N) for _ in mass]
    kept = []
    for row in mass:
        older = row[:N - recent].astype(np.float64)
        older = np.where(np.isnan(older), -np.inf, older)
        # (a NaN is below -inf too: by the second key)
        order = np.lexsort((np.arange(N - recent), np.isnan(row[:N - recent]), -older))
        kept.append(np.sort(np.concatenate([order[:budget - recent], np.arange(N - recent, N)])).astype(np.int64))
    return kept
