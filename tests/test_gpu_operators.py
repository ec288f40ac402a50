"""Operators beside the top-k decode (appends that normalise and rotate, dense and block-sparse decode, accumulated weights, eviction) on
the GPU, through the binding, against oracle/operators_ref.py in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

import helpers as H
from oracle import operators_ref as ref
from paper_2502_06766_amd import topk_attn as ta
from paper_2502_06766_amd import workloads as wl

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0) if torch.cuda.is_available() else None
U = 2.0 ** -24                                                   # half a step of fp32 relative to the value
HALF = {wl.F32: 2.0 ** -24, wl.F16: 2.0 ** -11, wl.BF16: 2.0 ** -8}
TINY = {wl.F32: 0.0, wl.F16: 2.0 ** -25, wl.BF16: 0.0}           # half a step of the smallest numbers (fp16)


def draw(g, *shape, dtype):
    return wl.quantize(g.standard_normal(shape).astype(np.float32), dtype)


def make(lens, Hq, Hkv, d, cap, dtype, seed=0, index=ta.INDEX_NONE, max_k=64, layers=1, layer=0):
    """A cache whose unused rows are NaN, sequence b of `layer` holding lens[b] Gaussian tokens -> cache, K, V (widened), per sequence."""
    g = np.random.default_rng(seed)
    cache = ta.TopkAttnCache(layers, len(lens), Hq, Hkv, d, cap, max_k, dtype, index_kind=index)
    cache.kv.fill_(255)
    Ks, Vs = [], []
    for b, n in enumerate(lens):
        K, V = draw(g, Hkv, n, d, dtype=dtype), draw(g, Hkv, n, d, dtype=dtype)
        if n:
            cache.append(layer, b, H.to_torch(K, dtype, DEV), H.to_torch(V, dtype, DEV), head_major=True)
        Ks.append(wl.widen(K, dtype))
        Vs.append(wl.widen(V, dtype))
    return cache, Ks, Vs


def rows_of(cache, dtype, B, Hkv, cap, d):
    """Views [B, Hkv, cap, d] of the keys and values of a one-layer cache."""
    size = B * Hkv * cap * d * wl.DTYPE_BYTES[dtype]
    half = (size + 255) // 256 * 256
    return [cache.kv[i * half:i * half + size].view(cache.torch_dtype()).view(B, Hkv, cap, d) for i in range(2)]


def weight_error(q, K, d):
    """Bound of a softmax weight's relative error before normalisation: the score's sum of d products in 32 bits (d u sum |q k|), its
    product with the scale and the difference to the maximum (each u of the largest exponent, twice for the maximum's own), the exponential
    (2 u), and what two parts of a 16-bit weight leave (2^-18)."""
    Hkv = K.shape[0]
    A = max((np.abs(K[h]) @ np.abs(q.reshape(Hkv, -1, d)[h]).T).max() for h in range(Hkv)) / np.sqrt(d)
    return (d + 6) * U * A + 4 * U + 2.0 ** -18


def check(out, lse, mass, mass0, want, q, K, V, d, label=""):
    r_out, r_lse, r_mass = want
    N = K.shape[1]
    dw = weight_error(q, K, d)
    sums = (N / 16 + 64) * U                                    # additions that follow each other: steps of a wave, waves, splits
    tol = 2 * (dw + sums) * np.abs(V).max()
    assert np.abs(out - r_out).max() <= tol, f"{label}: out off by {np.abs(out - r_out).max():.3g}, {tol:.3g} allowed"
    if lse is not None:
        tol = dw + sums + 4 * U * np.abs(r_lse).max()
        assert np.abs(lse - r_lse).max() <= tol, f"{label}: lse off by {np.abs(lse - r_lse).max():.3g}, {tol:.3g} allowed"
    if mass is not None:
        total = mass0[:, :N] + r_mass
        tol = (2 * (dw + sums) + 20 * U * np.abs(r_lse).max() + 130 * U) * r_mass + 2 * U * total + 1e-37
        off = np.abs(mass[:, :N] - total)
        assert (off <= tol).all(), f"{label}: mass off by {off.max():.3g}"
        assert (mass[:, N:] == mass0[:, N:]).all(), f"{label}: mass behind the sequence was touched"


DENSE = [  # dtype, Hq, Hkv, d, lens, cap
    (wl.BF16, 32, 8, 128, [500], 500),
    (wl.F16, 4, 1, 64, [1, 2, 63], 70),
    (wl.BF16, 5, 1, 32, [64, 65, 31, 33], 131),
    (wl.F32, 8, 2, 64, [1, 200, 129], 203),
    (wl.F32, 16, 1, 256, [77, 400], 401),
    (wl.F32, 3, 3, 128, [1000], 1001),
    (wl.F32, 2, 1, 32, [15, 16, 17], 17),
    (wl.F16, 16, 1, 128, [999, 3], 1000),
    (wl.BF16, 17, 1, 256, [130, 700], 700),
    (wl.F16, 80, 2, 64, [300, 129, 5], 301),
    (wl.BF16, 128, 1, 128, [1500], 1601),
    (wl.F16, 7, 7, 256, [4097], 4100),
    (wl.BF16, 64, 8, 128, [8191, 700, 1, 2048, 64], 8193),
    (wl.F16, 4, 1, 128, [70001], 70001),
    (wl.F16, 6, 2, 32, [40007, 39999], 40010),
]


@pytest.mark.parametrize("with_mass", [False, True])
@pytest.mark.parametrize("dtype,Hq,Hkv,d,lens,cap", DENSE)
def test_dense(dtype, Hq, Hkv, d, lens, cap, with_mass):
    cache, Ks, Vs = make(lens, Hq, Hkv, d, cap, dtype, seed=cap)
    try:
        g = np.random.default_rng(cap + 1)
        q = draw(g, len(lens), Hq, d, dtype=dtype)
        mass0 = g.random((len(lens), Hkv, cap)).astype(np.float32)
        mass = torch.from_numpy(mass0).to(DEV) if with_mass else None
        out, lse = cache.decode_dense(0, H.to_torch(q, dtype, DEV), mass=mass)
        for b, n in enumerate(lens):
            qb = wl.widen(q[b], dtype)
            check(out[b].cpu().numpy().astype(np.float64), lse[b].cpu().numpy(), mass[b].cpu().numpy() if with_mass else None, mass0[b],
                  ref.attend(qb, Ks[b], Vs[b]), qb, Ks[b], Vs[b], d, f"sequence {b} ({n} tokens)")
    finally:
        cache.close()


@pytest.mark.parametrize("dtype", [wl.F32, wl.F16, wl.BF16])
def test_dense_of_peaked_and_flat_scores(dtype):
    """One key far above the others, all keys equal, scores rising along the cache (the running maximum changes at every step) and
    falling; values of the largest magnitude the type's sums take."""
    d, n = 64, 1000
    g = np.random.default_rng(5)
    q = np.zeros((1, 4, d), np.float32)
    q[..., 0] = 16.0
    for kind in ("peak", "flat", "rise", "fall"):
        K = np.zeros((1, n, d), np.float32)
        K[0, :, 0] = {"peak": np.where(np.arange(n) == 700, 40.0, 0.0), "flat": np.full(n, 3.0), "rise": np.arange(n) / 8.0,
                      "fall": -np.arange(n) / 8.0}[kind]
        V = draw(g, 1, n, d, dtype=dtype)
        Kq, qq = wl.quantize(K, dtype), wl.quantize(q, dtype)
        cache = ta.TopkAttnCache(1, 1, 4, 1, d, n, 8, dtype)
        try:
            cache.append(0, 0, H.to_torch(Kq, dtype, DEV), H.to_torch(V, dtype, DEV), head_major=True)
            mass = torch.zeros((1, 1, n), device=DEV)
            out, lse = cache.decode_dense(0, H.to_torch(qq, dtype, DEV), mass=mass)
            q64, K64, V64 = wl.widen(qq[0], dtype), wl.widen(Kq, dtype), wl.widen(V, dtype)
            check(out[0].cpu().numpy().astype(np.float64), lse[0].cpu().numpy(), mass[0].cpu().numpy(), np.zeros((1, n), np.float32),
                  ref.attend(q64, K64, V64), q64, K64, V64, d, kind)
        finally:
            cache.close()


def test_dense_with_infinite_and_missing_scores():
    """Keys of -inf score weigh nothing, also where they fill whole steps and splits; a NaN key makes the head NaN; values behind the
    sequence (NaN here) and of keys without weight never show."""
    d, n = 64, 5000
    g = np.random.default_rng(6)
    K, V = draw(g, 1, n, d, dtype=wl.F32), draw(g, 1, n, d, dtype=wl.F32)
    K[0, :4000, 3] = -np.inf
    q = np.abs(draw(g, 1, 2, d, dtype=wl.F32)) + 0.1
    cache = ta.TopkAttnCache(1, 1, 2, 1, d, n + 9, 8, wl.F32)
    try:
        cache.kv.fill_(255)
        cache.append(0, 0, H.to_torch(K, wl.F32, DEV), H.to_torch(V, wl.F32, DEV), head_major=True)
        mass = torch.zeros((1, 1, n + 9), device=DEV)
        out, lse = cache.decode_dense(0, H.to_torch(q, wl.F32, DEV), mass=mass)
        q64 = q[0].astype(np.float64)
        want = ref.attend(q64, K[:, 4000:].astype(np.float64), V[:, 4000:].astype(np.float64))
        check(out[0].cpu().numpy().astype(np.float64), lse[0].cpu().numpy(), mass[0, :, 4000:].cpu().numpy(), np.zeros((1, n), np.float32)[:, :1009],
              want, q64, K[:, 4000:].astype(np.float64), V[:, 4000:].astype(np.float64), d)
        assert (mass[0, :, :4000] == 0).all()
        bad = torch.full((1, 1, d), float("nan"), device=DEV)
        cache.append(0, 0, bad, bad)
        assert torch.isnan(cache.decode_dense(0, H.to_torch(q, wl.F32, DEV))[0]).all()
    finally:
        cache.close()


BLOCKS = [  # dtype, Hq, Hkv, d, lens, cap, n_blocks
    (wl.BF16, 32, 8, 128, [5000], 5000, 7),
    (wl.F16, 4, 1, 64, [1, 64, 65, 700], 900, 3),
    (wl.F32, 8, 2, 32, [333, 1300], 1301, 2),
    (wl.F32, 4, 4, 256, [900, 129], 901, 4),
    (wl.F32, 5, 1, 128, [2000], 2000, 31),
    (wl.BF16, 20, 1, 64, [1999, 70], 2100, 1),
    (wl.F16, 128, 1, 128, [1500], 1501, 9),
    (wl.BF16, 16, 2, 256, [3001, 1], 3001, 20),
    (wl.F16, 6, 2, 32, [70003], 70003, 300),
    (wl.F16, 2, 2, 64, [640, 500], 640, 10),                     # as many as there are
    (wl.F16, 2, 2, 64, [640, 500], 700, 15),                     # more than there are
    (wl.BF16, 4, 1, 32, [150001], 150001, 1500),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,d,lens,cap,n_blocks", BLOCKS)
def test_blocks(dtype, Hq, Hkv, d, lens, cap, n_blocks):
    cache, Ks, Vs = make(lens, Hq, Hkv, d, cap, dtype, seed=cap + n_blocks, index=ta.INDEX_BOXES)
    try:
        g = np.random.default_rng(cap + 1)
        q = draw(g, len(lens), Hq, d, dtype=dtype)
        qt = H.to_torch(q, dtype, DEV)
        mass0 = g.random((len(lens), Hkv, cap)).astype(np.float32)
        mass = torch.from_numpy(mass0).to(DEV)
        out, blocks, lse = cache.decode_blocks(0, qt, n_blocks, mass=mass)
        for b, n in enumerate(lens):
            qb = wl.widen(q[b], dtype)
            pages = ref.pick_blocks(qb, Ks[b], n_blocks)
            got = blocks[b].cpu().numpy()
            for h in range(Hkv):
                assert list(got[h]) == pages[h] + [-1] * (n_blocks - len(pages[h])), f"sequence {b}, KV head {h}"
            at = ref.block_tokens(pages, n)
            check(out[b].cpu().numpy().astype(np.float64), lse[b].cpu().numpy(), mass[b].cpu().numpy(), mass0[b],
                  ref.attend(qb, Ks[b], Vs[b], at), qb, Ks[b], Vs[b], d, f"sequence {b} ({n} tokens)")
        bare = cache.decode_blocks(0, qt, n_blocks, want_blocks=False, want_lse=False)
        assert bare[1] is None and bare[2] is None and torch.equal(bare[0], out)
        # the top-k decode of such a handle is the exact one
        plain, _, _, _ = cache.decode(0, qt, 8)
        assert torch.isfinite(plain).all()
    finally:
        cache.close()


@pytest.mark.parametrize("kind", ["equal", "few_values", "infinite", "wide"])
def test_blocks_with_ties_and_extremes(kind):
    """Pages of equal score go by number, in the histogram and where its bin is crowded (more than 2048 equal pages); infinite scores and
    scores over many magnitudes are ordered too."""
    d, n, n_blocks = 32, 64 * 2600 + 5, 100
    g = np.random.default_rng(7)
    K = np.ones((1, n, d), np.float32)
    if kind == "few_values":
        K *= g.integers(-2, 3, (1, n // 64 + 1, 1)).repeat(64, 1)[:, :n]
    elif kind == "infinite":
        K[0, 64 * 50:64 * 51] = np.inf
        K[0, 64 * 60:64 * 62] = -np.inf
    elif kind == "wide":
        K *= (10.0 ** g.integers(-30, 30, (1, n // 64 + 1, 1))).astype(np.float32).repeat(64, 1)[:, :n]
    q = np.ones((1, 2, d), np.float32)
    cache = ta.TopkAttnCache(1, 1, 2, 1, d, n, 8, wl.F32, index_kind=ta.INDEX_BOXES)
    try:
        Kt = H.to_torch(K, wl.F32, DEV)
        cache.append(0, 0, Kt, torch.ones_like(Kt), head_major=True)
        _, blocks, _ = cache.decode_blocks(0, H.to_torch(q, wl.F32, DEV), n_blocks)
        assert list(blocks[0, 0].cpu().numpy()) == ref.pick_blocks(q[0].astype(np.float64), K.astype(np.float64), n_blocks)[0]
    finally:
        cache.close()


def boxes_of(cache, dtype, L, B, Hkv, cap, d):
    size = L * B * Hkv * cap * d * wl.DTYPE_BYTES[dtype]
    at, pages = 2 * ((size + 255) // 256 * 256), (cap + 63) // 64
    return cache.kv[at:at + L * B * Hkv * pages * 2 * d * wl.DTYPE_BYTES[dtype]].view(cache.torch_dtype()).view(L, B, Hkv, pages, 2, d)


@pytest.mark.parametrize("dtype,d", [(wl.F32, 256), (wl.F16, 32), (wl.BF16, 128), (wl.F16, 64)])
def test_boxes_follow_every_append(dtype, d):
    """Bulk imports, batched steps and rotary appends, in pieces that begin and end inside pages, of the second layer."""
    B, Hkv, cap = 2, 3, 300
    g = np.random.default_rng(8)
    cache = ta.TopkAttnCache(2, B, 6, Hkv, d, cap, 8, dtype, index_kind=ta.INDEX_BOXES)
    try:
        for n, how in ((63, "kv"), (1, "step"), (1, "step"), (70, "step"), (1, "rotary"), (65, "rotary"), (5, "kv")):
            k, v = (H.to_torch(draw(g, B, n, Hkv, d, dtype=dtype), dtype, DEV) for _ in range(2))
            if how == "kv":
                for b in range(B):
                    cache.append(1, b, k[b].contiguous(), v[b].contiguous())
            elif how == "step":
                cache.append_step(1, k, v)
            else:
                cache.append_rotary(1, None, k, v, torch.ones(d // 2, device=DEV))
        n = cache.length(1, 0)
        size = 2 * B * Hkv * cap * d * wl.DTYPE_BYTES[dtype]
        K = cache.kv[:size].view(cache.torch_dtype()).view(2, B, Hkv, cap, d)[1, :, :, :n].float()
        boxes = boxes_of(cache, dtype, 2, B, Hkv, cap, d)[1].float()
        for p in range((n + 63) // 64):
            rows = K[:, :, 64 * p:64 * p + 64]
            assert torch.equal(boxes[:, :, p, 0], rows.amin(2)) and torch.equal(boxes[:, :, p, 1], rows.amax(2)), p
    finally:
        cache.close()


ROTARY = [  # dtype, Hq, Hkv, d, B, n, rotary, interleaved, norm, base
    (wl.BF16, 32, 8, 128, 16, 1, 128, False, True, 200000),
    (wl.F16, 32, 8, 128, 1, 33, 64, False, True, 0),
    (wl.F32, 4, 2, 64, 3, 5, 64, True, True, 16777217),
    (wl.F32, 2, 1, 256, 2, 7, 254, False, False, 2000000000),
    (wl.F32, 5, 5, 32, 1, 1, 32, False, True, 3),
    (wl.BF16, 7, 1, 256, 2, 3, 256, True, False, 99),
    (wl.F16, 6, 3, 32, 2, 9, 6, False, True, 1000003),
    (wl.BF16, 3, 1, 64, 4, 2, 0, False, True, 0),
    (wl.F16, 128, 1, 64, 1, 4, 2, True, True, 17),
]


def rotary_case(g, dtype, Hq, Hkv, d, B, n, rotary, norm, base, tiny_row=False):
    qkv = draw(g, B, n, Hq + 2 * Hkv, d, dtype=dtype)
    if tiny_row:
        qkv[:, :, Hq] = 0
    w = [draw(g, d, dtype=dtype) if norm else None for _ in range(2)]
    freq = (10000.0 ** (-np.arange(rotary // 2) / max(1, rotary // 2))).astype(np.float32)
    pos = (base + g.integers(0, 50, (B, n))).astype(np.int32)
    return qkv, w, freq, pos


@pytest.mark.parametrize("dtype,Hq,Hkv,d,B,n,rotary,interleaved,norm,base", ROTARY)
def test_rotary(dtype, Hq, Hkv, d, B, n, rotary, interleaved, norm, base):
    g = np.random.default_rng(n * 7 + d)
    qkv, (wq, wk), freq, pos = rotary_case(g, dtype, Hq, Hkv, d, B, n, rotary, norm, base)
    t = H.to_torch(qkv, dtype, DEV)
    cap = 3 * n + 2
    cache = ta.TopkAttnCache(1, B, Hq, Hkv, d, cap, 8, dtype)
    cache.kv.fill_(255)
    try:
        wt = [None if w is None else H.to_torch(w, dtype, DEV) for w in (wq, wk)]
        first = H.to_torch(draw(g, 1, Hkv, d, dtype=dtype), dtype, DEV)
        cache.append(0, B - 1, first, first)                    # (the last sequence is one token ahead)
        args = dict(positions=torch.from_numpy(pos).to(DEV), q_norm=wt[0], k_norm=wt[1], eps=1e-5, interleaved=interleaved)
        q_out = cache.append_rotary(0, t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:], torch.from_numpy(freq).to(DEV), **args)
        assert q_out.shape == (B, n, Hq, d) and q_out.is_contiguous()
        lens = [n + (b == B - 1) for b in range(B)]
        assert [cache.length(0, b) for b in range(B)] == lens
        dev_len = cache.ws[:4 * B].view(torch.int32)
        assert dev_len.tolist() == lens
        K, V = rows_of(cache, dtype, B, Hkv, cap, d)
        x = wl.widen(qkv, dtype)
        for b in range(B):
            want_q = ref.rms_rotate(x[b, :, :Hq], None if wq is None else wl.widen(wq, dtype), np.float32(1e-5), pos[b], freq, interleaved)
            want_k = ref.rms_rotate(x[b, :, Hq:Hq + Hkv], None if wk is None else wl.widen(wk, dtype), np.float32(1e-5), pos[b], freq, interleaved)
            got_k = K[b, :, lens[b] - n:lens[b]].transpose(0, 1).double().cpu().numpy()
            for got, want in ((q_out[b].double().cpu().numpy(), want_q), (got_k, want_k)):
                # of the pair's length r: the norm's sum of d squares, root, quotient and two products ((d / 2 + 6) u), the fraction of a turn
                # in 32 bits and the two functions (2 pi u / 2 + 4 u), the product and sum (3 u); then the rounding of the value itself
                r = np.sqrt(want ** 2 + np.abs(want).max(-1, keepdims=True) ** 2)
                tol = (d / 2 + 20) * U * r + HALF[dtype] * np.abs(want) * 1.01 + TINY[dtype]
                assert (np.abs(got - want) <= tol).all(), f"sequence {b}: off by {np.abs(got - want).max():.3g}"
            assert torch.equal(V[b, :, lens[b] - n:lens[b]].transpose(0, 1), t[b, :, Hq + Hkv:])
            assert torch.isnan(K[b, :, lens[b]:].float()).all() and torch.isnan(V[b, :, lens[b]:].float()).all()
        # one sequence by itself, keys and values only, at the cache's own rows
        cache.append_rotary(0, None, t[:1, :, Hq:Hq + Hkv], t[:1, :, Hq + Hkv:], torch.from_numpy(freq).to(DEV), k_norm=wt[1], eps=1e-5,
                            interleaved=interleaved, seq=0)
        assert cache.length(0, 0) == lens[0] + n and dev_len.tolist()[0] == lens[0] + n
        at = np.arange(lens[0], lens[0] + n)
        want = ref.rms_rotate(x[0, :, Hq:Hq + Hkv], None if wk is None else wl.widen(wk, dtype), np.float32(1e-5), at, freq, interleaved)
        got = K[0, :, lens[0]:lens[0] + n].transpose(0, 1).double().cpu().numpy()
        tol = (d / 2 + 20) * U * np.abs(want).max(-1, keepdims=True) * 1.5 + HALF[dtype] * np.abs(want) * 1.01 + TINY[dtype]
        assert (np.abs(got - want) <= tol).all()
    finally:
        cache.close()


@pytest.mark.parametrize("index", [ta.INDEX_INT8, ta.INDEX_PAGES])
@pytest.mark.parametrize("dtype,d,n", [(wl.BF16, 128, 1), (wl.F16, 64, 70), (wl.F16, 256, 3), (wl.BF16, 64, 1)])
def test_rotary_keeps_the_index(index, dtype, d, n):
    """The index entries are those that an append of the rotated keys leaves, byte for byte; a row of zeros among them."""
    B, Hq, Hkv, cap = 2, 4, 2, 3 * n + 20
    g = np.random.default_rng(9)
    a, b = (ta.TopkAttnCache(1, B, Hq, Hkv, d, cap, 8, dtype, index_kind=index) for _ in range(2))
    try:
        for c in (a, b):
            c.kv.fill_(0)
        for step in range(3):
            qkv, (wq, wk), freq, pos = rotary_case(g, dtype, Hq, Hkv, d, B, n, d // 2, True, 70, tiny_row=step == 1)
            t = H.to_torch(qkv, dtype, DEV)
            a.append_rotary(0, t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:], torch.from_numpy(freq).to(DEV),
                            positions=torch.from_numpy(pos).to(DEV), k_norm=H.to_torch(wk, dtype, DEV))
            K, V = rows_of(a, dtype, B, Hkv, cap, d)
            at = a.length(0, 0)
            b.append_step(0, *(x[:, :, at - n:at].transpose(1, 2).contiguous() for x in (K, V)))
            assert torch.equal(a.kv, b.kv)
    finally:
        a.close()
        b.close()


EVICT = [  # dtype, Hkv, d, lens, cap, budget, recent, index
    (wl.BF16, 2, 128, [1000, 200, 300], 1001, 300, 50, ta.INDEX_NONE),
    (wl.F16, 1, 64, [100], 100, 99, 0, ta.INDEX_NONE),
    (wl.F32, 3, 32, [777], 800, 1, 0, ta.INDEX_NONE),
    (wl.F32, 1, 256, [777, 1], 800, 1, 1, ta.INDEX_NONE),
    (wl.F16, 2, 128, [5000], 5000, 4999, 0, ta.INDEX_NONE),       # all but one row move by one
    (wl.F16, 2, 128, [5000], 5000, 4999, 4999, ta.INDEX_NONE),    # the oldest goes
    (wl.BF16, 1, 32, [20001, 9000], 20001, 12345, 100, ta.INDEX_NONE),
    (wl.F16, 2, 128, [3000, 100], 3001, 1000, 10, ta.INDEX_INT8),
    (wl.BF16, 2, 64, [4444, 2222], 4500, 2222, 0, ta.INDEX_INT8),
    (wl.F16, 2, 256, [700, 100, 650], 701, 130, 30, ta.INDEX_PAGES),
    (wl.BF16, 1, 128, [3000, 64], 3001, 1000, 1000, ta.INDEX_BOXES),
    (wl.F32, 2, 64, [900], 900, 64, 3, ta.INDEX_BOXES),
    (wl.F16, 4, 128, [60000, 59000], 60000, 30000, 500, ta.INDEX_NONE),
    (wl.F16, 2, 32, [200001, 16500, 30, 49999], 200001, 16000, 100, ta.INDEX_NONE),      # chunks of more tokens than registers
    (wl.BF16, 1, 64, [16385, 32769, 16384], 32770, 16383, 0, ta.INDEX_INT8),
    (wl.F32, 1, 32, [131073, 131072], 131073, 131072, 1, ta.INDEX_NONE),
]


def masses(g, lens, Hkv, cap):
    """Light and heavy tokens, many of exactly equal weight, many of none."""
    m = np.exp(3 * g.standard_normal((len(lens), Hkv, cap))).astype(np.float32)
    m = np.where(g.random(m.shape) < 0.3, 0.0, np.where(g.random(m.shape) < 0.3, 0.25, m)).astype(np.float32)
    return m


@pytest.mark.parametrize("dtype,Hkv,d,lens,cap,budget,recent,index", EVICT)
def test_evict(dtype, Hkv, d, lens, cap, budget, recent, index):
    B = len(lens)
    cache, _, _ = make(lens, 2 * Hkv, Hkv, d, cap, dtype, seed=cap, index=index)
    other = None
    try:
        g = np.random.default_rng(cap + 2)
        mass0 = masses(g, lens, Hkv, cap)
        mass = torch.from_numpy(mass0).to(DEV)
        K0, V0 = (x.clone() for x in rows_of(cache, dtype, B, Hkv, cap, d))
        kept = cache.evict(0, mass, budget, recent)
        K, V = rows_of(cache, dtype, B, Hkv, cap, d)
        now = [min(n, budget) for n in lens]
        assert [cache.length(0, b) for b in range(B)] == now and cache.ws[:4 * B].view(torch.int32).tolist() == now
        bits = lambda x: x.view(torch.int32 if dtype == wl.F32 else torch.int16)
        for b, n in enumerate(lens):
            m = now[b]
            want = ref.survivors(mass0[b], n, budget, recent)
            for h in range(Hkv):
                at = torch.from_numpy(want[h]).to(DEV)
                assert torch.equal(kept[b, h, :m].long(), at) and (kept[b, h, m:] == -1).all(), (b, h)
                assert torch.equal(bits(K[b, h, :m]), bits(K0[b, h, at])) and torch.equal(bits(V[b, h, :m]), bits(V0[b, h, at])), (b, h)
                assert torch.equal(mass[b, h, :m].cpu(), torch.from_numpy(mass0[b, h, want[h]])), (b, h)
                assert (mass[b, h, m:n] == 0).all() and np.array_equal(mass[b, h, n:].cpu().numpy(), mass0[b, h, n:]), (b, h)
        if index != ta.INDEX_NONE:
            # what a fresh import of the survivors has
            other = ta.TopkAttnCache(1, B, 2 * Hkv, Hkv, d, cap, 64, dtype, index_kind=index)
            other.kv.copy_(cache.kv)
            at = 2 * ((B * Hkv * cap * d * wl.DTYPE_BYTES[dtype] + 255) // 256 * 256)
            if index == ta.INDEX_INT8:                            # (codes and scales of the rows there are)
                rows = torch.zeros((B, Hkv, cap), dtype=torch.bool, device=DEV)
                for b in range(B):
                    rows[b, :, :now[b]] = True
                split = (rows.numel() * d + 255) // 256 * 256
                parts = lambda c: (c.kv[at:at + rows.numel() * d].view(B, Hkv, cap, d)[rows], c.kv[at + split:at + split + 4 * rows.numel()].view(torch.int32).view(B, Hkv, cap)[rows])
            else:
                P, row = (cap + 63) // 64, d * wl.DTYPE_BYTES[dtype] * (2 if index == ta.INDEX_BOXES else 1)
                live = torch.zeros((B, Hkv, P), dtype=torch.bool, device=DEV)
                for b in range(B):
                    live[b, :, :(now[b] + 63) // 64] = True
                second = (live.numel() * row + 255) // 256 * 256
                parts = lambda c: (c.kv[at:at + live.numel() * row].view(B, Hkv, P, row)[live],) + (
                    (c.kv[at + second:at + second + 8 * live.numel()].view(B, Hkv, P, 8)[live],) if index == ta.INDEX_PAGES else ())
            kept_parts = [x.clone() for x in parts(cache)]
            for b in range(B):
                other.append(0, b, K[b, :, :now[b]].contiguous(), V[b, :, :now[b]].contiguous(), head_major=True)
            for x, y in zip(kept_parts, parts(other)):
                assert torch.equal(x, y)
        # nothing more to evict: nothing changes
        before = cache.kv.clone()
        again = cache.evict(0, mass, budget, 0)
        assert torch.equal(cache.kv, before) and all((again[b, :, :now[b]].cpu() == torch.arange(now[b])).all() for b in range(B))
    finally:
        cache.close()
        if other is not None:
            other.close()


@pytest.mark.parametrize("n,budget", [(3000, 1500), (16500, 400), (40000, 39990), (140000, 70000)])
@pytest.mark.parametrize("value", [0.0, 1.5])
def test_evict_among_equals_keeps_the_oldest(n, budget, value):
    """All weights equal but a few above and a few below, at the ends of waves and chunks."""
    cache, _, _ = make([n], 1, 1, 32, n, wl.F16, seed=n)
    try:
        mass0 = np.full((1, 1, n), value, np.float32)
        mass0[0, 0, [63, 64, n // 2, n - 1]] = 9.0
        mass0[0, 0, [0, 65, n // 3]] = -1.0
        kept = cache.evict(0, torch.from_numpy(mass0).to(DEV), budget, 7)
        assert np.array_equal(kept[0, 0].cpu().numpy(), ref.survivors(mass0[0], n, budget, 7)[0])
    finally:
        cache.close()


def test_evict_orders_unusual_weights():
    """Negative weights, both zeros, infinities and NaN: NaN goes first, then -inf; equal weights by position; without `kept`."""
    n, budget = 12, 5
    row = np.array([np.nan, -1.0, 0.0, -0.0, np.inf, -np.inf, 3.0, np.nan, 1e-40, 0.0, 3.0, -1e-40], np.float32)
    for recent in range(6):
        cache, _, _ = make([n], 1, 1, 32, n, wl.F32, seed=3)
        try:
            K0 = rows_of(cache, wl.F32, 1, 1, n, 32)[0].clone()
            mass = torch.from_numpy(row.copy()).to(DEV).view(1, 1, n)
            assert cache.evict(0, mass, budget, recent, want_kept=False) is None
            order = [4, 6, 10, 8, 2, 3, 9, 11, 1, 5, 0, 7]          # from the heaviest
            older = [p for p in order if p < n - recent][:budget - recent]
            want = sorted(older + list(range(n - recent, n)))
            assert torch.equal(rows_of(cache, wl.F32, 1, 1, n, 32)[0][0, 0, :budget], K0[0, 0, want])
        finally:
            cache.close()


@pytest.mark.parametrize("Hq,Hkv,k,lens,cap", [(32, 8, 64, [500], 500), (5, 1, 2000, [3000, 7], 3001), (6, 3, 1, [1, 40], 41), (64, 2, 4097, [5000], 6000)])
def test_add_mass(Hq, Hkv, k, lens, cap):
    d, B, G = 64, len(lens), Hq // Hkv
    g = np.random.default_rng(k)
    idx = np.full((B, Hq, k), -1, np.int32)
    vals = np.full((B, Hq, k), -np.inf, np.float32)
    lse = np.zeros((B, Hq), np.float32)
    for b, n in enumerate(lens):
        m = min(n, k)
        for h in range(Hq):
            idx[b, h, :m] = g.permutation(n)[:m]
            vals[b, h, :m] = 8 * g.standard_normal(m)
            lse[b, h] = np.log(np.exp(vals[b, h, :m].astype(np.float64) / 8).sum())
    idx[0, 0, 0] = cap + 5                                       # (not a position of the cache: passed over)
    mass0 = g.random((B, Hkv, cap)).astype(np.float32)
    cache = ta.TopkAttnCache(1, B, Hq, Hkv, d, cap, 8, wl.F16)
    try:
        mass = torch.from_numpy(mass0).to(DEV)
        args = [torch.from_numpy(x).to(DEV) for x in (idx, vals, lse)]
        cache.add_mass(0, *args, mass)
        again = torch.from_numpy(mass0).to(DEV)
        cache.add_mass(0, *args, again)
        assert torch.equal(mass, again)
        idx[0, 0, 0] = -1
        for b in range(B):
            want = ref.add_mass(mass0[b].astype(np.float64), idx[b], vals[b], lse[b].astype(np.float64), d, G)
            # a weight: the exponent's product, difference and the product with log2 e (3 u of at most 2^6), the exponential (2 u); G additions
            tol = (3 * 64 + 2 + G + 1) * U * want
            assert (np.abs(mass[b].cpu().numpy() - want) <= tol).all()
    finally:
        cache.close()


def test_mass_of_a_top_k_decode_is_its_weights():
    """add_mass of a top-k decode over all keys and the dense decode's mass are the same weights."""
    cache, Ks, _ = make([700, 300], 8, 2, 64, 701, wl.F16, seed=4, max_k=701)
    try:
        q = H.to_torch(draw(np.random.default_rng(5), 2, 8, 64, dtype=wl.F16), wl.F16, DEV)
        a, b = (torch.zeros((2, 2, 701), device=DEV) for _ in range(2))
        _, idx, vals, lse = cache.decode(0, q, 701)
        cache.add_mass(0, idx, vals, lse, a)
        cache.decode_dense(0, q, mass=b)
        assert torch.allclose(a, b, rtol=1e-4, atol=0.0) and abs(a.sum().item() - 16) < 1e-3
    finally:
        cache.close()


@pytest.mark.parametrize("dtype", [wl.F16, wl.F32])
def test_a_bounded_cache_over_many_steps(dtype):
    """The operators together, as a program with a bounded cache has them: a prompt and then single tokens appended with norms and
    rotation, dense and block-sparse steps that leave their weights, eviction whenever the cache is full, top-k decode in between; each
    step against 64 bits over the rows that are there."""
    B, Hq, Hkv, d, cap, budget, recent = 2, 8, 2, 64, 320, 200, 24
    g = np.random.default_rng(10)
    cache = ta.TopkAttnCache(1, B, Hq, Hkv, d, cap, 40, dtype, index_kind=ta.INDEX_BOXES)
    cache.kv.fill_(255)
    mass = torch.zeros((B, Hkv, cap), device=DEV)
    K, V = rows_of(cache, dtype, B, Hkv, cap, d)
    evictions, position = 0, 0
    try:
        for step in range(12):
            n = 250 if step == 0 else 30 if step % 3 else 1
            if cache.length(0, 0) + n > cap:
                before, m0, N = (K.clone(), V.clone()), mass.cpu().numpy(), cache.length(0, 0)
                kept = cache.evict(0, mass, budget, recent)
                evictions += 1
                for b in range(B):
                    for h, at in enumerate(ref.survivors(m0[b], N, budget, recent)):
                        assert np.array_equal(kept[b, h].cpu().numpy(), at)
                        assert torch.equal(K[b, h, :budget], before[0][b, h, at]) and torch.equal(V[b, h, :budget], before[1][b, h, at])
            qkv, (wq, wk), freq, _ = rotary_case(g, dtype, Hq, Hkv, d, B, n, d, True, 0)
            t = H.to_torch(qkv, dtype, DEV)
            pos = torch.arange(position, position + n, dtype=torch.int32, device=DEV).expand(B, n).contiguous()
            q = cache.append_rotary(0, t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:], torch.from_numpy(freq).to(DEV), positions=pos,
                                    q_norm=H.to_torch(wq, dtype, DEV), k_norm=H.to_torch(wk, dtype, DEV))[:, -1].contiguous()
            position += n
            N, m0 = cache.length(0, 0), mass.cpu().numpy()
            if step % 2:
                out, blocks, lse = cache.decode_blocks(0, q, 3, mass=mass)
            else:
                out, lse = cache.decode_dense(0, q, mass=mass)
            for b in range(B):
                q64, K64, V64 = (x.double().cpu().numpy() for x in (q[b], K[b, :, :N], V[b, :, :N]))
                at = None
                if step % 2:
                    pages = ref.pick_blocks(q64, K64, 3)
                    assert [list(x) for x in blocks[b].cpu().numpy()] == pages
                    at = ref.block_tokens(pages, N)
                check(out[b].cpu().numpy().astype(np.float64), lse[b].cpu().numpy(), mass[b].cpu().numpy(), m0[b],
                      ref.attend(q64, K64, V64, at), q64, K64, V64, d, f"step {step}")
            o, idx, vals, l2 = cache.decode(0, q, 40)
            cache.add_mass(0, idx, vals, l2, mass)
            assert torch.isfinite(o).all() and (idx < N).all() and torch.isfinite(mass).all()
        assert evictions >= 2
    finally:
        cache.close()


def test_captured_steps_replay():
    """Dense, block-sparse and accumulated steps in a HIP graph: every replay, with eager calls between, is what the eager call gives."""
    cache, _, _ = make([3000, 900], 8, 2, 64, 3001, wl.BF16, seed=11, index=ta.INDEX_BOXES, max_k=32)
    try:
        g = np.random.default_rng(12)
        q = H.to_torch(draw(g, 2, 8, 64, dtype=wl.BF16), wl.BF16, DEV)
        mass = torch.zeros((2, 2, 3001), device=DEV)

        def step():
            o1, l1 = cache.decode_dense(0, q, mass=mass)
            o2, bl, l2 = cache.decode_blocks(0, q, 6, mass=mass)
            o3, idx, vals, l3 = cache.decode(0, q, 32)
            cache.add_mass(0, idx, vals, l3, mass)
            return o1, l1, o2, bl, l2, o3
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for i in range(4):
            q.copy_(H.to_torch(draw(g, 2, 8, 64, dtype=wl.BF16), wl.BF16, DEV))
            mass.fill_(0.5)
            want = [x.clone() for x in step()]
            mass_want = mass.clone()
            mass.fill_(0.5)
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip(got, want):
                assert torch.equal(x, y), i
            assert torch.equal(mass, mass_want), i
    finally:
        cache.close()


def test_on_a_stream_of_the_callers():
    cache, Ks, Vs = make([2000], 4, 1, 128, 2001, wl.F16, seed=13)
    try:
        q = H.to_torch(draw(np.random.default_rng(1), 1, 4, 128, dtype=wl.F16), wl.F16, DEV)
        want = cache.decode_dense(0, q)[0]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            mass = torch.ones((1, 1, 2001), device=DEV)
            out, _ = cache.decode_dense(0, q, mass=mass)
            kept = cache.evict(0, mass, 500, 100)
        side.synchronize()
        assert torch.equal(out, want) and kept[0, 0, -1] == 1999 and cache.length(0, 0) == 500
    finally:
        cache.close()


def test_refusals():
    """Every refusal leaves the handle and the outputs as they were."""
    L = ta.lib()
    cache, _, _ = make([100, 0], 4, 2, 64, 128, wl.F16, seed=14, max_k=16)
    boxes, _, _ = make([100, 100], 4, 2, 64, 128, wl.F16, seed=14, index=ta.INDEX_BOXES)
    try:
        q = torch.zeros((2, 4, 64), dtype=torch.float16, device=DEV)
        out = torch.full((2, 4, 64), 5.0, device=DEV)
        mass = torch.full((2, 2, 128), 7.0, device=DEV)
        idx = torch.zeros((2, 4, 16), dtype=torch.int32, device=DEV)
        vals, lse = torch.zeros((2, 4, 16), device=DEV), torch.zeros((2, 4), device=DEV)
        p = lambda x: x.data_ptr()
        kv0 = cache.kv.clone()
        assert L.topk_attn_decode_dense(cache.h, 0, p(q), p(out), None, None, None) == ta.EINVAL          # an empty sequence
        assert L.topk_attn_decode_dense(boxes.h, 1, p(q), p(out), None, None, None) == ta.EINVAL
        assert L.topk_attn_decode_dense(boxes.h, 0, p(q) + 2, p(out), None, None, None) == ta.EINVAL
        assert L.topk_attn_decode_dense(boxes.h, 0, None, p(out), None, None, None) == ta.EINVAL
        assert L.topk_attn_decode_blocks(cache.h, 0, p(q), 2, p(out), None, None, None, None) == ta.EINVAL  # no block index
        for n in (0, -1):
            assert L.topk_attn_decode_blocks(boxes.h, 0, p(q), n, p(out), None, None, None, None) == ta.EINVAL
        assert L.topk_attn_set_path(boxes.h, ta.PATH_PAGES) == ta.EINVAL and L.topk_attn_set_path(boxes.h, ta.PATH_INDEX) == ta.EINVAL
        assert L.topk_attn_add_mass(cache.h, 0, p(idx), p(vals), p(lse), 0, p(mass), None) == ta.EINVAL
        assert L.topk_attn_add_mass(cache.h, 0, p(idx), p(vals), None, 16, p(mass), None) == ta.EINVAL
        for budget, recent in ((0, 0), (129, 0), (50, 51), (50, -1)):
            assert L.topk_attn_evict(cache.h, 0, p(mass), budget, recent, None, None) == ta.EINVAL
        assert L.topk_attn_evict(cache.h, 0, None, 50, 0, None, None) == ta.EINVAL
        k = torch.zeros((2, 1, 2, 64), dtype=torch.float16, device=DEV)
        freq = torch.ones(32, device=DEV)
        good = dict(struct_size=ctypes.sizeof(ta.Rotary), rotary_dim=64, interleaved=0, norm_eps=0.0, n_new=1, q=None, k=p(k), v=p(k),
                    k_seq_stride=128, k_token_stride=128, v_seq_stride=128, v_token_stride=128, inv_freq=p(freq))
        for bad, code in ((dict(struct_size=8), ta.EINVAL), (dict(rotary_dim=63), ta.EINVAL), (dict(rotary_dim=66), ta.EINVAL),
                          (dict(rotary_dim=-2), ta.EINVAL), (dict(n_new=-1), ta.EINVAL), (dict(n_new=29), ta.ECAPACITY),
                          (dict(q=p(q)), ta.EINVAL), (dict(q_out=p(q)), ta.EINVAL), (dict(inv_freq=None), ta.EINVAL),
                          (dict(k=None), ta.EINVAL), (dict(k=p(k) + 8), ta.EINVAL), (dict(v_seq_stride=130), ta.EINVAL),
                          (dict(v_token_stride=-128), ta.EINVAL), (dict(norm_eps=-1.0), ta.EINVAL), (dict(norm_eps=float("nan")), ta.EINVAL),
                          (dict(k_norm=p(k) + 2), ta.EINVAL), (dict(n_new=1 << 62), ta.ECAPACITY), (dict(n_new=0), ta.OK)):
            r = ta.Rotary(**{**good, **bad})
            assert L.topk_attn_append_rotary(cache.h, 0, -1, ctypes.byref(r), None) == code, bad
        for seq in (-2, 2):
            assert L.topk_attn_append_rotary(cache.h, 0, seq, ctypes.byref(ta.Rotary(**good)), None) == ta.EINVAL
        torch.cuda.synchronize()
        assert (out == 5.0).all() and (mass == 7.0).all() and torch.equal(cache.kv, kv0)
        assert [cache.length(0, b) for b in range(2)] == [100, 0]
        # a budget that all sequences are within, one of them empty
        kept = cache.evict(0, mass, 100, 10)
        assert (kept[0] == torch.arange(100, device=DEV)).all() and (kept[1] == -1).all() and (mass == 7.0).all()
        # and an eviction beside an empty sequence
        kept = cache.evict(0, mass, 10, 10)
        assert (kept[0] == torch.arange(90, 100, device=DEV)).all() and (kept[1] == -1).all() and cache.length(0, 1) == 0
    finally:
        cache.close()
        boxes.close()


def test_the_top_k_decode_is_unchanged_between_the_operators():
    """The calls share the handle's scratch with the filtered top-k decode: its results before, between and after them are the same bits."""
    cache, _, _ = make([70000, 50001], 8, 2, 128, 70000, wl.F16, seed=21, index=ta.INDEX_BOXES, max_k=500)
    try:
        q = H.to_torch(draw(np.random.default_rng(22), 2, 8, 128, dtype=wl.F16), wl.F16, DEV)
        mass = torch.zeros((2, 2, 70000), device=DEV)
        first = cache.decode(0, q, 500)
        order = torch.sort(first[1], dim=2)
        dense, _ = cache.decode_dense(0, q)
        blocks = cache.decode_blocks(0, q, 40)
        for step in (lambda: cache.decode_dense(0, q, mass=mass), lambda: cache.decode_blocks(0, q, 40, mass=mass),
                     lambda: cache.add_mass(0, first[1], first[2], first[3], mass), lambda: cache.evict(0, mass, 70000, 5)):
            step()
            again = cache.decode(0, q, 500)
            assert torch.equal(again[0], first[0]) and torch.equal(again[3], first[3])
            assert torch.equal(torch.sort(again[1], dim=2).values, order.values)
            assert torch.equal(cache.decode_dense(0, q)[0], dense)
            got = cache.decode_blocks(0, q, 40)
            assert torch.equal(got[0], blocks[0]) and torch.equal(got[1], blocks[1]) and torch.equal(got[2], blocks[2])
    finally:
        cache.close()


def test_two_handles_on_two_streams():
    caches, qs, want, got, streams = [], [], [], [], []
    try:
        for i in range(2):
            cache, _, _ = make([30000 + i], 8, 2, 64, 30001, wl.BF16, seed=30 + i, index=ta.INDEX_BOXES)
            caches.append(cache)
            qs.append(H.to_torch(draw(np.random.default_rng(40 + i), 1, 8, 64, dtype=wl.BF16), wl.BF16, DEV))
            want.append((cache.decode_dense(0, qs[i])[0], cache.decode_blocks(0, qs[i], 30)[0]))
            streams.append(torch.cuda.Stream())
        torch.cuda.synchronize()
        for _ in range(10):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    got.append((i, caches[i].decode_dense(0, qs[i])[0], caches[i].decode_blocks(0, qs[i], 30)[0]))
        torch.cuda.synchronize()
        for i, a, b in got:
            assert torch.equal(a, want[i][0]) and torch.equal(b, want[i][1])
    finally:
        for cache in caches:
            cache.close()


def test_many_short_sequences_and_many_layers():
    """Hundreds of sequences of one to a few tokens, on the last layer of several; the other layers stay as they are."""
    B, Hq, Hkv, d, cap = 300, 4, 2, 64, 9
    g = np.random.default_rng(50)
    cache = ta.TopkAttnCache(3, B, Hq, Hkv, d, cap, 8, wl.F16, index_kind=ta.INDEX_BOXES)
    try:
        k, v = (H.to_torch(draw(g, B, 7, Hkv, d, dtype=wl.F16), wl.F16, DEV) for _ in range(2))
        for b in range(B):
            cache.append(2, b, k[b, :1 + b % 7].contiguous(), v[b, :1 + b % 7].contiguous())
        q = draw(g, B, Hq, d, dtype=wl.F16)
        qt = H.to_torch(q, wl.F16, DEV)
        mass = torch.zeros((B, Hkv, cap), device=DEV)
        out, lse = cache.decode_dense(2, qt, mass=mass)
        out2, blocks, _ = cache.decode_blocks(2, qt, 1)
        assert torch.equal(out, out2) and (blocks == 0).all()
        for b in range(0, B, 37):
            K, V = (x[b, :1 + b % 7].transpose(0, 1).double().cpu().numpy() for x in (k, v))
            qb = wl.widen(q[b], wl.F16)
            check(out[b].cpu().numpy().astype(np.float64), lse[b].cpu().numpy(), mass[b].cpu().numpy(), np.zeros((Hkv, cap), np.float32),
                  ref.attend(qb, K, V), qb, K, V, d)
        kept = cache.evict(2, mass, 3, 1)
        assert [cache.length(2, b) for b in range(B)] == [min(3, 1 + b % 7) for b in range(B)]
        for b in range(0, B, 41):
            n = 1 + b % 7
            assert (kept[b, :, min(n, 3):] == -1).all() and (kept[b, :, min(n, 3) - 1] == n - 1).all()
        assert all(cache.length(layer, b) == 0 for layer in (0, 1) for b in range(0, B, 50))
        with pytest.raises(ta.TopkAttnError):
            cache.decode_dense(1, qt)
    finally:
        cache.close()
