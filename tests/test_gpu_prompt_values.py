"""Attention of a prompt's tokens, value by value: every output within what the roundings of its own weights and sums allow, over values that tell which tile of 64
keys they come from (each channel holds those of few tiles), against 64 bits on the GPU.  Keys walked whole and split, from one tile to a thousand."""
import math

import pytest
import torch

from oracle import coded_cache_ref as ref
from paper_2502_06766_amd import topk_attn as ta

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0) if torch.cuda.is_available() else None
U = 2.0 ** -24                                                   # half a step of fp32 relative to the value
HALF = {ta.F32: 2.0 ** -24, ta.F16: 2.0 ** -11, ta.BF16: 2.0 ** -8}
TORCH = {ta.F32: torch.float32, ta.F16: torch.float16, ta.BF16: torch.bfloat16}


def rows_of(Hkv, n, d, dtype, seed):
    """K, V [Hkv, n, d]: Gaussian keys; a value is other than zero in the channels that equal its tile's number modulo d and modulo d plus a half."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    K = torch.randn((Hkv, n, d), generator=g, device=DEV)
    V = 0.5 + torch.rand((Hkv, n, d), generator=g, device=DEV)
    tile, c = torch.arange(n, device=DEV)[:, None] // 64, torch.arange(d, device=DEV)
    V *= ((tile - c) % d == 0) | ((tile + d // 2 - c) % d == 0)
    return K.to(TORCH[dtype]), V.to(TORCH[dtype])


def held(x, fmt):
    return torch.stack([torch.from_numpy(ref.held(h.double().cpu().numpy(), fmt)).to(DEV) for h in x])


def chains(tiles, dtype, coded, few):
    """Additions of 32 bits that follow each other: of a row's weighted sum, and of its weights.  Few rows: four of a block, of 256 blocks at most (over codes; of an fp32 cache four
    of 16 keys, 64 times), then waves and splits.  Else as many tiles as there are between two times that sums are put aside, with one addition each (fp32, behind 32 of the
    tile's own), four (16 bits) or eight (codes, fp32 queries); those times, and splits; of weights 16 in a tile and 2."""
    if few:
        return 4 * min(tiles, 256) + 32 + 264, 16 + 32 + 264
    apart = 512 if dtype != ta.F32 else 128 if coded else 256
    per_tile = (4 if dtype != ta.F32 else 8) * min(tiles, apart) if coded or dtype != ta.F32 else 32 + min(tiles, apart)
    return per_tile + tiles / apart + 72, 18 + min(tiles, apart) + tiles / apart + 72


def check(cache, dtype, fmt, K, V, Hq, M, sinks, window, few, seed):
    Hkv, n, d = K.shape
    G = Hq // Hkv
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 1)
    q = torch.randn((1, M, Hq, d), generator=g, device=DEV).to(TORCH[dtype])
    out, lse = cache.prompt(0, q, window=window, sinks=sinks)
    one = max(1, M // 7)
    at = sorted({0, M - 1, *range(one // 2, M, one), *(x for x in (63, 64, 127) if x < M)})
    pos = torch.tensor([n - M + i for i in at], device=DEV)
    t = torch.arange(n, device=DEV)
    seen = (t <= pos[:, None]) & ((t < sinks) | (t > pos[:, None] - (window or n)))                      # [rows, n]
    tiles = (n + 63) // 64
    chain, chain_l = chains(tiles, dtype, fmt is not None, few)
    for h in range(Hkv):
        k, v = K[h].double(), V[h].double()
        qs = q[0, at][:, h * G:(h + 1) * G].double().reshape(-1, d)                                      # rows: query, head of the group
        mask = seen.repeat_interleave(G, 0)
        s = (qs @ k.t() / math.sqrt(d)).masked_fill(~mask, -math.inf)
        w_lse = torch.logsumexp(s, 1, keepdim=True)
        p = torch.exp(s - w_lse)
        want, size = p @ v, p @ v.abs()
        A = (qs.abs() @ k.abs().t() / math.sqrt(d)).masked_fill(~mask, 0.0).amax(1, keepdim=True)
        # a score's d products, its factor and the difference to a reference up to 13 away, the exponential; fp32 queries over codes in two parts
        dw = (d + 10) * U * A + 4 * U + 3 * 14 * U + (2.0 ** -22 if fmt is not None else 0.0)
        # rounding of the weights: none in fp32, two parts of few rows over codes, else one of the type; over codes fp16, and of the type over the rows behind the last full block
        if dtype == ta.F32 or few:
            rounding = (2.0 ** -22 if fmt is not None else 0.0) * size
        elif fmt is None:
            rounding = HALF[dtype] * size
        else:
            full = n // 64 * 64
            rounding = HALF[ta.F16] * size + HALF[dtype] * (p[:, full:] @ v[full:].abs())
        floor = 0.0 if dtype != ta.F16 and fmt is None else mask.sum(1, keepdim=True) * 2.0 ** -36 * p.amax(1, keepdim=True) * v.abs().max()
        tol = 2 * dw * size + rounding + chain * U * size + (chain_l + 3) * U * want.abs() + floor + HALF[dtype] * want.abs()
        got = out[0, at][:, h * G:(h + 1) * G].double().reshape(-1, d)
        off = (got - want).abs()
        worst = (off / tol.clamp(min=1e-300)).max().item()
        assert bool((off <= tol).all()), f"head {h}: an output is {worst:.3g} times as far off as its roundings allow"
        got = lse[0, at][:, h * G:(h + 1) * G].double().reshape(-1, 1)
        off, allowed = (got - w_lse).abs(), dw + (chain_l + 3) * U + 4 * U * (w_lse.abs() + 1)
        assert bool((off <= allowed).all()), f"head {h}: lse off by {off.max():.3g}"


PLAIN = [  # dtype, Hq, Hkv, d, tokens, M, sinks, window
    (ta.BF16, 32, 8, 128, 5000, 20, 0, None),                    # keys split, blocks of 128 rows
    (ta.F16, 4, 1, 64, 3000, 8, 0, None),                        # split, one wave
    (ta.F16, 4, 1, 128, 9000, 500, 100, 1000),                   # split, two stretches
    (ta.F32, 4, 1, 64, 3000, 9, 0, None),                        # the walk of single tokens
    (ta.F32, 16, 2, 256, 3000, 40, 0, None),
    (ta.BF16, 8, 2, 128, 20000, 8192, 70, 3000),                 # whole, windows
    (ta.BF16, 4, 1, 128, 70000, 8192, 0, None),                  # whole, more tiles than sums are kept for
    (ta.F16, 4, 1, 64, 70001, 8192, 3, 66000),
    (ta.F16, 8, 2, 32, 33333, 8192, 0, None),
    (ta.BF16, 8, 1, 256, 34000, 4096, 0, None),
    (ta.F32, 4, 1, 64, 40000, 8192, 0, None),
    (ta.F32, 4, 1, 128, 17000, 8200, 64, 16500),
    (ta.F32, 16, 1, 32, 30000, 2048, 0, None),
    (ta.F32, 8, 1, 256, 17000, 4096, 0, None),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,d,n,M,sinks,window", PLAIN)
def test_prompt(dtype, Hq, Hkv, d, n, M, sinks, window):
    K, V = rows_of(Hkv, n, d, dtype, n)
    cache = ta.TopkAttnCache(1, 1, Hq, Hkv, d, n, 64, dtype)
    try:
        cache.append(0, 0, K, V, head_major=True)
        check(cache, dtype, None, K, V, Hq, M, sinks, window, dtype == ta.F32 and M * Hq // Hkv <= 64, n)
    finally:
        cache.close()


CODED = [  # format, dtype, Hq, Hkv, d, tokens, M, sinks, window, whether few rows
    (ta.CODED_E4M3, ta.BF16, 8, 2, 64, 9000, 64, 0, None, False),        # split
    (ta.CODED_INT8, ta.BF16, 4, 1, 256, 5000, 16, 0, None, True),        # as many rows as the kernel of single tokens takes, and some more
    (ta.CODED_INT8, ta.BF16, 4, 1, 256, 5000, 17, 0, None, False),
    (ta.CODED_E4M3, ta.F16, 4, 1, 64, 5000, 4, 0, None, True),
    (ta.CODED_E4M3, ta.F16, 4, 1, 64, 5000, 5, 0, None, False),
    (ta.CODED_INT8, ta.BF16, 4, 1, 32, 5000, 4, 70, 1000, True),
    (ta.CODED_INT8, ta.BF16, 4, 1, 32, 5000, 5, 70, 1000, False),
    (ta.CODED_INT8, ta.F16, 8, 2, 128, 5000, 8, 0, None, True),
    (ta.CODED_INT8, ta.F16, 8, 2, 128, 5000, 9, 0, None, False),
    (ta.CODED_E4M3, ta.F32, 4, 2, 256, 3000, 64, 0, None, True),
    (ta.CODED_E4M3, ta.F32, 4, 2, 256, 3000, 65, 0, None, False),
    (ta.CODED_INT8, ta.F32, 4, 1, 128, 3000, 16, 0, None, True),
    (ta.CODED_INT8, ta.F32, 4, 1, 128, 3000, 17, 0, None, False),
    (ta.CODED_E4M3, ta.F16, 8, 2, 128, 20000, 8192, 70, 3000, False),    # whole, windows
    (ta.CODED_INT8, ta.F16, 4, 1, 128, 70050, 8192, 0, None, False),     # whole, more blocks than sums are kept for, and open rows
    (ta.CODED_E4M3, ta.BF16, 4, 1, 64, 40000, 8192, 0, None, False),
    (ta.CODED_INT8, ta.F32, 4, 1, 64, 20010, 8192, 0, None, False),
    (ta.CODED_INT8, ta.BF16, 8, 1, 256, 33000, 4096, 0, None, False),
    (ta.CODED_E4M3, ta.F32, 8, 1, 256, 9000, 4096, 5, 8500, False),
]


@pytest.mark.parametrize("fmt,dtype,Hq,Hkv,d,n,M,sinks,window,few", CODED)
def test_prompt_over_codes(fmt, dtype, Hq, Hkv, d, n, M, sinks, window, few):
    K, V = rows_of(Hkv, n, d, dtype, n)
    cache = ta.TopkAttnCodedCache(1, 1, Hq, Hkv, d, n, dtype, format=fmt)
    try:
        cache.append(0, K.transpose(0, 1)[None], V.transpose(0, 1)[None])
        check(cache, dtype, fmt, held(K, fmt), held(V, fmt), Hq, M, sinks, window, few, n)
    finally:
        cache.close()


@pytest.mark.parametrize("fmt", [None, ta.CODED_E4M3])
@pytest.mark.parametrize("dtype,n", [(ta.BF16, 34000), (ta.F32, 17000)])
def test_captured_long_prompts_replay(dtype, n, fmt):
    """Walks whose sums are put aside, recorded before any such call was made eagerly, replayed with other queries and eager calls between, on another stream beside them."""
    Hq, Hkv, d, M = 4, 1, 64, 8192
    K, V = rows_of(Hkv, n, d, dtype, n)
    caches = []
    for _ in range(2):
        if fmt is None:
            caches.append(ta.TopkAttnCache(1, 1, Hq, Hkv, d, n, 64, dtype))
            caches[-1].append(0, 0, K, V, head_major=True)
        else:
            caches.append(ta.TopkAttnCodedCache(1, 1, Hq, Hkv, d, n, dtype, format=fmt))
            caches[-1].append(0, K.transpose(0, 1)[None], V.transpose(0, 1)[None])
    try:
        g = torch.Generator(device=DEV)
        g.manual_seed(3)
        q = torch.empty((1, M, Hq, d), device=DEV, dtype=TORCH[dtype])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            recorded = caches[0].prompt(0, q)
        side = torch.cuda.Stream()
        for _ in range(3):
            q.copy_(torch.randn(q.shape, generator=g, device=DEV))
            side.wait_stream(torch.cuda.current_stream())
            graph.replay()
            with torch.cuda.stream(side):
                beside = caches[1].prompt(0, q)
            torch.cuda.synchronize()
            got = [x.clone() for x in recorded]
            eager = caches[0].prompt(0, q)
            assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(got, eager, beside))
    finally:
        for cache in caches:
            cache.close()


@pytest.mark.parametrize("fmt", [None, ta.CODED_INT8])
@pytest.mark.parametrize("dtype", [ta.F32, ta.F16, ta.BF16])
def test_prompts_without_lse_and_without_tokens(dtype, fmt):
    """Few rows, split and whole walks give the same output when nothing but it is asked for; no queries are no call."""
    Hq, Hkv, d, n = 4, 2, 64, 1500
    K, V = rows_of(Hkv, n, d, dtype, n)
    if fmt is None:
        cache = ta.TopkAttnCache(1, 1, Hq, Hkv, d, n, 64, dtype)
        cache.append(0, 0, K, V, head_major=True)
    else:
        cache = ta.TopkAttnCodedCache(1, 1, Hq, Hkv, d, n, dtype, format=fmt)
        cache.append(0, K.transpose(0, 1)[None], V.transpose(0, 1)[None])
    try:
        q = torch.randn((1, n, Hq, d), device=DEV).to(TORCH[dtype])
        for M in (1, 3, 100, n):
            last = q[:, n - M:].contiguous()
            out, lse = cache.prompt(0, last)
            alone, none = cache.prompt(0, last, want_lse=False)
            assert none is None and torch.equal(out, alone) and lse.shape == (1, M, Hq)
        out, lse = cache.prompt(0, q[:, :0])
        assert out.shape == (1, 0, Hq, d) and lse.shape == (1, 0, Hq)
    finally:
        cache.close()
