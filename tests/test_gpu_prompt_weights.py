"""Attention of a prompt's tokens where many small weights make up the result, on the GPU through the binding, against closed forms in 64 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import coded_cache_ref as ref
from paper_2502_06766_amd import topk_attn as ta

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0) if torch.cuda.is_available() else None
U = 2.0 ** -24                                                   # half a step of fp32 relative to the value
HALF = {ta.F32: 2.0 ** -24, ta.F16: 2.0 ** -11, ta.BF16: 2.0 ** -8}
TORCH = {ta.F32: torch.float32, ta.F16: torch.float16, ta.BF16: torch.bfloat16}


def cache_of(K, V, Hq, dtype, fmt):
    """A cache of one sequence that holds K, V [Hkv, n, d]; fmt None: in its own type."""
    Hkv, n, d = K.shape
    K, V = (x.to(TORCH[dtype]) for x in (K, V))
    if fmt is None:
        cache = ta.TopkAttnCache(1, 1, Hq, Hkv, d, n, 64, dtype)
        cache.append(0, 0, K, V, head_major=True)
    else:
        cache = ta.TopkAttnCodedCache(1, 1, Hq, Hkv, d, n, dtype, format=fmt)
        cache.append(0, K.transpose(0, 1)[None], V.transpose(0, 1)[None])
    return cache


def decode(cache, fmt, q):
    return cache.decode_dense(0, q) if fmt is None else cache.decode(0, q)


# ---- one key far above many others ---------------------------------------------------------------------------------------
def check_small_weights(dtype, fmt, n, nats):
    """A first token that scores `nats` above all others and whose value is zero: the output is made of the others' weights alone.  Rows that are walked whole, and
    few rows whose keys are split.

    The first token's key is 16 in one channel, a number that e4m3 holds as it is and int8 as 127 times the block's scale."""
    d, G = 64, 4
    K, V = torch.zeros((1, n, d), device=DEV), torch.ones((1, n, d), device=DEV)
    K[0, 0, 0], V[0, 0] = 16.0, 0.0
    cache = cache_of(K, V, G, dtype, fmt)
    try:
        top = 16.0
        if fmt == ta.CODED_INT8:
            m, e = math.frexp(float(np.float32(16) / np.float32(127)))
            top = 127 * math.ldexp(float(np.rint(m * 65536)) / 65536, e)
        top *= nats / 16
        for M in (8192, 2):
            q = torch.zeros((1, M, G, d), device=DEV, dtype=TORCH[dtype])
            q[..., 0] = nats / 2                                 # times 16 over sqrt(64)
            out, lse = cache.prompt(0, q)
            one, _ = decode(cache, fmt, q[:, -1].contiguous())
            p = torch.arange(n - M, n, device=DEV, dtype=torch.float64)
            total = math.exp(top) + p
            want = (p / total)[:, None, None]
            # the exponent is a product with a factor of 32 bits and a difference (3 u of it and of its integer reference, which is 13 more in fp16), the exponential
            # 4 u; a weight's rounding and the output's; sums one after the other, 16 keys at a time
            exponent = 3 * U * (top * 1.4427 + 14) + 4 * U
            # (over codes: half a step of 2^-37 of the largest weight, times a value scale that is at least half of the power of two it is relative to; fp32 queries: two
            # parts, 2^-22)
            weight = max(HALF[dtype] if dtype != ta.F32 else 2.0 ** -22, 0.0 if fmt is None else 2.0 ** -37 * math.exp(top))
            tol = (weight + HALF[dtype] + 2 * exponent + (n / 16 + 64) * U) * want
            off = (out[0].double() - want).abs()
            assert bool((off <= tol).all()), f"{M} rows: off by {(off / want).max():.3g} of the output, {(tol / want).max():.3g} allowed"
            off = (lse[0].double() - torch.log(total)[:, None]).abs().max().item()
            assert off <= exponent + (n / 16 + 64) * U + 4 * U * math.log(total.max()), f"{M} rows: lse off by {off:.3g}"
        # the single token's decode holds weights in two parts, with steps of 2^-37 of the largest where they are small: half of one is 2^-10.9 of a weight 18.75 nats below
        off = (one[0].double() - want[-1]).abs().max().item() / want[-1].item()
        assert off <= 2.0 ** -10.9 + 2 * exponent + (n / 16 + 64) * U
    finally:
        cache.close()


@pytest.mark.parametrize("nats", [14, 16, 17, 18, 18.75])
@pytest.mark.parametrize("n", [65537, 131073])
@pytest.mark.parametrize("dtype", [ta.F16, ta.BF16])
def test_small_weights_add_up(dtype, n, nats):
    check_small_weights(dtype, None, n, nats)


@pytest.mark.parametrize("nats", [14, 16, 17, 18, 18.75])
@pytest.mark.parametrize("n", [65537, 131073])
@pytest.mark.parametrize("fmt", [ta.CODED_INT8, ta.CODED_E4M3])
@pytest.mark.parametrize("dtype", [ta.F16, ta.BF16, ta.F32])
def test_small_weights_over_codes_add_up(dtype, fmt, n, nats):
    check_small_weights(dtype, fmt, n, nats)


def large_scores(d):
    """Queries and keys of one channel whose exponents of two lie between 2^24 and 2^27, where numbers of 32 bits are 2 to 8 apart."""
    for q0 in (16384.0, 19968.0, 24576.0):
        for k0 in range(4096, 32768, 1024):
            if 2 ** 24 <= q0 * k0 / math.sqrt(d) * math.log2(math.e) < 2 ** 27:
                yield q0, k0


@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype,fmt", [(ta.F16, None), (ta.BF16, None), (ta.F16, ta.CODED_INT8), (ta.BF16, ta.CODED_E4M3)])
def test_scores_beyond_2_24(dtype, fmt, d):
    """Equal scores that large: the weights stay in the type's range, and the output is the values' mean."""
    n, G, M = 333 if fmt is None else 320, 2, 100                 # (over codes: full blocks, whose keys all read as one number)
    V = torch.rand((1, n, d), device=DEV) + 0.5
    for q0, k0 in large_scores(d):
        K = torch.zeros((1, n, d), device=DEV)
        K[0, :, 0] = k0
        cache = cache_of(K, V, G, dtype, fmt)
        try:
            q = torch.zeros((1, M, G, d), device=DEV, dtype=TORCH[dtype])
            q[..., 0] = q0
            out, lse = cache.prompt(0, q)
            rows = V[0].to(TORCH[dtype]).double()
            if fmt is not None:
                rows = torch.from_numpy(ref.held(rows.cpu().numpy(), fmt)).to(DEV)
            want = (rows.cumsum(0) / torch.arange(1, n + 1, device=DEV, dtype=torch.float64)[:, None])[n - M:]
            # (all weights alike, rounded once; the output)
            assert bool(((out[0].double() - want[:, None]).abs() <= (2 * HALF[dtype] + 1024 * U) * want[:, None]).all()), (q0, k0)
            assert bool(torch.isfinite(lse).all())
        finally:
            cache.close()


@pytest.mark.parametrize("fmt", [ta.CODED_INT8, ta.CODED_E4M3])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [ta.F16, ta.BF16, ta.F32])
def test_single_tokens_and_few_rows_over_codes_beyond_2_24(dtype, d, fmt):
    """The same of the kernel of single tokens: one token, and the last two."""
    n, G = 320, 2
    V = torch.rand((1, n, d), device=DEV) + 0.5
    for q0, k0 in large_scores(d):
        K = torch.zeros((1, n, d), device=DEV)
        K[0, :, 0] = k0
        cache = cache_of(K, V, G, dtype, fmt)
        try:
            q = torch.zeros((1, 2, G, d), device=DEV, dtype=TORCH[dtype])
            q[..., 0] = q0
            rows = torch.from_numpy(ref.held(V[0].to(TORCH[dtype]).double().cpu().numpy(), fmt)).to(DEV)
            # (weights alike, in two parts of fp16: their reference is up to 24 powers above them, 13 are shifted, and the second part of 2^-11 has steps of 2^-24; 80 blocks)
            weight = 2.0 ** -13
            for out, m, half in ((cache.decode(0, q[:, -1].contiguous())[0][:, None], 1, 0.0), (cache.prompt(0, q)[0], 2, HALF[dtype])):
                want = (rows.cumsum(0) / torch.arange(1, n + 1, device=DEV, dtype=torch.float64)[:, None])[n - m:]
                assert bool(((out[0].double() - want[:, None]).abs() <= (weight + half + 600 * U) * want[:, None]).all()), (q0, k0, m)
        finally:
            cache.close()


# ---- sums of many equal weights ------------------------------------------------------------------------------------------
def equal_weights(fmt, dtype):
    """A score and a value that the cache reads back exactly, and a query whose weights do not end in 32 bits: key, value, query, score."""
    one = 127 / 128 if fmt == ta.CODED_INT8 else 1.0             # (int8: 127 times a power of two, e4m3 and the types: itself)
    q = torch.tensor(21.7).to(TORCH[dtype]).item()
    return one, one, q, q * one / 8.0


@pytest.mark.parametrize("dtype,fmt,n", [(ta.F32, None, 65537), (ta.F32, None, 200001), (ta.F32, ta.CODED_INT8, 200001), (ta.F32, ta.CODED_E4M3, 200001), (ta.F16, None, 1 << 20),
                                         (ta.BF16, None, 1 << 20), (ta.F16, ta.CODED_INT8, 1 << 20), (ta.BF16, ta.CODED_E4M3, 1 << 20)])
def test_sums_of_many_equal_weights(dtype, fmt, n):
    """Rows as many as fill the chip, so that their keys are not split: sums that grow along the whole cache, of numbers of one sign."""
    d, G, M = 64, 4, 8192
    k, v, q0, score = equal_weights(fmt, dtype)
    K, V = torch.zeros((1, n, d), device=DEV), torch.zeros((1, n, d), device=DEV)
    K[0, :, 0] = k
    V[0, :, 0] = v
    V[0, ::3, 1:] = v
    cache = cache_of(K, V, G, dtype, fmt)
    try:
        q = torch.zeros((1, M, G, d), device=DEV, dtype=TORCH[dtype])
        q[..., 0] = q0
        out, lse = cache.prompt(0, q)
        seen = torch.arange(n - M, n, device=DEV, dtype=torch.float64) + 1
        # a weight as the second product takes it, relative to the power of two above: 16 bits round it once
        w = torch.tensor(2.0 ** (score * math.log2(math.e) - math.ceil(score * math.log2(math.e))), dtype=torch.float64)
        if dtype != ta.F32:
            w = w.to(torch.float16 if fmt is not None else TORCH[dtype]).double() / w
        else:
            w = torch.ones(())
        want = torch.stack([torch.ones_like(seen), torch.floor((seen + 2) / 3) / seen], 1) * v * w.item()
        # Additions that follow each other, half a step of the sum each at most.  Weighted sum: in a tile 32 (fp32; and one of them to the sum so far), 4 (16 bits) or 8 (codes,
        # fp32 queries), as many tiles as there are between two times that the sums are put aside, and those times; weights: 16 in a tile and 2, then the same.
        apart = 512 if dtype != ta.F32 else 256 if fmt is None else 128
        folds = n / 64 / apart
        chain = (32 + apart if fmt is None else 8 * apart) if dtype == ta.F32 else 4 * apart
        sums = (chain + folds + 18 + apart + folds + 8) * U + (2.0 ** -22 if fmt is not None and dtype == ta.F32 else 0)
        off = (out[0, :, :, :2].double() / want[:, None] - 1).abs().max().item()
        # (the expected weight is that of 64 bits: 20 u of what 32 bits make of it may round to the neighbour, a step of the type)
        assert off <= sums + (HALF[dtype] + 20 * U if dtype != ta.F32 else 4 * U), f"out off by {off:.3g}, {sums:.3g} allowed for sums"
        off = (lse[0].double() - (score + torch.log(seen))[:, None]).abs().max().item()
        allowed = (18 + apart + folds) * U + 3 * U * (score * 1.4427 + 14) + 4 * U + 4 * U * (score + math.log(n))
        assert off <= allowed, f"lse off by {off:.3g}, {allowed:.3g} allowed"
    finally:
        cache.close()


@pytest.mark.parametrize("fmt", [ta.CODED_INT8, ta.CODED_E4M3])
def test_sums_of_few_rows_of_many_streams(fmt):
    """512 sequences of 2^20 tokens, 64 rows each: as many partial sums as the workspace has room for, and the walks between them of a length that does not
    grow with the cache.  (Every sequence holds the same rows.)"""
    d, n, B, M, dtype = 32, 1 << 20, 512, 64, ta.F32
    _, v, q0, _ = equal_weights(fmt, dtype)
    score = q0 * v / math.sqrt(d)                                # (the keys are the values, whose first channel alone meets the query)
    V = torch.zeros((n, d), device=DEV)
    V[:, 0] = v
    V[::3, 1:] = v
    cache = ta.TopkAttnCodedCache(1, B, 1, 1, d, n, dtype, format=fmt)
    try:
        ta.topk_attn_coded_append(cache.h, 0, -1, V.data_ptr(), V.data_ptr(), n, 0, d, d, torch.cuda.current_stream().cuda_stream)
        q = torch.zeros((B, M, 1, d), device=DEV)
        q[..., 0] = q0
        out, lse = cache.prompt(0, q)
        seen = torch.arange(n - M, n, device=DEV, dtype=torch.float64) + 1
        want = torch.stack([torch.ones_like(seen), torch.floor((seen + 2) / 3) / seen], 1) * v
        # additions that follow each other: four of a block, at most 256 blocks of a wave, then waves and splits; the weights' sum keeps what its additions round off
        sums = (4 * 256 + 4 + 16 + 32 + 8) * U + 2.0 ** -22
        off = (out[:, :, 0, :2].double() / want - 1).abs().max().item()
        assert off <= sums + 4 * U, f"out off by {off:.3g}, {sums:.3g} allowed for sums"
        off = (lse[:, :, 0].double() - (score + torch.log(seen))).abs().max().item()
        allowed = 60 * U + 3 * U * (score * 1.4427 + 1) + 4 * U + 4 * U * (score + math.log(n))
        assert off <= allowed, f"lse off by {off:.3g}, {allowed:.3g} allowed"
    finally:
        cache.close()
