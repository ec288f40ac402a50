"""Edges of the operators beside the top-k decode, on the GPU through the binding: NaN among keys, products and sums beyond the range or the
length that 32 bits take, calls recorded before a sequence grew, and sums held to a few roundings."""
import ctypes

import numpy as np
import pytest
import torch

import helpers as H
import operator_bounds as ob
from oracle import operators_ref as ref
from paper_2502_06766_amd import topk_attn as ta
from paper_2502_06766_amd import workloads as wl

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0) if torch.cuda.is_available() else None
U = 2.0 ** -24                                                   # half a step of fp32 relative to the value
TYPES = [wl.F32, wl.F16, wl.BF16]


def draw(g, *shape, dtype):
    return wl.quantize(g.standard_normal(shape).astype(np.float32), dtype)


def filled(K, V, dtype, Hq, index=ta.INDEX_NONE, room=0, max_k=8):
    """A cache of one sequence with keys and values [Hkv, n, d] in the storage type; unused rows are NaN."""
    Hkv, n, d = K.shape
    cache = ta.TopkAttnCache(1, 1, Hq, Hkv, d, n + room, max_k, dtype, index_kind=index)
    cache.kv.fill_(255)
    cache.append(0, 0, H.to_torch(K, dtype, DEV), H.to_torch(V, dtype, DEV), head_major=True)
    return cache


def close(got, want, K, q, V, d, label):
    """out of finite heads: scores off by (d + 6) u sum |q k| / sqrt(d), weights by as much, values up to max |V|."""
    Hkv = K.shape[0]
    A = max((np.abs(K[h]) @ np.abs(q.reshape(Hkv, -1, d)[h]).T).max() for h in range(Hkv)) / np.sqrt(d)
    tol = 2 * ((d + 6) * U * A + (K.shape[1] / 16 + 64) * U + 2.0 ** -18) * np.abs(V).max()
    assert np.abs(got - want).max() <= tol, f"{label}: off by {np.abs(got - want).max():.3g}, {tol:.3g} allowed"


@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,before", [(1, 0), (17, 0), (33, 0), (33, 8), (65, 0), (97, 0), (97, 64), (129, 0), (641, 0), (5000, 0), (40001, 200)])
def test_a_nan_key_is_not_lost(n, before, dtype, blocks):
    """The newest key of KV head 1 is NaN, alone in its step or its split, or behind keys of -inf: its heads, their lse and their weights are
    NaN, whatever else there is; the other heads' are those of finite keys."""
    Hq, Hkv, d, n_blocks = 8, 4, 128, 3
    g = np.random.default_rng(n + before)
    K, V = draw(g, Hkv, n, d, dtype=dtype), draw(g, Hkv, n, d, dtype=dtype)
    q = np.abs(wl.widen(draw(g, 1, Hq, d, dtype=dtype), dtype)).astype(np.float32) + np.float32(0.1)
    q = wl.quantize(q, dtype)
    Kf = wl.widen(K, dtype).astype(np.float32)
    Kf[1, n - 1 - before:n - 1, 3] = -np.inf
    Kf[1, n - 1, 7] = np.nan
    K = wl.quantize(Kf, dtype) if dtype != wl.BF16 else (Kf.view(np.uint32) >> 16).astype(np.uint16)
    cache = filled(K, V, dtype, Hq, ta.INDEX_BOXES if blocks else ta.INDEX_NONE, room=3)
    try:
        for mass in (None, torch.zeros((1, Hkv, n + 3), device=DEV)):
            if blocks:
                out, pages, lse = cache.decode_blocks(0, H.to_torch(q, dtype, DEV), n_blocks, mass=mass)
                at = ref.block_tokens([[p for p in x if p >= 0] for x in pages[0].cpu().numpy()], n)
            else:
                out, lse = cache.decode_dense(0, H.to_torch(q, dtype, DEV), mass=mass)
                at = [np.arange(n)] * Hkv
            out, lse = out[0].double().cpu().numpy(), lse[0].double().cpu().numpy()
            assert np.isnan(out[2:4]).all() and np.isnan(lse[2:4]).all()
            q64, V64 = wl.widen(q[0], dtype), wl.widen(V, dtype)
            fine = [0, 2, 3]
            K64 = Kf.astype(np.float64)
            K64[1] = 0.0
            want, want_lse, want_mass = ref.attend(q64, K64, V64, at)
            heads = [0, 1, 4, 5, 6, 7]
            close(out[heads], want[heads], K64, q64, V64, d, f"{n} tokens")
            assert np.isfinite(lse[heads]).all()
            if mass is not None:
                m = mass[0].cpu().numpy()
                assert np.isnan(m[1, at[1]]).all() and (m[:, n:] == 0).all()
                for h in fine:
                    assert np.isfinite(m[h]).all() and abs(m[h].sum() - 2) < 1e-3
    finally:
        cache.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [33, 65, 641])
def test_an_infinite_key_is_nan_for_the_heads_that_meet_it_with_zero(n, dtype):
    """One infinite channel of the newest key: heads of a zero there score NaN, of a positive number +inf (NaN too), of a negative one -inf: the
    key has no weight."""
    d, Hq = 64, 3
    g = np.random.default_rng(n)
    K, V = draw(g, 1, n, d, dtype=dtype), draw(g, 1, n, d, dtype=dtype)
    Kf, qf = wl.widen(K, dtype).astype(np.float32), wl.widen(draw(g, 1, Hq, d, dtype=dtype), dtype).astype(np.float32)
    Kf[0, n - 1, 5] = np.inf
    qf[0, :, 5] = [0.0, 1.0, -1.0]
    K, q = wl.quantize(Kf, dtype), wl.quantize(qf, dtype)
    cache = filled(K, V, dtype, Hq)
    try:
        out, lse = cache.decode_dense(0, H.to_torch(q, dtype, DEV))
        out, lse = out[0].double().cpu().numpy(), lse[0].double().cpu().numpy()
        assert np.isnan(out[:2]).all() and np.isnan(lse[:2]).all()
        q64, K64, V64 = wl.widen(q[0], dtype), wl.widen(K, dtype)[:, :n - 1], wl.widen(V, dtype)[:, :n - 1]
        want, want_lse, _ = ref.attend(q64, K64, V64)
        close(out[2:], want[2:], K64, q64, V64, d, f"{n} tokens")
    finally:
        cache.close()


def page_order(q, K, n_blocks):
    """The pages attended, by the definition with NaN: a page whose score is NaN comes before all numbers (equal ones by page)."""
    d = K.shape[2]
    lists = []
    for h in range(K.shape[0]):
        rows = K[h].astype(np.float64)
        group = q.reshape(K.shape[0], -1, d)[h].astype(np.float64)
        score = []
        for p in range(0, rows.shape[0], 64):
            lo, hi = rows[p:p + 64].min(0), rows[p:p + 64].max(0)         # (numpy's keep a NaN)
            with np.errstate(invalid="ignore"):
                score.append(np.where(group >= 0, group * hi, group * lo).sum(1).max())
        older = sorted(range(len(score) - 1), key=lambda p: (0 if np.isnan(score[p]) else 1, 0 if np.isnan(score[p]) else -score[p], p))
        lists.append(sorted(older[:n_blocks - 1] + [len(score) - 1]))
    return lists


@pytest.mark.parametrize("dtype,pages", [(wl.F32, 40), (wl.F16, 40), (wl.BF16, 40), (wl.F16, 1500), (wl.F32, 5000)])
def test_a_page_of_nan_scores_comes_first(dtype, pages):
    """A NaN key, a page of nothing but NaN, an infinite edge that a zero of the query meets: the page is attended, and its heads are NaN as in
    the dense decode; more such pages than are asked for go by their number."""
    Hq, Hkv, d, n = 4, 2, 32, 64 * pages - 13
    g = np.random.default_rng(pages)
    Kf = wl.widen(draw(g, Hkv, n, d, dtype=dtype), dtype).astype(np.float32)
    qf = wl.widen(draw(g, 1, Hq, d, dtype=dtype), dtype).astype(np.float32)
    qf[0, 0, 9] = 0.0
    Kf[0, 64 * 7 + 63, 31] = np.nan                              # one number of one key
    Kf[0, 64 * 20:64 * 21] = np.nan                              # a whole page
    Kf[0, 64 * 30 + 5, 9] = np.inf                               # where head 0 has a zero
    Kf[1, 64 * 11:64 * 12, 4] = np.nan                           # a channel of all keys
    K = wl.quantize(Kf, dtype) if dtype != wl.BF16 else (Kf.view(np.uint32) >> 16).astype(np.uint16)
    K32 = wl.widen(K, dtype)
    q, V = wl.quantize(qf, dtype), draw(g, Hkv, n, d, dtype=dtype)
    cache = filled(K, V, dtype, Hq, ta.INDEX_BOXES)
    try:
        for n_blocks in (1, 2, 3, 4, 6, 25):
            out, blocks, lse = cache.decode_blocks(0, H.to_torch(q, dtype, DEV), n_blocks)
            want = page_order(wl.widen(q[0], dtype), K32, n_blocks)
            assert [list(x) for x in blocks[0].cpu().numpy()] == want, n_blocks
            assert torch.isnan(out[0, 2:]).all().item() == (n_blocks > 1) and torch.isnan(lse[0, :2]).all().item() == (n_blocks > 1)
    finally:
        cache.close()


@pytest.mark.parametrize("dtype", TYPES)
def test_the_boxes_keep_a_nan(dtype):
    """A NaN written by one append is in the box after the next ones, after an eviction that keeps its row, and gone after one that does not."""
    d, Hkv, cap = 64, 1, 300
    cache = ta.TopkAttnCache(1, 1, 1, Hkv, d, cap, 8, dtype, index_kind=ta.INDEX_BOXES)
    try:
        size = (cap * d * wl.DTYPE_BYTES[dtype] + 255) // 256 * 256
        boxes = cache.kv[2 * size:2 * size + 5 * 2 * d * wl.DTYPE_BYTES[dtype]].view(cache.torch_dtype()).view(5, 2, d)
        one = torch.ones((1, Hkv, d), dtype=cache.torch_dtype(), device=DEV)
        odd = one.clone()
        odd[0, 0, 17] = float("nan")
        cache.append(0, 0, one.expand(70, Hkv, d).contiguous(), one.expand(70, Hkv, d).contiguous())
        cache.append_step(0, odd[None], one[None])
        for step in range(3):
            want = torch.zeros((2, d), dtype=torch.bool, device=DEV)
            want[:, 17] = True
            assert torch.equal(torch.isnan(boxes[1]), want) and not torch.isnan(boxes[0]).any(), step
            if step == 0:
                cache.append_step(0, one[None].expand(1, 20, Hkv, d).contiguous(), one[None].expand(1, 20, Hkv, d).contiguous())
            else:
                cache.append_rotary(0, None, one[None], one[None], torch.ones(0, device=DEV))
        mass = torch.zeros((1, Hkv, cap), device=DEV)
        mass[0, 0, 70] = 1.0
        cache.evict(0, mass, 80, 0)                               # (the oldest of equal weights and row 70)
        assert torch.isnan(boxes[1, :, 17]).all() and not torch.isnan(boxes[0]).any()
        cache.evict(0, mass, 65, 0)
        assert cache.length(0, 0) == 65
        assert torch.isnan(boxes[1, :, 17]).all() and not torch.isnan(boxes[0]).any()
        mass[0, 0] = torch.arange(cap, 0, -1, device=DEV)         # (row 64 holds the NaN: the lightest)
        cache.evict(0, mass, 64, 0)
        assert not torch.isnan(boxes[0]).any()
    finally:
        cache.close()


@pytest.mark.parametrize("dtype", [wl.BF16, wl.F32])
@pytest.mark.parametrize("q_size,low,high", [(1e30, -30, 30), (1.0, -30, 30), (1e-30, -36, -15)])
def test_page_scores_beyond_the_range_of_32_bits(dtype, q_size, low, high):
    """Products of a query and a box edge above 2^128 or below 2^-149: pages are ordered by them all the same."""
    d, pages, n_blocks = 32, 700, 60
    n = 64 * pages - 5
    g = np.random.default_rng(17)
    size = (10.0 ** g.uniform(low, high, (1, pages, 1))).astype(np.float32) * np.where(g.random((1, pages, 1)) < 0.5, -1, 1).astype(np.float32)
    K = wl.quantize((size.repeat(64, 1)[:, :n] * g.uniform(0.5, 1.0, (1, 1, d))).astype(np.float32), dtype)
    q = wl.quantize((q_size * g.uniform(0.5, 1.0, (1, 2, d))).astype(np.float32), dtype)
    cache = filled(K, draw(g, 1, n, d, dtype=dtype), dtype, 2, ta.INDEX_BOXES)
    try:
        _, blocks, _ = cache.decode_blocks(0, H.to_torch(q, dtype, DEV), n_blocks)
        assert list(blocks[0, 0].cpu().numpy()) == ref.pick_blocks(wl.widen(q[0], dtype), wl.widen(K, dtype), n_blocks)[0]
    finally:
        cache.close()


@pytest.mark.parametrize("dtype,n,with_mass", [(wl.F16, 131072, False), (wl.BF16, 131072, True), (wl.F32, 65536, False)])
def test_sums_of_many_equal_weights(dtype, n, with_mass):
    """As many key streams as there are compute units, so that a sequence is one split: one key above all the others, whose weights
    are equal and not powers of two.  Added up one after the other in 32 bits such weights round the same way for as long as the sum
    stays between two powers of two (8192 of them: off by up to 9e-5)."""
    B, Hkv, G, d = 32, 8, 4, 32
    cache = ta.TopkAttnCache(1, B, Hkv * G, Hkv, d, n, 8, dtype)
    try:
        dt = cache.torch_dtype()
        K = torch.zeros((Hkv, n, d), dtype=dt, device=DEV)
        V = torch.zeros((Hkv, n, d), dtype=dt, device=DEV)
        K[:, 1:, 0] = -1.0
        V[:, :, 0] = 1.0
        V[:, :, 1] = ((torch.arange(n, device=DEV) // 64) % 2).to(dt)
        V[:, 1:, 2] = 1.0
        for b in range(B):
            cache.append(0, b, K, V, head_major=True)
        g = np.random.default_rng(3)
        q = torch.zeros((B, Hkv * G, d), device=DEV)
        gap = torch.from_numpy(g.integers(16, 256, (B, Hkv * G)).astype(np.float32) / 32).to(DEV)
        q[:, :, 0] = gap
        mass = torch.zeros((B, Hkv, n), device=DEV) if with_mass else None
        out, lse = cache.decode_dense(0, q.to(dt), mass=mass)
        w = torch.exp(-gap.double() / np.sqrt(d))
        total = 1.0 + (n - 1) * w
        odd = (torch.arange(n) // 64 % 2).sum().item()
        # a weight: the exponent's rounding, up to 2^4 in fp16 (8 u), its factor's (2 u of at most 3), the exponential (2 u), the parts (4 u);
        # a sum: 64 steps of a wave, the larger sums of those (n / 2048 of fp32 at most), steps, lanes, waves (16), an addition each
        weight, sums = 16 * U, (64 + n / 2048 + 16) * U
        assert ((lse.double() - total.log()).abs() <= weight + sums + 3 * U * total.log()).all(), (lse.double() - total.log()).abs().max()
        # of the weighted sum, whose steps are up to 8 roundings of the sum each
        for c, want in ((0, torch.ones_like(w)), (1, odd * w / total), (2, (n - 1) * w / total)):
            off = ((out[:, :, c].double() - want).abs() / want).max().item()
            assert off <= 2 * weight + 8 * sums, f"channel {c}: off by {off:.3g}, {2 * weight + 8 * sums:.3g} allowed"
        assert (out[:, :, 3:] == 0).all()
        if with_mass:
            want = (w / total).view(B, Hkv, G).sum(2)
            assert ((mass[:, :, -1].double() - want).abs() <= (weight + sums + 20 * U * total.log().max()) * want).all()
    finally:
        cache.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_blocks", [0, 290])
def test_long_splits_of_changing_scores(dtype, n_blocks):
    """Splits of thousands of keys, dense and over lists of pages, with weights: scores that rise, fall and begin with thousands of -inf, so that
    what a wave has put aside is rescaled in every way; lengths that end within and right after its first steps."""
    B, Hkv, G, d, cap = 32, 8, 2, 32, 20001
    lens = [cap - 331 * b for b in range(B - 3)] + [8192, 8193, 4097]
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    cache = ta.TopkAttnCache(1, B, Hkv * G, Hkv, d, cap, 8, dtype, index_kind=ta.INDEX_BOXES if n_blocks else ta.INDEX_NONE)
    try:
        dt = cache.torch_dtype()
        q = torch.randn((B, Hkv * G, d), generator=g, device=DEV)
        q[:, :, 0] = 1.0
        q, q_in = q.to(dt).double(), q.to(dt)
        K = torch.randn((Hkv, cap, d), generator=g, device=DEV)
        ramp = torch.linspace(0, 60, cap, device=DEV)
        K[0, :, 0], K[1, :, 0], K[2, :, 0] = ramp, -ramp, 30 * torch.sin(ramp)
        K[3, :9000, 0] = -float("inf")
        V = torch.randn((Hkv, cap, d), generator=g, device=DEV).to(dt)
        K = K.to(dt)
        for b, n in enumerate(lens):
            cache.append(0, b, K[:, :n].contiguous(), V[:, :n].contiguous(), head_major=True)
        mass = torch.zeros((B, Hkv, cap), device=DEV)
        if n_blocks:
            out, blocks, lse = cache.decode_blocks(0, q_in, n_blocks, mass=mass)
        else:
            out, lse = cache.decode_dense(0, q_in, mass=mass)
        A = 0.0
        for b in (0, 5, 17, B - 3, B - 2, B - 1):
            n = lens[b]
            finite = torch.nan_to_num(K[:, :n].double(), neginf=0.0)
            A = torch.matmul(finite.abs(), q[b].abs().view(Hkv, G, d).transpose(1, 2).contiguous()).max().item() / np.sqrt(d)
            s = torch.matmul(K[:, :n].double(), q[b].view(Hkv, G, d).transpose(1, 2).contiguous()) / np.sqrt(d)          # [Hkv, n, G]
            if n_blocks:
                held = torch.zeros((Hkv, (n + 63) // 64), dtype=torch.bool, device=DEV)
                for h in range(Hkv):
                    held[h, blocks[b, h][blocks[b, h] >= 0].long()] = True
                s = torch.where(held.repeat_interleave(64, 1)[:, :n, None], s, -float("inf"))
            w = torch.softmax(s, 1)
            want = torch.matmul(w.transpose(1, 2).contiguous(), V[:, :n].double()).view(Hkv * G, d)
            dw = (d + 6) * U * A + 4 * U + 2.0 ** -18 + (n / 16 + 64) * U
            live = torch.isfinite(want).all(1)                   # (a head whose keys are all of -inf has no result)
            assert live.sum() >= (Hkv - 1) * G
            off = (out[b].double() - want)[live].abs().max().item()
            assert off <= 2 * dw * V.abs().max().item(), f"sequence {b}: off by {off:.3g}"
            want = torch.logsumexp(s, 1).view(Hkv * G)
            assert ((lse[b].double() - want)[live].abs() <= dw + 4 * U * want[live].abs()).all()
            m, live = w.sum(2), live.view(Hkv, G).all(1)
            assert ((mass[b, :, :n].double() - m)[live].abs() <= (2 * dw + 200 * U) * m[live] + 1e-37).all()
            assert (mass[b, :, n:] == 0).all()
    finally:
        cache.close()


@pytest.mark.parametrize("with_mass", [False, True])
@pytest.mark.parametrize("n,Hq", [(100, 4), (700, 4), (700, 64), (3000, 4)])
def test_a_replay_after_the_cache_has_grown_leaves_the_handle_sound(n, Hq, with_mass):
    """A decode recorded at n tokens and replayed at 40000, which its contract rules out: nothing waits for splits that the recorded launch does
    not have, and later calls give what they gave before."""
    Hkv, d, cap = 2, 64, 40000
    g = np.random.default_rng(n)
    K, V = draw(g, Hkv, cap, d, dtype=wl.F16), draw(g, Hkv, cap, d, dtype=wl.F16)
    q = draw(g, 1, Hq, d, dtype=wl.F16)
    cache = ta.TopkAttnCache(1, 1, Hq, Hkv, d, cap, 8, wl.F16)
    try:
        up = lambda x: H.to_torch(np.ascontiguousarray(x), wl.F16, DEV)
        cache.append(0, 0, up(K[:, :n]), up(V[:, :n]), head_major=True)
        qt = up(q)
        mass = torch.zeros((1, Hkv, cap), device=DEV) if with_mass else None
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            first = cache.decode_dense(0, qt, mass=mass)[0]
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got, got_lse = cache.decode_dense(0, qt, mass=mass)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, first)
        cache.append(0, 0, up(K[:, n:]), up(V[:, n:]), head_major=True)
        want, want_lse = cache.decode_dense(0, qt)
        for _ in range(3):
            graph.replay()
            torch.cuda.synchronize()
            assert (got - want).abs().max() < 1e-4 and (got_lse - want_lse).abs().max() < 1e-4
            again, again_lse = cache.decode_dense(0, qt)
            assert torch.equal(again, want) and torch.equal(again_lse, want_lse)
        counted = torch.zeros((1, Hkv, cap), device=DEV)
        cache.decode_dense(0, qt, mass=counted)
        assert abs(counted.sum().item() - Hq) < 1e-2
    finally:
        cache.close()


def test_static_scratch_does_not_count_what_only_the_block_decode_uses():
    """The top-k decode through the built-in scratch, on a handle whose workspace exceeds it by the block index's page scores and lists alone."""
    Hq, Hkv, d, k = 1, 1, 32, 64
    limit = 96 << 20
    cfg = lambda cap, index: ta.make_config(1, 1, Hq, Hkv, d, cap, k, ta.F16, index_kind=index)
    lo, hi = 1 << 10, 1 << 26
    while hi - lo > 1:                                            # the longest cache that fits without a block index
        mid = (lo + hi) // 2
        lo, hi = (mid, hi) if ta.topk_attn_workspace_bytes(cfg(mid, ta.INDEX_NONE)) - 512 <= limit else (lo, mid)
    assert ta.topk_attn_workspace_bytes(cfg(lo, ta.INDEX_BOXES)) - 512 > limit
    cache = ta.TopkAttnCache(1, 1, Hq, Hkv, d, lo, k, wl.F16, index_kind=ta.INDEX_BOXES)
    try:
        g = np.random.default_rng(1)
        kv = H.to_torch(draw(g, Hkv, 5000, d, dtype=wl.F16), wl.F16, DEV)
        cache.append(0, 0, kv, kv, head_major=True)
        q = H.to_torch(draw(g, 1, Hq, d, dtype=wl.F16), wl.F16, DEV)
        want = cache.decode(0, q, k)[0]
        out = torch.empty_like(want)
        st = torch.cuda.current_stream().cuda_stream
        assert ta.lib().topk_attn_decode_static(cache.h, 0, q.data_ptr(), k, out.data_ptr(), None, None, None, st) == ta.OK
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    finally:
        cache.close()


@pytest.mark.parametrize("size", [1e25, 3e38, 1e-22, 1e-30, 1e-37])
@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
def test_norms_of_rows_whose_squares_leave_32_bits(dtype, size):
    """Rows of very large and very small numbers, without and with an eps of their own size: normalised as the formula says."""
    Hq, Hkv, d, n = 4, 2, 64, 5
    g = np.random.default_rng(11)
    x = wl.quantize((size * g.uniform(-1, 1, (1, n, Hq + 2 * Hkv, d))).astype(np.float32), dtype)
    w = wl.quantize(g.uniform(0.5, 2.0, d).astype(np.float32), dtype)
    freq = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    t, wt = H.to_torch(x, dtype, DEV), H.to_torch(w, dtype, DEV)
    half_step = {wl.F32: 2.0 ** -24, wl.BF16: 2.0 ** -8}[dtype]
    for eps in (0.0, 1e-40, 1e-6):
        cache = ta.TopkAttnCache(1, 1, Hq, Hkv, d, n, 8, dtype)
        try:
            out = cache.append_rotary(0, t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:], torch.from_numpy(freq).to(DEV), q_norm=wt,
                                      k_norm=wt, eps=eps)
            want = ref.rms_rotate(wl.widen(x[0, :, :Hq], dtype), wl.widen(w, dtype), np.float32(eps), np.arange(n), freq, False)
            got = out[0].double().cpu().numpy()
            # as for ordinary rows (the norm's sum, root, quotient and products, the turn), and half a step of the smallest numbers of 32 bits
            r = np.sqrt(want ** 2 + np.abs(want).max(-1, keepdims=True) ** 2)
            tol = (d / 2 + 24) * U * r + half_step * np.abs(want) * 1.01 + 2.0 ** -126
            assert (np.abs(got - want) <= tol).all(), f"eps {eps}: off by {np.abs(got - want).max():.3g} of {np.abs(want).max():.3g}"
        finally:
            cache.close()


@pytest.mark.parametrize("dtype", TYPES)
def test_every_weight_to_its_last_bits(dtype):
    """64 keys of exact scores, the value of key c one in channel c: the outputs are the weights themselves."""
    d, n, Hq = 64, 64, 4
    q1, k1 = ob.grid_scores(np.random.default_rng(0), Hq, n)
    q, K = np.zeros((1, Hq, d), np.float32), np.zeros((1, n, d), np.float32)
    q[0, :, 0], K[0, :, 0] = q1, k1
    cache = filled(wl.quantize(K, dtype), wl.quantize(np.eye(n, d, dtype=np.float32)[None], dtype), dtype, Hq)
    try:
        out, _ = cache.decode_dense(0, H.to_torch(wl.quantize(q, dtype), dtype, DEV))
        w = np.exp(q1[:, None].astype(np.float64) * k1 / np.sqrt(d))
        want = w / w.sum(1, keepdims=True)
        # additions of a sum: three in a step, one to the steps before, two of lanes, four of waves
        off = (np.abs(out[0].double().cpu().numpy() - want) / want).max()
        assert off <= ob.quotient_bound(dtype, 10), f"off by {off:.3g}, {ob.quotient_bound(dtype, 10):.3g} allowed"
    finally:
        cache.close()


@pytest.mark.parametrize("dtype,n,blocks", [(wl.F16, 70001, 0), (wl.BF16, 40007, 0), (wl.F32, 30001, 0), (wl.F16, 700, 0), (wl.BF16, 700, 11),
                                            (wl.F32, 130, 0), (wl.F16, 30001, 200), (wl.F32, 20003, 150)])
def test_every_stretch_of_the_cache_shows(dtype, n, blocks):
    """The values of each 64th of the cache are one in a channel of its own: a stretch that is lost, counted twice or joined with another one's
    factor shows in that channel."""
    d, Hq, Hkv = 64, 8, 2
    g = np.random.default_rng(n)
    q, K, V = np.zeros((1, Hq, d), np.float32), np.zeros((Hkv, n, d), np.float32), np.zeros((Hkv, n, d), np.float32)
    part = np.arange(n) * d // n
    V[:, np.arange(n), part] = 1.0
    k1 = []
    for h in range(Hkv):
        q[0, 4 * h:4 * h + 4, 0], k = ob.grid_scores(g, 4, n)
        K[h, :, 0] = k
        k1.append(k.astype(np.float64))
    cache = filled(wl.quantize(K, dtype), wl.quantize(V, dtype), dtype, Hq, ta.INDEX_BOXES if blocks else ta.INDEX_NONE)
    try:
        qt = H.to_torch(wl.quantize(q, dtype), dtype, DEV)
        at = [np.arange(n)] * Hkv
        if blocks:
            out, pages, _ = cache.decode_blocks(0, qt, blocks)
            at = ref.block_tokens([[p for p in x if p >= 0] for x in pages[0].cpu().numpy()], n)
        else:
            out, _ = cache.decode_dense(0, qt)
        out = out[0].double().cpu().numpy()
        # (16 steps of a wave at most here, each up to 8 roundings of each of three parts' sums; 64 splits in each of four sums, and the join)
        bound = ob.quotient_bound(dtype, 16 * 24 + 64 + 10)
        for h in range(Hq):
            w = np.exp(q[0, h, 0] * k1[h // 4][at[h // 4]] / np.sqrt(d))
            want = np.bincount(part[at[h // 4]], w, minlength=d) / w.sum()
            assert (np.abs(out[h] - want) <= bound * want).all(), f"head {h}: off by {(np.abs(out[h] - want) / want.clip(1e-9)).max():.3g}"
    finally:
        cache.close()
