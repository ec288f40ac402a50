// Attention of one query per sequence and head over all cached tokens, or over a list of 64-token pages (topk_attn_decode_dense and
// the last step of topk_attn_decode_blocks): out = sum_i p_i V_i / sum_i p_i with p_i = exp(q . K_i / sqrt(d)), in one pass over K and V.
//
//   attend_kernel       splits of a sequence, a workgroup each: running maximum, sum of weights and weighted value sum, per wave; the
//                       last workgroup of a key stream to finish puts the splits together
//   attend_later_kernel with `mass`: the splits put together there, and the weights of the keys added up; also for many splits of many heads
//
// Bound by the read of K and V: 16 384 bytes per 32 keys and KV head against 24 (fp16) or 32 (bf16) MFMA (d = 128), a tenth of the time the read takes.
// A million tokens, 8 KV heads: 716 us (6.0 TB/s; plain reads reach 6.0 to 6.1); 128k tokens 94 us a call; 500 tokens 8.8 us, all latency.
#include "device_utils.h"
#include "internal.h"
#include "ops.h"
#include "scan_tiles.h"

namespace tka {

// A step of the walk: STEP keys against 16 heads.  The products are taken transposed (keys x channels times channels x heads, then
// channels x keys times keys x heads), so that a lane holds scores and weighted sums of one head, lane % 16, and the running maximum
// is a number per lane.  The scores come out of the first product in lane (j, head) for keys 4 j .. 4 j + 3 of each 16-key tile; the
// second product takes its keys in that same order, so the weights are its operand as they are.
template <int DT, int D> struct AttendTile {
    static constexpr int SUB = DT == DT_F32 ? 1 : 2;             // 16-key tiles of a step: one contraction of the second product
    static constexpr int STEP = 16 * SUB, KEYS = 4 * SUB;        // keys of a step, and those whose values a lane holds
    static constexpr int ROW = D * Elem<DT>::kBytes;
    static constexpr int KCH = ROW / 64;                         // 16-byte pieces of a key row per lane
    static constexpr int VLOAD = ROW / 16 < 16 ? ROW / 16 : 16;  // bytes of a value row a lane loads at a time
    static constexpr int VQ = ROW / 16 / VLOAD;                  // such loads
    static constexpr int EV = VLOAD / Elem<DT>::kBytes;          // channels of a load
    static constexpr int T = D / 16;                             // 16-channel tiles
    // channel of row m of tile t
    static __device__ __forceinline__ constexpr int channel(int t, int m) { return ((t / EV) * 16 + m) * EV + t % EV; }
    static constexpr bool kPipelined = ROW <= 256 || (DT == DT_F32 && ROW <= 512);
    u32x4 k[SUB][KCH];
    uint32_t v[KEYS][VQ * VLOAD / 4];
};

template <int BYTES>
__device__ __forceinline__ void buffer_read(const __amdgpu_buffer_rsrc_t rsrc, int off, uint32_t* to) {
    if constexpr (BYTES == 16) {
        const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, 0, 0);
        to[0] = x.x; to[1] = x.y; to[2] = x.z; to[3] = x.w;
    } else if constexpr (BYTES == 8) {
        const auto x = __builtin_amdgcn_raw_buffer_load_b64(rsrc, off, 0, 0);
        to[0] = x[0]; to[1] = x[1];
    } else {
        to[0] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, off, 0, 0);
    }
}

__device__ __forceinline__ float max_over_rows(float v) {      // largest of lanes l, l ^ 16, l ^ 32, l ^ 48
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Weights of 16-bit caches are the operand of an MFMA and go in as parts, each the rounding to the type of what the ones before it left: two of
// fp16 (to 2^-22 of a weight, half of what the rounding of its exponent leaves) and three of bf16 (to 2^-24).  (One part of fp16 alone: 2^-11 of a
// weight; two of bf16: 2^-16; bf16's third costs nothing that shows: the MFMA of a step take a tenth of the time its rows do.)
// fp16 has no numbers below 2^-24, so there the weights are relative to the maximum less 13 powers of two: one below 2^-16 of the maximum is off by
// 2^-38 of that at most.
template <int DT> struct WeightShift { static constexpr float value = DT == DT_F16 ? 13.f : 0.f; };

constexpr int kFold = 64;        // steps of a wave whose sums follow each other

// Pages of a sequence of N tokens that are attended, and their splits: no more than the launch has.  (A recorded call may be replayed after the
// sequence has grown, though its contract says otherwise: the last split then takes what there is, and the splits that are waited for are
// those that come.)
__device__ __forceinline__ int64_t attend_pages(const AttendCall& a, int64_t N) {
    const int64_t pages = (N + 63) / 64;
    return a.list && a.n_list < pages ? a.n_list : pages;
}
__device__ __forceinline__ int attend_splits(const AttendCall& a, int64_t pages) {
    const int64_t splits = (pages + a.chunk - 1) / a.chunk;
    return (int)(splits < a.n_split ? splits : a.n_split);
}
// What the splits leave is read by a workgroup of the same launch, maybe on another XCD: written and read past the caches that are not shared.
__device__ __forceinline__ void put(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float2 get2(const float* p) {
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
// log2 of the sum of a head's weights (not shifted), over its splits; one wave.  `f` (or null) gets the factor of each split's weighted sum.
__device__ __forceinline__ float head_log2_sum(const AttendCall& a, int64_t bh, int n_split, float shift, float* f) {
    const float* lm = a.part_lm + bh * a.n_split * 2;
    constexpr int U = kMaxSplits / kWave;
    float2 v[U];
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = u * kWave + lane_id();
        v[u] = make_float2(0.f, -INFINITY);
        if (u * kWave < n_split && i < n_split) v[u] = get2(lm + 2 * i);
        top = fmaxf(top, v[u].y);
    }
    top = wave_max(top);
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        v[u].y = v[u].y == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(v[u].y - top);     // (nothing but -inf: no part in the sum)
        if (v[u].y != 0.f) sum = fmaf(v[u].y, v[u].x, sum);
    }
    sum = group_reduce<AddOp, 64>(sum);
    const float inv = 1.0f / sum;
    if (f) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * kWave + lane_id() < n_split) f[u * kWave + lane_id()] = v[u].y * inv;
    }
    return (top - shift) + log2f(sum);
}
// Weighted sum of the splits of `quads` groups of four channels.  Four sums, by split modulo four, whichever thread takes them: the result does
// not depend on how many heads are joined at a time.
template <int NT, int SHARES>
__device__ __forceinline__ void sum_splits(const AttendCall& a, int64_t head0, int quads, int n_split, const float* f, f32x4* part) {
    constexpr int U = 16, SUMS = 4 / SHARES;                       // splits in flight (a trip to memory each otherwise); sums of a thread
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc(a.part_acc + head0 * a.n_split * a.D, 0, 16 * a.n_split * a.D * 4, 0x00020000);
    const int quarter = a.D / 4, first = SHARES > 1 ? (int)threadIdx.x / quads : 0;
    for (int i = SHARES > 1 ? (int)threadIdx.x % quads : (int)threadIdx.x; i < quads && first < SHARES; i += NT) {
        const int h = i / quarter, c = 4 * (i - h * quarter);
        const float* const fh = f + h * n_split;
        const uint32_t off = (uint32_t)(h * a.n_split * a.D + c) * 4;
        f32x4 sum[SUMS] = {};
        for (int x0 = first; x0 < n_split; x0 += U * SHARES) {
            f32x4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {                          // (sc1: past the L2 of this XCD)
                const int x = x0 + u * SHARES < n_split ? x0 + u * SHARES : x0;
                v[u] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(off + (uint32_t)(x * a.D) * 4), 0, 16));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float w = x0 + u * SHARES < n_split ? fh[x0 + u * SHARES] : 0.f;
                if (w != 0.f) {                                     // (a split of nothing but -inf may hold anything)
#pragma unroll
                    for (int y = 0; y < 4; ++y) sum[u % SUMS][y] = fmaf(w, v[u][y], sum[u % SUMS][y]);
                }
            }
        }
        if (SHARES > 1) {
#pragma unroll
            for (int y = 0; y < SUMS; ++y) part[(first + y * SHARES) * quads + i] = sum[y];
        } else {
#pragma unroll
            for (int y = 0; y < 4; ++y) a.out[(head0 + h) * a.D + c + y] = (sum[0][y] + sum[1 % SUMS][y]) + (sum[2 % SUMS][y] + sum[3 % SUMS][y]);
        }
    }
    if (SHARES > 1) {
        __syncthreads();
        if ((int)threadIdx.x < quads) {
            const f32x4* q = part + threadIdx.x;
            const f32x4 sum = (q[0] + q[quads]) + (q[2 * quads] + q[3 * quads]);
            float* out = a.out + (head0 + (int)threadIdx.x / quarter) * a.D + 4 * ((int)threadIdx.x % quarter);
#pragma unroll
            for (int y = 0; y < 4; ++y) out[y] = sum[y];
        }
    }
}
// out and lse of `heads` neighbouring heads (at most 16) from their splits; a workgroup of NT threads, f: [heads][n_split] in LDS.
template <int NT>
__device__ __forceinline__ void join_splits(const AttendCall& a, int64_t head0, int heads, int n_split, float shift, float* f, f32x4* part) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    for (int h = wave; h < heads; h += NT / kWave) {
        const float lg2 = head_log2_sum(a, head0 + h, n_split, shift, f + h * n_split);
        if (lane_id() == 0 && a.lse) a.lse[head0 + h] = lg2 * 0.69314718055994531f;
    }
    __syncthreads();
    // Four channels a thread; with few of them two or four threads share a group's splits.
    const int quads = heads * (a.D / 4);
    if (quads <= NT / 4) sum_splits<NT, 4>(a, head0, quads, n_split, f, part);
    else if (quads <= NT / 2) sum_splits<NT, 2>(a, head0, quads, n_split, f, part);
    else sum_splits<NT, 1>(a, head0, quads, n_split, f, part);
}

// FOLD: for splits of more than kFold steps a wave.  (Shorter ones without the code for it, which takes registers: 32 sequences of 800 to 16384
// tokens of d = 64 with mass 167 us, 176 with it.)
template <int DT, int D, bool LIST, bool MASS, bool FOLD>
__global__ void __launch_bounds__(256, (AttendTile<DT, D>::ROW <= 512 ? 2 : 1)) attend_kernel(AttendCall a) {
    using Tile = AttendTile<DT, D>;
    constexpr int SUB = Tile::SUB, STEP = Tile::STEP, KEYS = Tile::KEYS, KCH = Tile::KCH, T = Tile::T, ROW = Tile::ROW, EV = Tile::EV;
    constexpr int SPP = 64 / STEP;
    constexpr int NW = 4, NT = NW * kWave, RED = NW * 16 * (D + 4), JOIN = 16 * kMaxSplits + 8 * NT;
    __shared__ __align__(16) float lds[RED > JOIN ? RED : JOIN];
    float (*const red)[16][D + 4] = reinterpret_cast<float (*)[16][D + 4]>(lds);
    __shared__ float red_m[NW][16], red_l[NW][16], kept_m[NW][kWave], kept_l[NW][kWave];
    __shared__ uint32_t arrived;
    const int lane = lane_id(), j = lane >> 4, n = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    // The head blocks of one split follow each other eight workgroups apart: on the same XCD, whose L2 holds the keys for them.
    int unit = (int)blockIdx.x, rb = 0;
    if (a.row_blocks > 1) {
        const int group = unit / (8 * a.row_blocks), in = unit - group * 8 * a.row_blocks;
        rb = in >> 3;
        unit = group * 8 + (in & 7);
    }
    // Splits of one rank follow each other, stream after stream, beginning a stream later with each rank.  (Workgroups go to the XCDs in turn:
    // with the splits of a stream next to each other, eight or sixteen of them, each XCD had the same ranks of all sequences, and those of the
    // last ranks, which short sequences do not have, stood idle: 24 sequences of 400 to 8192
    // tokens in splits of 8 pages 124 us, now 92.)
    const int streams = a.B * a.Hkv, split = unit / streams;
    if (split >= a.n_split) return;                           // (the last group of eight may be cut short)
    int stream = unit - split * streams - split % streams;
    if (stream < 0) stream += streams;
    const int b = stream / a.Hkv, kvh = stream - b * a.Hkv;
    const int64_t N = a.len[b];
    const int64_t pages = attend_pages(a, N);
    const int ns = attend_splits(a, pages);
    if (split >= ns) return;                                  // (the join knows how many splits a sequence has)
    const int64_t p0 = (int64_t)split * a.chunk, p1 = split + 1 < ns ? p0 + a.chunk : pages;
    const int n_steps = (int)(p1 - p0) * SPP;
    const int heads = a.G - 16 * rb < 16 ? a.G - 16 * rb : 16;
    const int64_t head0 = (int64_t)b * a.Hq + (int64_t)kvh * a.G + 16 * rb;
    const char* const Kh = a.K + (int64_t)stream * a.Ncap * ROW;
    const char* const Vh = a.V + (int64_t)stream * a.Ncap * ROW;
    const int32_t* const list = LIST ? a.list + (int64_t)stream * a.list_stride + p0 : nullptr;

    // queries: lane (j, head) holds the channels its lane (j, key) holds of a key row
    u32x4 q[KCH];
    {
        const char* p = static_cast<const char*>(a.q) + (head0 + (n < heads ? n : 0)) * ROW + j * 16;
#pragma unroll
        for (int s = 0; s < KCH; ++s) {
            q[s] = *reinterpret_cast<const u32x4*>(p + 64 * s);
            if (n >= heads) q[s] = u32x4{0, 0, 0, 0};
        }
    }
    uint32_t k_off[SUB], v_off[SUB];
#pragma unroll
    for (int g = 0; g < SUB; ++g) {
        k_off[g] = (uint32_t)((16 * g + n) * ROW + j * 16);
        v_off[g] = (uint32_t)((16 * g + 4 * j) * ROW + n * Tile::VLOAD);
        asm volatile("" : "+v"(k_off[g]), "+v"(v_off[g]));
    }
    uint32_t pages_ahead = 0;                                 // LIST: lane i holds the page of the wave's step i (of the next 64)
    // First row of the wave's step i (steps wave, wave + NW, ... of the split), asked for in order.
    auto row_of = [&](int i) -> int64_t {
        const int s = wave + NW * i;
        if (!LIST) return p0 * 64 + (int64_t)s * STEP;
        if ((i & 63) == 0) {
            const int at = wave + NW * (i + lane);
            pages_ahead = (uint32_t)list[at < n_steps ? at / SPP : 0];
        }
        const uint32_t page = (uint32_t)__builtin_amdgcn_readlane((int)pages_ahead, i & 63);
        return (int64_t)page * 64 + (s % SPP) * STEP;
    };
    auto rows_from = [&](int64_t row0, bool live) -> int {      // rows of the step that the cache holds
        const int64_t left = live ? N - row0 : 0;
        int r = (int)(left < 0 ? 0 : left > STEP ? STEP : left);
        r = __builtin_amdgcn_readfirstlane(r);
        asm("" : "+s"(r));
        return r;
    };
    auto load = [&](Tile& t, int i, int& rows) {
        const int64_t row0 = row_of(i);
        rows = rows_from(row0, wave + NW * i < n_steps);
        // what lies behind the rows there are reads as zero and is not fetched: no weight of zero meets a value of infinity
        const int64_t at = rows > 0 ? row0 * ROW : 0;
        const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(Kh + at), 0, rows * ROW, 0x00020000);
        const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(Vh + at), 0, rows * ROW, 0x00020000);
#pragma unroll
        for (int g = 0; g < SUB; ++g) {
#pragma unroll
            for (int s = 0; s < KCH; ++s) t.k[g][s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, (int)k_off[g] + 64 * s, 0, 0));
        }
#pragma unroll
        for (int e = 0; e < KEYS; ++e) {
#pragma unroll
            for (int c = 0; c < Tile::VQ; ++c)
                buffer_read<Tile::VLOAD>(rv, (int)v_off[e / 4] + (e % 4) * ROW + 256 * c, &t.v[e][c * (Tile::VLOAD / 4)]);
        }
    };
    f32x4 acc[T];
#pragma unroll
    for (int t = 0; t < T; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;                              // (m: raw score times scale; l: this lane's keys)
    auto use = [&](const Tile& t, int i, int rows) {
        f32x4 s[SUB];
#pragma unroll
        for (int g = 0; g < SUB; ++g) {
            s[g] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (DT == DT_F32) {
                // four sums of a quarter of the channels each: shorter chains, whose roundings are what a score's error is
                f32x4 part[4] = {};
#pragma unroll
                for (int c = 0; c < KCH; ++c) {
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        part[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.k[g][c][x]), __uint_as_float(q[c][x]), part[x], 0, 0, 0);
                }
                s[g] = (part[0] + part[1]) + (part[2] + part[3]);
            } else {
                using v8 = typename Mfma<DT>::v8;
#pragma unroll
                for (int c = 0; c < KCH; ++c) s[g] = Mfma<DT>::mac(__builtin_bit_cast(v8, t.k[g][c]), __builtin_bit_cast(v8, q[c]), s[g]);
            }
        }
        if (MASS) {
            // kept in the order of the walk; a head's four scores of neighbouring keys in one store
            float* to = a.scores + (head0 + n) * a.score_stride + p0 * 64 + (int64_t)(wave + NW * i) * STEP + 4 * j;
#pragma unroll
            for (int g = 0; g < SUB; ++g) {
                if (n < heads) {
                    if (16 * g + 4 * j + 3 < rows) {
                        __builtin_memcpy(to + 16 * g, &s[g], 16);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (16 * g + 4 * j + r < rows) to[16 * g + r] = s[g][r];
                    }
                }
            }
        }
        float p[KEYS];
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < KEYS; ++e) {
            p[e] = s[e / 4][e % 4];
            if (rows < STEP && 16 * (e / 4) + 4 * j + e % 4 >= rows) p[e] = -INFINITY;
            top = fmaxf(top, p[e]);
        }
        const float m_new = fmaxf(m, max_over_rows(top) * a.scale_log2e);
        const float ref = (m_new == -INFINITY ? 0.f : m_new) - WeightShift<DT>::value;      // (nothing but -inf so far: weights of zero)
        const float alpha = __builtin_amdgcn_exp2f(m - (m_new == -INFINITY ? 0.f : m_new));
        m = m_new;
#pragma unroll
        for (int e = 0; e < KEYS; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(p[e], a.scale_log2e, -ref));
        float step = (p[0] + p[1]) + (p[2] + p[3]);
        if constexpr (KEYS == 8) step += (p[4] + p[5]) + (p[6] + p[7]);
        l = fmaf(l, alpha, step);
#pragma unroll
        for (int c = 0; c < T; ++c) {
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[c][r] *= alpha;
        }
        if constexpr (DT == DT_F32) {
#pragma unroll
            for (int c = 0; c < T; ++c) {
#pragma unroll
                for (int e = 0; e < KEYS; ++e) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[e][c]), p[e], acc[c], 0, 0, 0);
            }
        } else {
            using v8 = typename Mfma<DT>::v8;
            constexpr int PARTS = DT == DT_F16 ? 2 : 3;
            v8 part[PARTS];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float rest = p[e];
#pragma unroll
                for (int x = 0; x < PARTS; ++x) {
                    part[x][e] = (decltype(+part[x][0]))rest;
                    rest -= (float)part[x][e];
                }
            }
#pragma unroll
            for (int c = 0; c < T; ++c) {
                // channel column of the lane's eight keys: pairs of rows, one 16-bit half each
                const int w = (c / EV) * (Tile::VLOAD / 4) + (c % EV) / 2;
                const uint32_t half = c % 2 ? 0x07060302u : 0x05040100u;
                u32x4 col;
#pragma unroll
                for (int x = 0; x < 4; ++x) col[x] = __builtin_amdgcn_perm(t.v[2 * x + 1][w], t.v[2 * x][w], half);
#pragma unroll
                for (int x = 0; x < PARTS; ++x) acc[c] = Mfma<DT>::mac(__builtin_bit_cast(v8, col), part[x], acc[c]);
            }
        }
    };
    // Every kFold steps the sums so far are put aside (the weighted one in LDS), and begin again: 32 bits that grow without end round every small
    // weight the same way (131072 tokens in one split, equal weights below one: 3.1e-5 of their sum before).  A maximum of -inf is the
    // beginning: the next step's alpha is zero.
    auto fold = [&](bool first) {
        int at = lane_id();
        asm volatile("" : "+v"(at));                           // (addresses worked out here, not kept in registers along the walk)
        const float m_before = first ? -INFINITY : kept_m[wave][at], l_before = first ? 0.f : kept_l[wave][at];
        const float top = fmaxf(m_before, m), ref = top == -INFINITY ? 0.f : top;
        const float f = __builtin_amdgcn_exp2f(m_before - ref), f_now = __builtin_amdgcn_exp2f(m - ref);
        kept_m[wave][at] = top;
        kept_l[wave][at] = fmaf(l_before, f, l * f_now);
#pragma unroll
        for (int c = 0; c < T; ++c) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float& x = red[wave][at & 15][Tile::channel(c, 4 * (at >> 4) + r)];
                x = first ? acc[c][r] * f_now : fmaf(x, f, acc[c][r] * f_now);
            }
            __builtin_amdgcn_sched_barrier(0);                 // (four registers at a time)
        }
        m = -INFINITY;
    };
    const int mine = n_steps > wave ? (n_steps - wave + NW - 1) / NW : 0;
    if constexpr (Tile::kPipelined) {
        Tile ta, tb;
        int ra = 0, rb_ = 0;
        if (mine > 0) load(ta, 0, ra);
        for (int i = 0; i < mine; i += 2) {
            load(tb, i + 1, rb_);
            __builtin_amdgcn_sched_barrier(0);
            use(ta, i, ra);
            if (i + 1 >= mine) break;
            load(ta, i + 2, ra);
            __builtin_amdgcn_sched_barrier(0);
            use(tb, i + 1, rb_);
            if (FOLD && (i + 2) % kFold == 0) fold(i + 2 == kFold);
        }
    } else {
        Tile t;
        int r = 0;
        for (int i = 0; i < mine; ++i) {
            load(t, i, r);
            __builtin_amdgcn_sched_barrier(0);
            use(t, i, r);
            if (FOLD && (i + 1) % kFold == 0) fold(i + 1 == kFold);
        }
    }
    if (FOLD && mine >= kFold) {
        fold(false);
        m = kept_m[wave][lane];
        l = kept_l[wave][lane];
    } else {
#pragma unroll
        for (int c = 0; c < T; ++c) {
#pragma unroll
            for (int r = 0; r < 4; ++r) red[wave][n][Tile::channel(c, 4 * j + r)] = acc[c][r];
        }
    }
    l = add_lanes_32(add_lanes_16(l));
    // A maximum passes over NaN: a wave of nothing but NaN and -inf would count as one without a key.  With a maximum of +inf its factor is NaN, here
    // and where splits are joined.
    if (l != l) m = INFINITY;
    // the waves' sums, relative to the largest of their maxima
    if (j == 0) { red_m[wave][n] = m; red_l[wave][n] = l; }
    __syncthreads();
    const bool whole = a.join_later ? a.n_split == 1 : ns == 1;        // the sequence's only split (a later join does all or none)
    for (int i = (int)threadIdx.x; i < heads * D; i += NT) {
        const int h = i / D, c = i - h * D;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, red_m[w][h]);
        float sum = 0.f, total = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = red_m[w][h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(red_m[w][h] - top);
            if (f != 0.f) { sum = fmaf(f, red[w][h][c], sum); total = fmaf(f, red_l[w][h], total); }
        }
        const int64_t bh = head0 + h;
        if (whole) {
            a.out[bh * D + c] = sum * (1.0f / total);              // (as join_splits() has it)
            if (c == 0 && a.lse) a.lse[bh] = ((top - WeightShift<DT>::value) + log2f(total)) * 0.69314718055994531f;
        } else {
            put(&a.part_acc[(bh * a.n_split + split) * D + c], sum);
        }
        if (c == 0 && (MASS || !whole)) {
            put(&a.part_lm[(bh * a.n_split + split) * 2], total);
            put(&a.part_lm[(bh * a.n_split + split) * 2 + 1], top);
        }
    }
    if (a.join_later || whole) return;
    // the last split of the stream's head block to get here joins them (and leaves the counter at zero for the next call)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    uint32_t* const counter = a.arrive + (int64_t)stream * a.row_blocks + rb;
    if (threadIdx.x == 0) arrived = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (arrived + 1u != (uint32_t)ns) return;
    if (threadIdx.x == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    join_splits<NT>(a, head0, heads, ns, WeightShift<DT>::value, lds, reinterpret_cast<f32x4*>(lds + 16 * kMaxSplits));
}

// The first workgroups put a head's, or a block of heads', splits together; the others add each key's weights, the heads of the group in order, from the
// scores that the walk left: 4 bytes per key and head written and read, where a second walk over the keys reads 2 d / G.
// 24 sequences of 400 to 8192 tokens, 64 heads over 8: 16 us beside the walk's 100.
__global__ void __launch_bounds__(256) attend_later_kernel(AttendCall a, float shift, int n_join) {
    __shared__ float lg[128];
    __shared__ float f[16 * kMaxSplits];
    __shared__ f32x4 sums[512];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if ((int)blockIdx.x < n_join) {
        const int blocks = a.join_heads == 1 ? a.G : a.row_blocks, group = (int)blockIdx.x / blocks, in = (int)blockIdx.x - group * blocks;
        const int left = a.G - in * a.join_heads, heads = left < a.join_heads ? left : a.join_heads;
        join_splits<256>(a, (int64_t)group * a.G + in * a.join_heads, heads, attend_splits(a, attend_pages(a, a.len[group / a.Hkv])), shift, f, sums);
        return;
    }
    const int per_stream = (int)((a.walk + kMassPerBlock - 1) / kMassPerBlock);
    const int stream = ((int)blockIdx.x - n_join) / per_stream, part = ((int)blockIdx.x - n_join) - stream * per_stream;
    const int b = stream / a.Hkv, kvh = stream - b * a.Hkv;
    const int64_t N = a.len[b];
    const int64_t i0 = (int64_t)part * kMassPerBlock;
    const int64_t pages = attend_pages(a, N);
    if (i0 >= pages * 64) return;
    const int64_t head0 = (int64_t)b * a.Hq + (int64_t)kvh * a.G;
    const int ns = attend_splits(a, pages);
    for (int g = wave; g < a.G; g += 4) {
        const float v = head_log2_sum(a, head0 + g, ns, shift, nullptr);
        if (lane_id() == 0) lg[g] = v;
    }
    __syncthreads();
    const float* const s0 = a.scores + head0 * a.score_stride;
    float* const mass = a.mass + (int64_t)stream * a.Ncap;
    // four neighbouring keys a thread (of one page)
    const int64_t at = i0 + 4 * (int)threadIdx.x;
    if (at >= pages * 64) return;
    const int64_t pos = a.list ? (int64_t)a.list[(int64_t)stream * a.list_stride + at / 64] * 64 + at % 64 : at;
    const int left = N - pos < 4 ? (int)(N - pos) : 4;
    if (left <= 0) return;
    float w[4] = {0.f, 0.f, 0.f, 0.f}, old[4];
    if (left == 4) __builtin_memcpy(old, mass + pos, 16);
#pragma unroll 8
    for (int g = 0; g < a.G; ++g) {
        float s[4];
        // (a row's room ends with the cache, which may be within the last four)
        if (left == 4) __builtin_memcpy(s, s0 + g * a.score_stride + at, 16);
        else for (int u = 0; u < 4; ++u) s[u] = u < left ? s0[g * a.score_stride + at + u] : 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] += __builtin_amdgcn_exp2f(fmaf(s[u], a.scale_log2e, -lg[g]));
    }
    if (left == 4) {
#pragma unroll
        for (int u = 0; u < 4; ++u) old[u] += w[u];
        __builtin_memcpy(mass + pos, old, 16);
    } else {
        for (int u = 0; u < left; ++u) mass[pos + u] += w[u];
    }
}

hipError_t launch_attend(const AttendCall& a, hipStream_t st) {
    const int64_t n_join = attend_join_wgs(a), n_mass = attend_mass_wgs(a);
    const bool fold = (int64_t)a.chunk * 64 > (int64_t)kFold * 4 * (a.dtype == DT_F32 ? AttendTile<DT_F32, 32>::STEP : AttendTile<DT_F16, 32>::STEP);
    const dim3 grid((unsigned)attend_walk_wgs(a)), wg(256);
#define TKA_ATTEND_(DT_, D_, LIST_, MASS_)                                                                              \
    do {                                                                                                                \
        if (fold) hipLaunchKernelGGL((attend_kernel<DT_, D_, LIST_, MASS_, true>), grid, wg, 0, st, a);                 \
        else hipLaunchKernelGGL((attend_kernel<DT_, D_, LIST_, MASS_, false>), grid, wg, 0, st, a);                     \
    } while (0)
#define TKA_ATTEND(DT_, D_)                                                                                             \
    do {                                                                                                                \
        if (a.list && a.mass) TKA_ATTEND_(DT_, D_, true, true);                                                         \
        else if (a.list) TKA_ATTEND_(DT_, D_, true, false);                                                             \
        else if (a.mass) TKA_ATTEND_(DT_, D_, false, true);                                                             \
        else TKA_ATTEND_(DT_, D_, false, false);                                                                        \
    } while (0)
    TKA_BY_TYPE_AND_DIM(TKA_ATTEND, a.dtype, a.D);
#undef TKA_ATTEND
#undef TKA_ATTEND_
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || n_join + n_mass == 0) return e;
    hipLaunchKernelGGL(attend_later_kernel, dim3((unsigned)(n_join + n_mass)), dim3(256), 0, st, a, a.dtype == DT_F16 ? 13.f : 0.f, (int)n_join);
    return hipGetLastError();
}

}  // namespace tka
