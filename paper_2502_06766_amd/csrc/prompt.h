// Attention of the last M tokens of a sequence over what each sees (topk_attn_prompt, topk_attn_coded_prompt): the kernel, shared by prompt.hip (caches in
// their own type) and coded_prompt.hip (the 8-bit cache).
//
//   out_m = sum_t w_t V_t / sum_t w_t,  w_t = exp(q_m . K_t / sqrt(d)),  t <= p_m and (t < sinks or t > p_m - window)
//
// A row is a query and a head of the group, m G + g: the heads of a group read the same keys, and a block of rows covers few queries, so little of what
// it computes is masked.  A wave has 32 rows, the workgroup walks the keys in tiles of 64 through LDS.  Products are taken transposed (keys x channels
// times channels x rows, then channels x keys times keys x rows): a lane holds scores and weighted sums of one row, lane % 32, the running maximum is
// a number per lane, and the scores come out of the first product in the order in which the second one takes the weights:
//   score register i of a 32-key tile is key 8 (i / 4) + 4 (lane / 32) + i % 4; step x of 16 keys takes registers 8 x .. 8 x + 7.
// Weights are rounded once to the type of the values (16 bits: what the second product takes; half a step of 2^-8 or 2^-11, as large as that of the output, which is 1.4 times as
// far off with both; what of fp16's range they use: WeightRange); their sum is of the unrounded ones.  Two parts of a weight take 1.4 times as long (the prompt of 8192
// tokens below 751 us).
//
// Bound by the matrix unit, and behind it by the vector instructions of the weights, which only the other wave of a SIMD's products cover.  32 heads over 8, d = 128:
// a prompt of 8192 tokens, bf16, 533 us (1.03 PFLOP/s; a library product of 8192^3 has 1.23, MFMA alone on random numbers 1.5 to 1.8); the last 2048 of 24000 tokens of the 8-bit
// cache 861 (0.90: the codes are widened on the way); eight tokens of four sequences of up to 20000, bf16, 44.7, 34.4 of it this kernel (4.8 TB/s), 5.4 the joint.  16 heads over 4,
// 16001 tokens in a window of 2048, fp16: 313 (0.81).
// Tiles go to LDS in two buffers (16 bits up to d = 128) by loads that pass no register; their reads meet no bank twice.  Two waves a SIMD with 32 rows each, in 16 bits up to
// d = 128, else one: one with 64 spilled.
#pragma once
#include <type_traits>

#include "coded.h"
#include "device_utils.h"
#include "internal.h"

namespace tka {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct PromptCall {
    const char* K;              // rows [S][Hkv][Ncap][D] of the call's first sequence
    const char* V;
    CodedArrays c;              // or the coded cache
    const void* q;              // [S][M][Hq][D]
    void* out;                  // [S][M][Hq][D] in the type of q
    float* lse;                 // [S][M][Hq] or null
    const int32_t* len;         // [S]
    int64_t Ncap, M;
    int64_t sinks, window;
    float* part_acc;            // [S Hkv][row_blocks][n_split][rows of a block][D], where keys are split
    float* part_lm;             // [...][rows of a block][2]
    int S, Hq, Hkv, G, D, dtype, format;
    int n_split, chunk;         // most splits of a row block's keys, tiles of 64 keys in each
    int row_blocks, block_rows;
};
constexpr int kPromptSplits = 64;      // (of 256 their joint takes 1.3 us more)
// Tiles of 64 keys that the rows of the last block, which see most, see of a sequence of N tokens.
inline int64_t prompt_tiles(int64_t N, int64_t last_queries, int64_t sinks, int64_t window) {
    const int64_t before = N - last_queries, from = window < before ? (before - window) / 64 : 0, front = ((sinks < N ? sinks : N) + 63) / 64;
    return (N + 63) / 64 - from + (front < from ? front : from);
}
// Rows of a block, and the splits of its keys, where there are fewer blocks than compute units: runs of `chunk` tiles, as many as there are compute units, twice that where the
// matrix unit has most of the time (512 queries at 32768 tokens, 32 heads over 8: 340 and 291 us).  (room: bytes there are for partial sums.  Eight queries of four
// sequences of 1k to 20k tokens in runs of 6 / 10 / 14 / 20 / 28 / 40 tiles, one of 20 to a compute unit: 65 / 54 / 57 / 45 / 52 / 62 us; in as many runs for every
// sequence, the longest's of 20: 48.  64 queries of one sequence of 20000, 20 tiles to a compute unit: 55 / 47 / 47 / 41 / 48 / 61.  A wave of few rows has
// a tile on its way, 32 KB at d = 128: of fewer channels as many more waves, d = 64, 8 sequences of 16000 tokens 62 and 48.)
inline void plan_prompt(PromptCall* a, const int64_t* len, size_t room, int n_cu) {
    const int64_t rows = a->M * a->G, streams = (int64_t)a->S * a->Hkv;
    a->block_rows = rows <= 32 && a->format < 0 && a->dtype != DT_F32 ? 32 : 128;          // (few rows of 32 bits or the 8-bit cache: dense.hip, coded_decode.hip)
    a->row_blocks = (int)((rows + a->block_rows - 1) / a->block_rows);
    int64_t longest = 1, all = 0;
    for (int b = 0; b < a->S; ++b) {
        const int64_t n = prompt_tiles(len[b], (a->block_rows + a->G - 1) / a->G, a->sinks, a->window);
        longest = n > longest ? n : longest;
        all += n;
    }
    const int64_t wgs = streams * a->row_blocks, want = (rows >= 512 ? 2 : rows <= 32 && a->D < 128 ? 128 / a->D : 1) * n_cu;
    int64_t most = (int64_t)(room / ((size_t)wgs * a->block_rows * (a->D + 2) * sizeof(float)));     // splits
    if (most > kPromptSplits) most = kPromptSplits;
    int64_t chunk = wgs >= n_cu || most < 2 ? longest : (all * a->Hkv * a->row_blocks + want - 1) / want;
    if (chunk < 4) chunk = 4;
    if (most > 1 && chunk < (longest + most - 1) / most) chunk = (longest + most - 1) / most;
    a->chunk = (int)(chunk < longest ? chunk : longest);
    a->n_split = (int)((longest + a->chunk - 1) / a->chunk);
}
inline void place_prompt_parts(PromptCall* a, void* room) {
    a->part_acc = static_cast<float*>(room);
    a->part_lm = a->part_acc + (size_t)a->S * a->Hkv * a->row_blocks * a->n_split * a->block_rows * a->D;
}
// Rows of a key stream up to which tokens of a 32-bit cache go through the walk of single tokens (dense.hip), whose products take 16 rows and whose tiles
// lie in registers; this kernel's take 32, and 64 KB to 256 KB of LDS leave a wave or four to a compute unit.  The two, in us, of 8 / 16 / 32 / 48 / 64 rows:
//   d = 128, 8 KV heads, 30000 tokens           44 / 46 / 54 / 77 / 95       and 140 / 141 / 141 / 203 / 203
//   d = 64, 8 KV heads, 4 sequences of 8000     27 / 29 / 42 / 48 / 72       and 82 / 82 / 82 / 82 / 82
//   d = 256, the same                           100 / 104 / 152 / 235 / 270  and 342 / 342 / 344 / 472 / 473
// 16 bits stay here (d = 128, 24000 tokens, 16 / 32 / 64 rows 25 / 26 / 40 and 25 / 26 / 29; 4 sequences of 1000 to 20000 46 / 50 / 75 and 41 / 41 / 52).
constexpr int kFewRowsF32 = 64;
constexpr int64_t kMostPromptRows = 1 << 30;      // of a stream: counted in 32 bits
hipError_t launch_prompt(const PromptCall& a, hipStream_t st);
hipError_t launch_prompt_coded(const PromptCall& a, hipStream_t st);
hipError_t launch_prompt_join(const PromptCall& a, hipStream_t st);

// ---- tiles in LDS ----
// Rows of 64 keys lie one after the other; the 16-byte pieces of a row change places among each other by its number, so that the lanes that read at a time meet
// all banks: 32 rows at one piece (keys), 8 rows at four neighbouring pieces (values, 16 bits), two rows four apart (values, 32 bits).
template <int ROWB> __device__ __forceinline__ constexpr int key_piece(int row, int piece) {
    constexpr int P = ROWB / 16, L = P < 16 ? P : 16;
    return piece ^ ((row / (16 / L)) % L);
}
template <int ROWB, int EB> __device__ __forceinline__ constexpr int value_piece(int row, int piece) {
    constexpr int P = ROWB / 16;
    if (EB == 4) return P >= 16 ? piece ^ (8 * ((row >> 2) & 1)) : piece;
    return P >= 16 ? piece ^ ((4 * (row & 3)) ^ ((row >> 2) & 3)) : P == 8 ? piece ^ (4 * ((row >> 1) & 1)) : piece;
}

template <int CT> struct TileType;      // what a tile's products are taken in
template <> struct TileType<DT_F16> { using v8 = f16x8; static constexpr int bytes = 2; };
template <> struct TileType<DT_BF16> { using v8 = bf16x8; static constexpr int bytes = 2; };
template <> struct TileType<DT_F32> { static constexpr int bytes = 4; };

__device__ __forceinline__ f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// Queries of a wave's rows as the second operand: 16 bits, 16 channels of a row in eight-channel halves; 32 bits, 8 channels in four-channel halves.
template <int CT, int D, int PQ> struct QueryFrag {
    using type = typename std::conditional<CT == DT_F32, f32x4, typename std::conditional<CT == DT_BF16, bf16x8, f16x8>::type>::type;
    static constexpr int N = CT == DT_F32 ? D / 8 : D / 16;
    type v[PQ][N];
};

template <int D> struct RowState {
    f32x16 acc[D / 32];
    float m, l, e;              // what the weights are relative to (a power of two), their sum, power of two of the weighted sum
    int pos, hidden;            // token of the row; the newest one its window leaves out
};

__device__ __forceinline__ float other_half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Values of a tile for channels 32 ct + lane % 32, the keys of step x: FRAG: laid out as the operand; else rows, read transposed.
template <int D, bool FRAG>
__device__ __forceinline__ u32x4 value_frag(const char* lds, int ct, int x) {
    const int lane = lane_id();
    if (FRAG) return *reinterpret_cast<const u32x4*>(lds + ((x * (D / 32) + ct) * 64 + lane) * 16);
    constexpr int ROWB = 2 * D;
    const int i = lane & 15, hh = lane >> 5, col = 32 * ct + 16 * ((lane >> 4) & 1) + 4 * (i & 3);
    u32x4 r;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        const int row = 16 * x + 8 * y + 4 * hh + (i >> 2);
        const char* p = lds + row * ROWB + value_piece<ROWB, 2>(row, col >> 3) * 16 + (col & 7) * 2;
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
        const uint2 w = __builtin_bit_cast(uint2, v);
        r[2 * y] = w.x; r[2 * y + 1] = w.y;
    }
    return r;
}

// 16-bit halves that are an infinity or a NaN: as ones in their place, and the word without them
template <int CT> __device__ __forceinline__ uint32_t finite_halves(uint32_t w) {
    constexpr uint32_t E = CT == DT_F16 ? 0x7C00u : 0x7F80u;
    uint32_t keep = 0;
    if ((w & E) != E) keep |= 0xFFFFu;
    if (((w >> 16) & E) != E) keep |= 0xFFFF0000u;
    return w & keep;
}
template <int CT> __device__ __forceinline__ bool has_no_number(uint32_t w) {
    if (CT == DT_F32) return (w & 0x7F800000u) == 0x7F800000u;
    return finite_halves<CT>(w) != w;
}

// The maximum that the weights are relative to follows the scores' only when those are more than 2^kSlack above: the weighted sums are scaled seldom
// (scores of a normal distribution, 8192 tokens, 32 rows: after the first tile at none of the others, with 2 powers of slack at ten of 127, with none at 33), and a
// weight stays below 2^kSlack.
constexpr float kSlack = 8.f;
// fp16 has whole steps of its bits down to 2^-14 and nothing below 2^-25, and weights of that size may be many: one key 17 nats above 65536 others is 400 of
// them, and without a shift nothing of those was left.  Weights of fp16 are held times 2^13 with 2 powers of slack, below 2^15: all of the type's bits down to 2^-27 of the
// largest and steps of 2^-37 below, as in the single token's decode.  (8 powers of slack and a shift of 7 would leave steps of 2^-31, 2^-6 of a weight 18 nats below: 8192 tokens,
// 32 heads over 8, d = 128, 590 us against 582.)  Over codes that goes for the product with a block's value scale, relative to a power of two that is up to twice the
// largest: steps of 2^-36 (5 powers and 10 left 2^-33, 0.8 % of weights 18.75 nats below: a prompt of 8192 tokens, int8, bf16, 619 us against 616).
constexpr float kSlack16 = 2.f, kShift16 = 13.f;
template <int CT, bool VSCALE> struct WeightRange {
    static constexpr float slack = CT == DT_F16 && !VSCALE ? kSlack16 : kSlack, shift = CT == DT_F16 && !VSCALE ? kShift16 : 0.f;
};

// Whether some of a lane's words has an infinity or a NaN: the largest magnitudes, two halves at a time.
template <int CT, int N>
__device__ __forceinline__ bool any_no_number(const u32x4 (&w)[N]) {
    if (CT == DT_F32) {
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < N; ++u) {
#pragma unroll
            for (int y = 0; y < 4; ++y) { const uint32_t m = w[u][y] & 0x7FFFFFFFu; top = m > top ? m : top; }
        }
        return top >= 0x7F800000u;
    }
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top = {0, 0};
#pragma unroll
    for (int u = 0; u < N; ++u) {
#pragma unroll
        for (int y = 0; y < 4; ++y) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w[u][y] & 0x7FFF7FFFu));
    }
    constexpr uint16_t E = CT == DT_F16 ? 0x7C00 : 0x7F80;
    return top[0] >= E || top[1] >= E;
}

// One tile of 64 keys from token t0 on.  f (and f_lo, of 32-bit rows): score times this is the exponent of two.  VSCALE: the values are times `sv` (a block's scale),
// the weighted sum has a power of two of its own (coded_decode.hip).  MASKED: not all rows of the workgroup see all keys;
// suspect: some value of the tile is no number.
template <int CT, bool FRAG, bool VSCALE, bool EXACT, bool MASKED, int D, int PQ, int PP>
__device__ __forceinline__ void prompt_tile(const char* ldsK, const char* ldsV, const QueryFrag<CT, D, PQ>& q, RowState<D>& st, float f, float f_lo, float sv,
                                            int t0, int sinks, bool suspect) {
    constexpr int EB = TileType<CT>::bytes, ROWB = D * EB, N = QueryFrag<CT, D, PQ>::N, T = D / 32;
    const int lane = lane_id(), hh = lane >> 5, row = lane & 31;
    f32x16 s[2];
    if constexpr (CT == DT_F32) {
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            s[sub] = f32x16{};
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const u32x4 k = *reinterpret_cast<const u32x4*>(ldsK + (32 * sub + row) * ROWB + key_piece<ROWB>(32 * sub + row, 2 * c + hh) * 16);
#pragma unroll
                for (int y = 0; y < 4; ++y) s[sub] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[y]), q.v[0][c][y], s[sub], 0, 0, 0);
            }
        }
    } else {
        // (all reads of a pass first: a product that waits for its own read stalls the wave for the trip)
        constexpr int PASS = D <= 128 ? 2 : 1;                       // 32-key tiles whose operands are in registers at a time
#pragma unroll
        for (int s0 = 0; s0 < 2; s0 += PASS) {
            u32x4 k[PASS][N];
#pragma unroll
            for (int u = 0; u < PASS; ++u) {
#pragma unroll
                for (int c = 0; c < N; ++c)
                    k[u][c] = *reinterpret_cast<const u32x4*>(ldsK + (32 * (s0 + u) + row) * ROWB + key_piece<ROWB>(32 * (s0 + u) + row, 2 * c + hh) * 16);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < PASS; ++u) {
                s[s0 + u] = f32x16{};
#pragma unroll
                for (int c = 0; c < N; ++c) {
#pragma unroll
                    for (int z = 0; z < PQ; ++z) s[s0 + u] = mfma32(__builtin_bit_cast(typename TileType<CT>::v8, k[u][c]), q.v[z][c], s[s0 + u]);
                }
            }
        }
    }
    u32x4 v[2][T];                                                   // values of the first step: on their way during the weights
    if constexpr (CT != DT_F32) {
#pragma unroll
        for (int ct = 0; ct < T; ++ct) v[0][ct] = value_frag<D, FRAG>(ldsV, ct, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
    // ---- weights, in place of the scores ----
    if (MASKED) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int t = t0 + 32 * (i / 16) + 8 * (i % 16 / 4) + 4 * hh + i % 4;
            if (t > st.pos || (t <= st.hidden && t >= sinks)) s[i / 16][i % 16] = -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = fmaxf(top, s[i / 16][i % 16]);
    top = other_half_max(top);
    const bool none = top == -INFINITY;                              // (also of nothing but NaN: the weights are NaN then)
    // A whole number that the largest exponent is not above, and the product of 32 bits, which from 2^23 on is off by ones, is not below.
    const float product = top * f, bm = none ? -INFINITY : ceilf(product) + floorf(fabsf(product) * 0x1p-23f);
    using Range = WeightRange<CT, VSCALE>;
    const float to = bm - Range::shift, m_new = to > st.m + Range::slack || st.m == -INFINITY ? to : st.m, ref = m_new == -INFINITY ? 0.f : m_new;
    float turn = __builtin_amdgcn_exp2f(st.m - ref), e_new = 0.f;
    int ke = 0;
    st.l *= turn;
    if (VSCALE) {                                                    // (the weighted sum goes by its own)
        ke = (int)(__float_as_uint(sv) >> 23) - 126;                 // sv < 2^ke
        const float e_tile = bm + (float)ke;
        e_new = sv > 0.f && !none && (e_tile > st.e + kSlack16 || st.e == -INFINITY) ? e_tile : st.e;
        turn = st.e == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.e - e_new);
    }
    if (__any(turn != 1.f)) {
#pragma unroll
        for (int ct = 0; ct < T; ++ct) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st.acc[ct][i] *= turn;
        }
    }
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const float x = s[i / 16][i % 16];
        float w = __builtin_amdgcn_exp2f(EXACT ? fmaf(x, f, fmaf(x, f_lo, -ref)) : fmaf(x, f, -ref));
        if (((VSCALE && MASKED) || EXACT) && x == -INFINITY) w = 0.f;  // (a factor of zero, or of two parts)
        s[i / 16][i % 16] = w;
        sum[i & 1] += w;
    }
    st.l += sum[0] + sum[1];
    if (VSCALE) {
        float g = sv;
        if (sv > 0.f) g = ldexpf(sv, (int)fmaxf(fminf(ref - e_new + kShift16, (float)(127 - ke)), -300.f));
        if (none) g = 0.f;                                           // (a block of NaN that the row does not see)
        st.e = e_new;
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i / 16][i % 16] *= g;
    }
    st.m = m_new;
    // ---- values that are no numbers, in a tile that not all rows see ----
    bool poison = false;
    if constexpr (!FRAG && MASKED) {
        uint64_t keys = 0;
        for (int at = 0; suspect && at < 64 * ROWB; at += 1024) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(ldsV + at + lane * 16);
            const uint64_t bad = __ballot(has_no_number<CT>(w.x) || has_no_number<CT>(w.y) || has_no_number<CT>(w.z) || has_no_number<CT>(w.w));
            if (bad) {
                if (ROWB >= 1024) keys |= 1ull << (at / ROWB);
                else
                    for (int y = 0; y < 1024 / ROWB; ++y)
                        if ((bad >> (y * (ROWB / 16))) & (ROWB / 16 == 64 ? ~0ull : (1ull << (ROWB / 16 % 64)) - 1)) keys |= 1ull << (at / ROWB + y);
            }
        }
        poison = keys != 0;
        // such a value goes to the rows that see it, one key at a time; the products below take zero in its place
        while (keys) {
            const int key = __builtin_ctzll(keys);
            keys &= keys - 1;
            const int reg = (key >> 5) * 16 + ((key & 31) >> 3) * 4 + (key & 3), t = t0 + key;
            float p = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i == reg) p = s[i / 16][i % 16];
            p = __shfl(p, row + 32 * ((key >> 2) & 1), 64);
            const bool sees = !(t > st.pos || (t <= st.hidden && t >= sinks));
#pragma unroll
            for (int ct = 0; ct < T; ++ct) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int ch = 32 * ct + 8 * (i / 4) + 4 * hh + i % 4;
                    const char* at = ldsV + key * ROWB + value_piece<ROWB, EB>(key, ch * EB / 16) * 16 + ch * EB % 16;
                    float x;
                    if (CT == DT_F32) x = *reinterpret_cast<const float*>(at);
                    else if (CT == DT_F16) x = (float)*reinterpret_cast<const _Float16*>(at);
                    else x = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(at) << 16);
                    if (sees && !(fabsf(x) < INFINITY)) st.acc[ct][i] = fmaf(p, x, st.acc[ct][i]);
                }
            }
        }
    }
    // ---- weighted sum ----
    if constexpr (CT == DT_F32) {
#pragma unroll
        for (int ct = 0; ct < T; ++ct) {
            f32x16 part = {};                                        // (an addition to the sum so far for a tile, not for every two keys: 2 % of the time)
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int key = 32 * (i / 16) + 8 * (i % 16 / 4) + 4 * hh + i % 4, ch = 32 * ct + row;
                float x = *reinterpret_cast<const float*>(ldsV + key * ROWB + value_piece<ROWB, 4>(key, ch >> 2) * 16 + (ch & 3) * 4);
                if (poison && !(fabsf(x) < INFINITY)) x = 0.f;
                part = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[i / 16][i % 16], part, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) st.acc[ct][i] += part[i];
        }
    } else {
        using v8 = typename TileType<CT>::v8;
        using E = typename std::conditional<CT == DT_F16, _Float16, __bf16>::type;
        v8 p[PP][4];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float rest = s[i / 16][i % 16];
            if (PP > 1) asm("" : "+v"(rest));                        // (not rounded together with the multiplication in front of it: coded_decode.hip)
#pragma unroll
            for (int z = 0; z < PP; ++z) {
                p[z][i / 8][i % 8] = (E)rest;
                rest -= (float)p[z][i / 8][i % 8];
            }
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (x < 3) {
#pragma unroll
                for (int ct = 0; ct < T; ++ct) v[(x + 1) & 1][ct] = value_frag<D, FRAG>(ldsV, ct, x + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int ct = 0; ct < T; ++ct) {
                u32x4 w = v[x & 1][ct];
                if (!FRAG && poison) {
#pragma unroll
                    for (int y = 0; y < 4; ++y) w[y] = finite_halves<CT>(w[y]);
                }
#pragma unroll
                for (int z = 0; z < PP; ++z) st.acc[ct] = mfma32(__builtin_bit_cast(v8, w), p[z][x], st.acc[ct]);
            }
        }
    }
}

// 64 rows of a type into LDS, straight from memory; rows behind `rows` are zeros.  Not waited for: s_waitcnt vmcnt(0) in front of the barrier.  (The instruction is
// written out, since for the builtin the compiler waits in front of the next transposed read from LDS, whichever part of it that reads: the next tile was waited for
// in the middle of this one.  It has no register output; nothing else here uses m0.)
template <int ROWB, int NW, bool VALUES, int EB> struct RowFetch {
    static constexpr int I = 64 * ROWB / 1024 / NW, STEP = NW * 1024;       // loads of a wave; bytes from one to the next
    // pieces are moved alike 16 rows on: in every VARIANTS-th of a wave's loads (kept in registers where those are few)
    static constexpr int VARIANTS = 16 * ROWB > STEP ? 16 * ROWB / STEP : 1;
    static constexpr bool KEPT = VARIANTS <= 4;
    static_assert(I >= 1, "a load for every wave");
    int at[KEPT ? VARIANTS : 1];
    // where the piece comes from that lane's load u puts into its place
    static __device__ __forceinline__ int source(int u) {
        const uint32_t at = ((threadIdx.x >> 6) + NW * u) * 64 + (threadIdx.x & 63), row = at / (ROWB / 16), piece = at % (ROWB / 16);
        return (int)(row * ROWB) + (VALUES ? value_piece<ROWB, EB>((int)row, (int)piece) : key_piece<ROWB>((int)row, (int)piece)) * 16;
    }
    __device__ __forceinline__ RowFetch() {
#pragma unroll
        for (int u = 0; u < (KEPT ? VARIANTS : 1); ++u) {
            at[u] = source(u);
            asm volatile("" : "+v"(at[u]));
        }
    }
    // Whether some number that the wave itself has fetched (and waited for) is none.
    template <int CT> static __device__ __forceinline__ bool no_number(const char* lds) {
        u32x4 w[I];
#pragma unroll
        for (int u = 0; u < I; ++u) w[u] = *reinterpret_cast<const u32x4*>(lds + (((int)threadIdx.x >> 6) + NW * u) * 1024 + lane_id() * 16);
        return __any(any_no_number<CT, I>(w));
    }
    __device__ __forceinline__ void operator()(const char* from, int rows, char* lds) const;
};
template <int ROWB, int NW, bool VALUES, int EB>
__device__ __forceinline__ void RowFetch<ROWB, NW, VALUES, EB>::operator()(const char* from, int rows, char* lds) const {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    const uint64_t base = (uint64_t)from;
    i32x4 rsrc = {(int)(uint32_t)base, (int)((uint32_t)(base >> 32) & 0xFFFFu), rows * ROWB, 0x00020000};
#pragma unroll
    for (int y = 0; y < 4; ++y) rsrc[y] = __builtin_amdgcn_readfirstlane(rsrc[y]);
    const uint32_t to = (uint32_t)(uint64_t)(__attribute__((address_space(3))) char*)lds;
#pragma unroll
    for (int u = 0; u < I; ++u) {
        const int off = KEPT ? at[u % VARIANTS] : source(u), ahead = KEPT ? u / VARIANTS * VARIANTS * STEP : 0;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :: "s"(__builtin_amdgcn_readfirstlane((int)(to + (wave + NW * u) * 1024))), "v"(off), "s"(rsrc), "s"(ahead) : "memory");
    }
}

// 32 bits that grow without end round every small addition the same way (65536 equal weights, fp32: 2.6e-4 of the sum, when every two keys were an addition).
// Splits of more tiles than this put a lane's sums aside after as many, and begin again (FOLD).  Additions that follow each other: one for a tile (fp32), four (16 bits) or
// eight (codes and fp32 queries), as many as there are tiles between two times, and then as many as there are times.
template <int DT, bool CODED> constexpr int kFoldTiles = DT != DT_F32 ? 512 : CODED ? 128 : 256;
// The sums put aside, of a lane: in scratch memory, since there are no registers or LDS for them beside two workgroups (d = 128 in 16 bits), relative to the powers of two
// they were put aside with, which only rise.  (35 MB there and back a time, if all workgroups of d = 128 do it at once.  2048 tokens at the end of 200000, 16 heads
// over 4, fp16: 3815 us and 3806 without; every 128 tiles 3 % of the time.)
template <int D, bool FOLD> struct KeptSums {
    typedef __attribute__((address_space(5))) float* Place;
    static constexpr int M = D / 2, E = D / 2 + 1, L = D / 2 + 2, SIZE = D / 2 + 3;
    Place at;
    // (passed through a register: as an array that the compiler sees through it would be in registers)
    __device__ __forceinline__ explicit KeptSums(float* room) : at((Place)room) { if (FOLD) asm volatile("" : "+v"(at)); }
    // (nothing so far but keys of -inf or NaN: the sums are zero or NaN)
    static __device__ __forceinline__ float turn(float before, float now) { return before == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(before - now); }
    // VSCALE: the weighted sums have a power of two of their own.  first: nothing is there yet
    template <bool VSCALE> __device__ __forceinline__ void put(RowState<D>& st, bool first) const {
        if (!first) take<VSCALE>(st);
        at[M] = st.m;
        at[E] = st.e;
        at[L] = st.l;
        st.l = 0.f;
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                at[16 * ct + i] = st.acc[ct][i];
                st.acc[ct][i] = 0.f;
            }
        }
    }
    template <bool VSCALE> __device__ __forceinline__ void take(RowState<D>& st) const {
        const float f = turn(at[M], st.m), f_acc = VSCALE ? turn(at[E], st.e) : f;
        st.l = fmaf(at[L], f, st.l);
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st.acc[ct][i] = fmaf(at[16 * ct + i], f_acc, st.acc[ct][i]);
        }
    }
};

// DT: type of queries, output and open rows; FMT: the coded cache's format, or -1: rows of DT.  NW waves of 32 rows.  FOLD: more than kFoldTiles tiles a split.
template <int DT, int FMT, int D, int NW, bool FOLD>
__global__ void __launch_bounds__(64 * NW, (NW > 1 && D <= 128 && DT != DT_F32 ? 2 : 1)) prompt_kernel(PromptCall a) {
    constexpr bool CODED = FMT >= 0;
    constexpr int CT = CODED ? DT_F16 : DT, PARTS = CODED && DT == DT_F32 ? 2 : 1;
    constexpr int EB = TileType<CT>::bytes, ROWB = D * EB, TILE = 64 * ROWB, OPEN_ROWB = D * TileType<DT>::bytes;
    constexpr int NBUF = 4 * TILE <= 131072 ? 2 : 1;
    constexpr int LDS = 2 * NBUF * TILE > 128 * OPEN_ROWB || !CODED ? 2 * NBUF * TILE : 128 * OPEN_ROWB;
    constexpr int NT = 64 * NW, ROWS = 32 * NW, FM = CODED ? FMT : CODED_E4M3;
    __shared__ __align__(16) char lds[LDS];
    __shared__ uint32_t suspects[2][NW];                            // waves that have fetched a value that is no number
    const int lane = lane_id(), hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const auto any_suspect = [&](int buf) {
        uint32_t x = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) x |= suspects[buf][w];
        return __builtin_amdgcn_readfirstlane((int)x) != 0;
    };
    // Streams next to each other (workgroups go to the XCDs in turn: a stream stays on one where their number is a multiple of eight), the last rows, which see most, first.
    const int streams = a.S * a.Hkv, stream = (int)blockIdx.x % streams, rest = (int)blockIdx.x / streams;
    const int split = rest % a.n_split, rb = a.row_blocks - 1 - rest / a.n_split;
    const int b = stream / a.Hkv, kvh = stream - b * a.Hkv;
    const int N = a.len[b], M = (int)a.M, n_rows = M * a.G, row0 = rb * ROWS;
    const int sinks = (int)(a.sinks < N ? a.sinks : N);
    const int before = N - M;                                       // tokens in front of the first query's
    const auto query_of = [&](int row) { return (row < n_rows ? row : n_rows - 1) / a.G; };
    const auto hidden_of = [&](int p) { return a.window <= p ? p - (int)a.window : -1; };

    // tiles that some row of the workgroup sees: `front` of the sinks, then from .. to
    const int p_lo = before + query_of(row0), p_hi = before + query_of(row0 + ROWS - 1);
    const int first = hidden_of(p_lo) + 1;
    int front = ((sinks < p_hi + 1 ? sinks : p_hi + 1) + 63) / 64, from = first / 64;
    if (front >= from) { front = 0; from = 0; }
    const int full = CODED ? N / 64 : 0x7FFFFFFF;                   // (open rows after the loop)
    if (front > full) front = full;
    int to = p_hi / 64 + 1;
    if (to > full) to = full;
    if (from > to) from = to;
    const int n_tiles = front + to - from;
    // (a block that sees more tiles than the call was planned for, as after a replay on a longer sequence: the last split takes them)
    const int i0 = split * a.chunk < n_tiles ? split * a.chunk : n_tiles, i1 = split + 1 < a.n_split && i0 + a.chunk < n_tiles ? i0 + a.chunk : n_tiles;
    const auto tile_of = [&](int i) { return i < front ? i : from + (i - front); };
    // Of those, all rows see all keys of [0, all0) (sinks), and of [all1, all2): behind the newest token that a window leaves out, up to the first row's.
    const int last_hidden = hidden_of(p_hi), up_to = (p_lo + 1) / 64;
    const auto index_of = [&](int tile) { const int i = tile - from + front; return i < 0 ? 0 : i > n_tiles ? n_tiles : i; };
    int all0 = sinks / 64 < up_to ? sinks / 64 : up_to;
    if (from > 0 && all0 > front) all0 = front;
    if (all0 > n_tiles) all0 = n_tiles;
    int all1 = index_of(last_hidden < 0 ? 0 : last_hidden / 64 + 1), all2 = index_of(up_to);
    if (all1 < front) all1 = front;
    if (all1 < all0) all1 = all0;
    if (all2 < all1) all2 = all1;
    const auto within = [&](int i) { return i < i0 ? i0 : i > i1 ? i1 : i; };
    const int end0 = within(all0), end1 = within(all1), end2 = within(all2);

    RowState<D> st;
    const int at0 = row0 + 32 * wave, wave_lo = before + query_of(at0), wave_hi = before + query_of(at0 + 31);
    st.m = st.e = -INFINITY;
    st.l = 0.f;
    st.pos = before + query_of(at0 + (lane & 31));
    st.hidden = hidden_of(st.pos);
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct) st.acc[ct] = f32x16{};
    float room[FOLD ? KeptSums<D, FOLD>::SIZE : 1];
    const KeptSums<D, FOLD> kept(room);
    // The walk over tiles lo to hi - 1, in runs between two times that the sums are put aside.
    constexpr int RUN = kFoldTiles<DT, CODED>;
    const auto in_runs = [&](auto walk, auto masked, int lo, int hi) {
        if (!FOLD) return walk(masked, lo, hi);
        while (lo < hi) {
            const int next = i0 + ((lo - i0) / RUN + 1) * RUN, end = next < hi ? next : hi;
            walk(masked, lo, end);
            lo = end;
            if (lo == next && lo < i1) kept.template put<CODED>(st, lo - i0 == RUN);
        }
    };
    const auto end_walk = [&] { if (FOLD && i1 - i0 > RUN) kept.template take<CODED>(st); };
    const bool idle = at0 >= n_rows;
    const int wave_first = hidden_of(wave_lo) + 1;                  // oldest token that a window of the wave has
    const auto seen = [&](int t0) { return !idle && t0 <= wave_hi && (t0 + 63 >= wave_first || t0 < sinks); };

    constexpr double kScale = 1.4426950408889634 / (D == 32 ? 5.656854249492381 : D == 64 ? 8.0 : D == 128 ? 11.313708498984761 : 16.0);
    constexpr float kScaleHi = (float)kScale, kScaleLo = (float)(kScale - (double)kScaleHi);

    int64_t query_row;                                              // the lane's row in q and out, in elements
    {
        const int row = at0 + (lane & 31) < n_rows ? at0 + (lane & 31) : n_rows - 1, m = row / a.G;
        query_row = (((int64_t)b * M + m) * a.Hq + kvh * a.G + (row - m * a.G)) * D;
    }
    const char* const query = static_cast<const char*>(a.q) + query_row * TileType<DT>::bytes;
    const auto load_row = [&](auto& frag) {                         // the query in its own type
#pragma unroll
        for (int c = 0; c < D * TileType<DT>::bytes / 32; ++c)
            frag.v[0][c] = __builtin_bit_cast(typename std::remove_reference<decltype(frag.v[0][c])>::type, *reinterpret_cast<const u32x4*>(query + 32 * c + 16 * hh));
    };

    if constexpr (!CODED) {
        QueryFrag<DT, D, 1> q;
        load_row(q);
        // (arrived before the loop: the compiler, which does not know the loads of the tiles, would wait for them with the queries)
#pragma unroll
        for (int c = 0; c < QueryFrag<DT, D, 1>::N; ++c) asm volatile("" : "+v"(q.v[0][c]));
        const char* const Kh = a.K + (int64_t)stream * a.Ncap * ROWB;
        const char* const Vh = a.V + (int64_t)stream * a.Ncap * ROWB;
        const RowFetch<ROWB, NW, false, EB> keys;
        const RowFetch<ROWB, NW, true, EB> values;
        const auto fetch = [&](int i, int buf) {
            const int t0 = 64 * tile_of(i), rows = N - t0 < 64 ? N - t0 : 64;
            keys(Kh + (int64_t)t0 * ROWB, rows, lds + buf * 2 * TILE);
            values(Vh + (int64_t)t0 * ROWB, rows, lds + buf * 2 * TILE + TILE);
        };
        if (NBUF == 2 && i0 < i1) fetch(i0, 0);
        const auto walk = [&](auto masked, int lo, int hi) {
            for (int i = lo; i < hi; ++i) {
                const int buf = NBUF == 2 ? (i - i0) & 1 : 0;
                if (NBUF == 1) {
                    __syncthreads();
                    fetch(i, 0);
                }
                const char* const at = lds + buf * 2 * TILE;
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                if (decltype(masked)::value) {
                    const bool bad = RowFetch<ROWB, NW, true, EB>::template no_number<DT>(at + TILE);
                    if (lane == 0) suspects[buf][wave] = bad;
                }
                __syncthreads();
                if (NBUF == 2 && i + 1 < i1) fetch(i + 1, buf ^ 1);
                const int t0 = 64 * tile_of(i);
                if (decltype(masked)::value ? seen(t0) : !idle)
                    prompt_tile<DT, false, false, DT == DT_F32, decltype(masked)::value, D, 1, 1>(at, at + TILE, q, st, kScaleHi, kScaleLo, 1.f, t0, sinks,
                                                                                                   decltype(masked)::value && any_suspect(buf));
            }
        };
#pragma unroll 1
        for (int x = 0; x < 2; ++x) {
            in_runs(walk, std::false_type{}, x ? end1 : i0, x ? end2 : end0);
            in_runs(walk, std::true_type{}, x ? end2 : end0, x ? i1 : end1);
        }
        end_walk();
    } else {
        // ---- blocks: codes through registers, into LDS as fp16 ----
        float unit_q;
        {
            QueryFrag<DT_F16, D, PARTS> q;
            {
                float amax = 0.f;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    float x[8];
#pragma unroll
                    for (int y = 0; y < 8; y += Elem<DT>::kPerLoad)
                        Elem<DT>::widen(*reinterpret_cast<const u32x4*>(query + (16 * c + 8 * hh + y) * TileType<DT>::bytes), x + y);
#pragma unroll
                    for (int y = 0; y < 8; ++y) amax = fmaxf(amax, fabsf(x[y]));
                }
                amax = other_half_max(amax);
                int up = 13 - ((int)(__float_as_uint(amax) >> 23) - 127);       // amax times 2^up lies in [2^13, 2^14)
                up = amax == 0.f || up > 120 ? 120 : up < -114 ? -114 : up;
                const float by = __uint_as_float((uint32_t)(up + 127) << 23);
                unit_q = __uint_as_float((uint32_t)(127 - up) << 23) * CodeUnit<FM>::value;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    float x[8];
#pragma unroll
                    for (int y = 0; y < 8; y += Elem<DT>::kPerLoad)
                        Elem<DT>::widen(*reinterpret_cast<const u32x4*>(query + (16 * c + 8 * hh + y) * TileType<DT>::bytes), x + y);
#pragma unroll
                    for (int y = 0; y < 8; ++y) {
                        float left = x[y] * by;                     // (exact)
#pragma unroll
                        for (int z = 0; z < PARTS; ++z) {
                            q.v[z][c][y] = (_Float16)left;
                            left -= (float)q.v[z][c][y];
                        }
                    }
                }
            }
            constexpr int CB = coded_block_bytes(D), PT = CB / 16 / NT;         // pieces of 16 bytes of a thread
            static_assert(CB / 16 % NT == 0 || CB / 16 < NT, "whole passes");
            constexpr int P = PT ? PT : 1;
            u32x4 k[P], v[P];
            float2 scale = make_float2(0.f, 0.f), next = scale;
            const char* const Kb = a.c.codes[0] + (int64_t)stream * a.c.blocks * CB;
            const char* const Vb = a.c.codes[1] + (int64_t)stream * a.c.blocks * CB;
            const float* const Sb = a.c.scales + (int64_t)stream * a.c.blocks * 2;
            const bool mine = PT || (int)threadIdx.x < CB / 16;
            const auto load = [&](int i) {
                const int64_t block = tile_of(i);
                if (mine) {
#pragma unroll
                    for (int u = 0; u < P; ++u) {
                        const int at = (u * NT + (int)threadIdx.x) * 16;
                        k[u] = *reinterpret_cast<const u32x4*>(Kb + block * CB + at);
                        v[u] = *reinterpret_cast<const u32x4*>(Vb + block * CB + at);
                    }
                }
                next = *reinterpret_cast<const float2*>(Sb + 2 * block);
            };
            const auto place = [&](int buf) {
                char* const to = lds + buf * 2 * TILE;
                if (!mine) return;
#pragma unroll
                for (int u = 0; u < P; ++u) {
                    const int x = u * NT + (int)threadIdx.x, pair = x / 64, j = (x >> 4) & 3, n = x & 15;
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int unit = 2 * pair + y, key = 16 * (unit / (D / 32)) + n, piece = 4 * (unit % (D / 32)) + j;
                        *reinterpret_cast<f16x8*>(to + key * ROWB + key_piece<ROWB>(key, piece) * 16) = code_values<FM>(k[u][2 * y], k[u][2 * y + 1]);
                    }
                    const int ch = 16 * pair + n;
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const u32x4 w = __builtin_bit_cast(u32x4, code_values<FM>(v[u][2 * y], v[u][2 * y + 1]));
#pragma unroll
                        for (int z = 0; z < 2; ++z)                  // keys 16 (2 y + z) + 4 j .. + 3
                            *reinterpret_cast<uint2*>(to + TILE + (((2 * y + z) * (D / 32) + ch / 32) * 64 + (j & 1) * 32 + ch % 32) * 16 + (j >> 1) * 8) =
                                make_uint2(w[2 * z], w[2 * z + 1]);
                    }
                }
            };
            // (in vector registers: moved into scalar ones, as the compiler would have a block's numbers, they were waited for where they are asked for)
            const auto take_scale = [&] {
                scale = next;
                asm volatile("" : "+v"(scale.x), "+v"(scale.y));
            };
            if (i0 < i1) {
                load(i0);
                place(0);
                take_scale();
            }
            const auto walk = [&](auto masked, int lo, int hi) {
                for (int i = lo; i < hi; ++i) {
                    const int buf = NBUF == 2 ? (i - i0) & 1 : 0;
                    if (i + 1 < i1) load(i + 1);
                    __syncthreads();
                    const int t0 = 64 * tile_of(i);
                    const char* const at = lds + buf * 2 * TILE;
                    if (decltype(masked)::value ? seen(t0) : !idle) {
                        const float by = scale.x * unit_q, f = by * kScaleHi, f_lo = fmaf(by, kScaleHi, -f) + by * kScaleLo;
                        prompt_tile<DT_F16, true, true, DT == DT_F32, decltype(masked)::value, D, PARTS, PARTS>(at, at + TILE, q, st, f, f_lo, scale.y, t0, sinks, false);
                    }
                    if (NBUF == 1) __syncthreads();
                    if (i + 1 < i1) {
                        place(NBUF == 2 ? buf ^ 1 : 0);
                        take_scale();
                    }
                }
            };
#pragma unroll 1
            for (int x = 0; x < 2; ++x) {
                in_runs(walk, std::false_type{}, x ? end1 : i0, x ? end2 : end0);
                in_runs(walk, std::true_type{}, x ? end2 : end0, x ? i1 : end1);
            }
        }
        end_walk();
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st.acc[ct][i] *= CodeUnit<FM>::value;
        }
        // ---- open rows, in their own type, with the last blocks ----
        const int t0 = 64 * full;
        if (p_hi >= t0 && (i1 == n_tiles && (i0 < i1 || split == 0))) {
            const char* const open = a.c.open + (int64_t)stream * 2 * 64 * OPEN_ROWB;
            __syncthreads();
            RowFetch<OPEN_ROWB, NW, false, TileType<DT>::bytes>()(open, N - t0, lds);
            RowFetch<OPEN_ROWB, NW, true, TileType<DT>::bytes>()(open + 64 * OPEN_ROWB, N - t0, lds + 64 * OPEN_ROWB);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const bool bad = RowFetch<OPEN_ROWB, NW, true, TileType<DT>::bytes>::template no_number<DT>(lds + 64 * OPEN_ROWB);
            if (lane == 0) suspects[0][wave] = bad;
            __syncthreads();
            if (seen(t0)) {
                QueryFrag<DT, D, 1> q;
                load_row(q);
                prompt_tile<DT, false, true, DT == DT_F32, true, D, 1, 1>(lds, lds + 64 * OPEN_ROWB, q, st, kScaleHi, kScaleLo, 1.f, t0, sinks, any_suspect(0));
            }
        }
    }
    // ---- what the rows leave ----
    float l = st.l, m = st.m;
    {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    const int at = 32 * wave + (lane & 31);
    float by = 1.f;                                                 // brings the weighted sum to 2^m
    if (CODED) by = st.e == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.e - (m == -INFINITY ? 0.f : m) - kShift16);       // (beyond 2^24 one of them less 13 is no number)
    if (row0 + at >= n_rows) return;
    if (a.n_split == 1) {
        const float inv = by / l;
        char* const o = static_cast<char*>(a.out) + query_row * TileType<DT>::bytes;
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int ch = 32 * ct + 8 * x + 4 * hh;
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = st.acc[ct][4 * x + e] * inv;
                if constexpr (DT == DT_F32) {
                    *reinterpret_cast<f32x4*>(o + ch * 4) = f32x4{y[0], y[1], y[2], y[3]};
                } else {
                    using E = typename std::conditional<DT == DT_F16, _Float16, __bf16>::type;
                    typedef E e4 __attribute__((ext_vector_type(4)));
                    *reinterpret_cast<e4*>(o + ch * 2) = e4{(E)y[0], (E)y[1], (E)y[2], (E)y[3]};
                }
            }
        }
        if (hh == 0 && a.lse) a.lse[query_row / D] = (m + log2f(l)) * 0.69314718055994531f;
    } else {
        // (a maximum passes over NaN: a split of nothing but NaN would count as one without a key)
        if (l != l) m = INFINITY;
        const int64_t slot = ((int64_t)(stream * a.row_blocks + rb) * a.n_split + split) * ROWS + at;
        float* const o = a.part_acc + slot * D;
        if (hh == 0) { a.part_lm[2 * slot] = l; a.part_lm[2 * slot + 1] = m; }
        if (m == -INFINITY) return;                                 // (no key that the row sees: the joint does not look at the sum)
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
                *reinterpret_cast<f32x4*>(o + 32 * ct + 8 * x + 4 * hh) =
                    f32x4{st.acc[ct][4 * x] * by, st.acc[ct][4 * x + 1] * by, st.acc[ct][4 * x + 2] * by, st.acc[ct][4 * x + 3] * by};
        }
    }
}

}  // namespace tka
