// Partial sums of the splits of a head's keys, put together: out = sum_i f_i acc_i / sum_i f_i l_i with f_i = 2^(m_i - max m).
#pragma once
#include <type_traits>

#include "device_utils.h"
#include "internal.h"
#include "ops.h"

namespace tka {

// What the splits leave is read by a workgroup of the same launch, maybe on another XCD: written and read past the caches that are not shared.
__device__ __forceinline__ void put(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float2 get2(const float* p) {
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
// log2 of the sum of a head's weights (not shifted), over its splits; one wave.  `f` (or null) gets the factor of each split's weighted sum.
__device__ __forceinline__ float head_log2_sum(const SplitParts& a, int64_t bh, int n_split, float shift, float* f) {
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
// Where the heads of a joint go: out [heads][D] and lse [heads] of the call.
struct JoinedHeads {
    const SplitParts& a;
    int64_t head0;
    __device__ __forceinline__ void sum(int h, int c, f32x4 v) const {
        float* const out = a.out + (head0 + h) * a.D + c;
#pragma unroll
        for (int y = 0; y < 4; ++y) out[y] = v[y];
    }
    __device__ __forceinline__ void lse(int h, float v) const { if (a.lse) a.lse[head0 + h] = v; }
};
// Where rows of a key stream go, from the row0-th on, if they are those of a prompt's tokens: row m G + g is head g of the group of token m.
template <int DT, typename Call> struct JoinedRows {
    const Call& a;
    int stream, row0;
    __device__ __forceinline__ int64_t at(int h) const {
        const int row = row0 + h, m = row / a.G, b = stream / a.Hkv;
        return ((int64_t)b * a.M + m) * a.Hq + (stream - b * a.Hkv) * a.G + (row - m * a.G);
    }
    __device__ __forceinline__ void one(int h, int c, float v) const {
        using E = typename std::conditional<DT == DT_F32, float, typename std::conditional<DT == DT_F16, _Float16, __bf16>::type>::type;
        static_cast<E*>(a.out_rows)[at(h) * a.D + c] = (E)v;
    }
    __device__ __forceinline__ void sum(int h, int c, f32x4 v) const {
#pragma unroll
        for (int y = 0; y < 4; ++y) one(h, c + y, v[y]);
    }
    __device__ __forceinline__ void lse(int h, float v) const { if (a.lse) a.lse[at(h)] = v; }
};

// Weighted sum of the splits of `quads` groups of four channels.  Four sums, by split modulo four, whichever thread takes them: the result does
// not depend on how many heads are joined at a time.
template <int NT, int SHARES, typename To>
__device__ __forceinline__ void sum_splits(const SplitParts& a, int64_t head0, const To& to, int quads, int n_split, const float* f, f32x4* part) {
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
            to.sum(h, c, (sum[0] + sum[1 % SUMS]) + (sum[2 % SUMS] + sum[3 % SUMS]));
        }
    }
    if (SHARES > 1) {
        __syncthreads();
        if ((int)threadIdx.x < quads) {
            const f32x4* q = part + threadIdx.x;
            to.sum((int)threadIdx.x / quarter, 4 * ((int)threadIdx.x % quarter), (q[0] + q[quads]) + (q[2 * quads] + q[3 * quads]));
        }
    }
}
// Sums and lse of `heads` neighbouring heads (at most 16) from their splits; a workgroup of NT threads, f: [heads][n_split] in LDS.
template <int NT, typename To>
__device__ __forceinline__ void join_splits(const SplitParts& a, int64_t head0, const To& to, int heads, int n_split, float shift, float* f, f32x4* part) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    for (int h = wave; h < heads; h += NT / kWave) {
        const float lg2 = head_log2_sum(a, head0 + h, n_split, shift, f + h * n_split);
        if (lane_id() == 0) to.lse(h, lg2 * 0.69314718055994531f);
    }
    __syncthreads();
    // Four channels a thread; with few of them two or four threads share a group's splits.
    const int quads = heads * (a.D / 4);
    if (quads <= NT / 4) sum_splits<NT, 4>(a, head0, to, quads, n_split, f, part);
    else if (quads <= NT / 2) sum_splits<NT, 2>(a, head0, to, quads, n_split, f, part);
    else sum_splits<NT, 1>(a, head0, to, quads, n_split, f, part);
}
template <int NT>
__device__ __forceinline__ void join_splits(const SplitParts& a, int64_t head0, int heads, int n_split, float shift, float* f, f32x4* part) {
    join_splits<NT>(a, head0, JoinedHeads{a, head0}, heads, n_split, shift, f, part);
}

}  // namespace tka
