// New tokens' projections into the cache (topk_attn_append_rotary): keys and queries normalised per head and turned by their position,
// values copied, in one pass: every element is read once and written once, which is what bounds it.  8191 tokens of 32 + 2 x 8 heads, d = 128: 47 us for
// 201 MB (4.3 TB/s; a large copy reaches 4.8); one token of 16 sequences 6.3 us, all latency.
#include "device_utils.h"
#include "internal.h"
#include "ops.h"

namespace tka {

// float to the storage type, round to nearest even
template <int DT>
__device__ __forceinline__ uint32_t round_bits(float v) {
    if (DT == DT_F32) return __float_as_uint(v);
    if (DT == DT_F16) return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v);
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v);
}
template <int DT>
__device__ __forceinline__ u32x4 pack_row(const float* f) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (DT == DT_F32) r[i] = round_bits<DT>(f[i]);
        else r[i] = round_bits<DT>(f[(2 * i) % Elem<DT>::kPerLoad]) | (round_bits<DT>(f[(2 * i + 1) % Elem<DT>::kPerLoad]) << 16);
    }
    return r;
}

// Sums of squares that a row is scaled for: above the one infinity is near, below the other squares of its numbers lose bits.
constexpr float kLargeSquares = 0x1p+120f, kSmallSquares = 0x1p-80f;

// A workgroup per token.  D e / 16 lanes hold a row (a head of the token); a channel's partner, which lies in another lane when halves
// are paired, comes through LDS.  The angle is pos * inv_freq in 64 bits, reduced to a fraction of a turn there: in 32 bits a position of
// 10^6 leaves 0.06 radian of error.
template <int DT, int D>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryCall a) {
    constexpr int EPL = Elem<DT>::kPerLoad, ROW = D * Elem<DT>::kBytes, LPR = ROW / 16, RPP = 256 / LPR, U = 4;
    __shared__ float2 turn[D / 2];
    __shared__ float part[RPP][D];
    const int64_t t = blockIdx.x % a.n;
    const int b = (int)(blockIdx.x / a.n);
    const int c = (int)threadIdx.x % LPR, slot = (int)threadIdx.x / LPR;
    const int heads_q = a.q ? a.Hq : 0, rows = heads_q + 2 * a.Hkv;
    const int64_t at = (a.base >= 0 ? a.base : (int64_t)a.len[b]) + t;      // row of the cache
    const int half = a.rotary / 2;
    u32x4 raw[U];
    // rows of the token: query heads, key heads, value heads
    auto source = [&](int r) -> const char* {
        if (r < heads_q) return a.q + b * a.q_seq + t * a.q_token + (int64_t)r * ROW;
        r -= heads_q;
        if (r < a.Hkv) return a.k + b * a.k_seq + t * a.k_token + (int64_t)r * ROW;
        return a.v + b * a.v_seq + t * a.v_token + (int64_t)(r - a.Hkv) * ROW;
    };
    auto load = [&](int r0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = r0 + u * RPP + slot;
            raw[u] = *reinterpret_cast<const u32x4*>(source(r < rows ? r : rows - 1) + c * 16);
        }
    };
    load(0);
    if ((int)threadIdx.x < half) {
        const double pos = a.positions ? (double)a.positions[b * a.n + t] : (double)at;
        const double turns = pos * (double)a.inv_freq[threadIdx.x] * 0.15915494309189533577;
        float s, co;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &co);
        turn[threadIdx.x] = make_float2(co, s);
    }
    float qw[EPL], kw[EPL];
    if (a.q_norm) Elem<DT>::widen(*reinterpret_cast<const u32x4*>(static_cast<const char*>(a.q_norm) + c * 16), qw);
    if (a.k_norm) Elem<DT>::widen(*reinterpret_cast<const u32x4*>(static_cast<const char*>(a.k_norm) + c * 16), kw);
    __syncthreads();
    for (int r0 = 0; r0 < rows; r0 += U * RPP) {
        if (r0) load(r0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = r0 + u * RPP + slot;
            const bool is_q = r < heads_q, is_k = !is_q && r < heads_q + a.Hkv;
            u32x4 done = raw[u];
            float x[EPL];
            if (is_q || is_k) {                                     // (whole groups of LPR lanes; the others copy)
                Elem<DT>::widen(raw[u], x);
                if (is_q ? a.q_norm != nullptr : a.k_norm != nullptr) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < EPL; ++e) ss = fmaf(x[e], x[e], ss);
                    ss = group_reduce<AddOp, LPR>(ss);
                    float eps = a.eps;
                    if (DT != DT_F16 && (ss > kLargeSquares || (ss < kSmallSquares && eps < kSmallSquares))) {
                        // squares beyond 32 bits: of the row times a power of two
                        const float s = ss > kLargeSquares ? 0x1p-80f : 0x1p+90f;
                        ss = 0.f;
#pragma unroll
                        for (int e = 0; e < EPL; ++e) { x[e] *= s; ss = fmaf(x[e], x[e], ss); }
                        ss = group_reduce<AddOp, LPR>(ss);
                        eps = eps * s * s;
                    }
                    const float inv = 1.0f / sqrtf(ss * (1.0f / D) + eps);
#pragma unroll
                    for (int e = 0; e < EPL; ++e) x[e] = x[e] * inv * (is_q ? qw[e] : kw[e]);
                }
#pragma unroll
                for (int e = 0; e < EPL; ++e) part[slot][c * EPL + e] = x[e];
            }
            wave_sync();                                            // (a row lies within a wave)
            if (is_q || is_k) {
#pragma unroll
                for (int e = 0; e < EPL; ++e) {
                    const int ch = c * EPL + e;
                    if (ch < a.rotary) {
                        const bool second = a.interleaved ? ch & 1 : ch >= half;
                        const int i = a.interleaved ? ch >> 1 : second ? ch - half : ch;
                        const float p = part[slot][a.interleaved ? ch ^ 1 : second ? ch - half : ch + half];
                        const float2 w = turn[i];
                        x[e] = second ? fmaf(x[e], w.x, p * w.y) : fmaf(x[e], w.x, -(p * w.y));
                    }
                }
                done = pack_row<DT>(x);
            }
            wave_sync();                                            // (before the next rows take their places)
            if (r < rows) {
                if (is_q) {
                    *reinterpret_cast<u32x4*>(a.q_out + ((int64_t)blockIdx.x * a.Hq + r) * ROW + c * 16) = done;
                } else {
                    const int h = is_k ? r - heads_q : r - heads_q - a.Hkv;
                    const int64_t row = ((int64_t)b * a.Hkv + h) * a.Ncap + at;
                    *reinterpret_cast<u32x4*>((is_k ? a.K : a.V) + row * ROW + c * 16) = done;
                    if constexpr (DT != DT_F32 && D >= 64) {
                        // code = rint(x 127 / amax), scale = amax / 127 of the row as it is stored
                        if (is_k && a.codes) {
                            Elem<DT>::widen(done, x);
                            float amax = 0.f;
#pragma unroll
                            for (int e = 0; e < EPL; ++e) amax = fmaxf(amax, fabsf(x[e]));
                            amax = group_reduce<MaxOp, LPR>(amax);
                            const bool live = amax >= kTinyRow;
                            const float inv = live ? 127.0f / amax : 0.f;
                            uint32_t w[2];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                uint32_t p = 0;
#pragma unroll
                                for (int e = 0; e < 4; ++e) p |= ((uint32_t)(int)rintf(x[4 * i + e] * inv) & 0xFFu) << (8 * e);
                                w[i] = p;
                            }
                            *reinterpret_cast<uint2*>(a.codes + row * D + c * 8) = make_uint2(w[0], w[1]);
                            if (c == 0) a.scales[row] = live ? amax / 127.0f : 0.f;
                        }
                    }
                }
            }
        }
    }
    // the length, where no workgroup reads it but this one
    if (a.base >= 0 ? t == 0 : a.n == 1) {
        __syncthreads();
        if (threadIdx.x == 0 && a.advance) a.len[b] = (int32_t)(at - t + a.n);
    }
}

hipError_t launch_rotary(const RotaryCall& a, hipStream_t st) {
    const int64_t blocks = (int64_t)a.B * a.n;
    if (blocks > kMostWorkgroups) return hipErrorInvalidValue;
#define TKA_ROTARY(DT_, D_) hipLaunchKernelGGL((rotary_kernel<DT_, D_>), dim3((unsigned)blocks), dim3(256), 0, st, a)
    TKA_BY_TYPE_AND_DIM(TKA_ROTARY, a.dtype, a.D);
#undef TKA_ROTARY
    return hipGetLastError();
}

}  // namespace tka
