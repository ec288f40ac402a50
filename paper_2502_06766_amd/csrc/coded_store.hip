// Rows into the 8-bit cache and back (topk_attn_coded_append, topk_attn_coded_read).  A block of 64 tokens of a KV head is coded once, when its last
// row is there, from the rows as they came: what the cache holds does not depend on how the rows were handed over.
//   int8   scale = amax / 127 to 16 significant bits, code = the integer nearest to x / scale (ties to even).  A code has 7 bits, so
//          code * scale is exact in 32.  (The scale is rounded down where 127 of it would not be a number.)
//   e4m3   scale = the smallest power of two with amax <= 448 scale: x / scale is exact, and rounding it to e4m3 the only rounding.
// Blocks whose amax is below 2^-100 are zeros; a block with a NaN or an infinity has a scale of NaN, and all of it reads as NaN.
//
// Bound by the rows read and the codes written, 3 bytes an element of 16 bits; reading back 3 as well.  8 KV heads of d = 128: 8191 tokens into the cache
// 17 us, back 13.9 (3.6 TB/s); 48000 tokens 72.6 and 60.4 (4.1 and 4.9 TB/s; a copy reaches 4.9); one token of 16 sequences 2.8, of a step's 7.9 with the call.
#include "coded.h"

namespace tka {

namespace {

// The integer nearest to x / scale, ties to even; inv is 1 / scale to 32 bits.  x inv is off by 2^-23 of itself, 2^-16 for quotients up to 128, so the nearest
// integer r can be wrong only where x inv is within that of a half.  There x - r scale decides: r scale has 7 + 16 bits, the difference is a multiple
// of the last place of x or of the scale and at most 0.6 scale, so both are exact.
__device__ __forceinline__ float nearest_code(float x, float scale, float inv) {
    const float t = x * inv;
    float r = rintf(t);
    if (fabsf(fabsf(t - r) - 0.5f) < 0x1p-14f) {
        const float e = fmaf(-r, scale, x), h = 0.5f * scale;
        const bool odd = ((int)r) & 1;
        if (e > h || (e == h && odd)) r += 1.f;
        else if (e < -h || (e == -h && odd)) r -= 1.f;
    }
    return r;
}

// Scale of a block whose largest magnitude has the bits `amax` (of a NaN or an infinity: NaN).
template <int FMT>
__device__ __forceinline__ float block_scale(uint32_t amax) {
    if (amax >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    const float a = __uint_as_float(amax);
    if (a < kTinyRow) return 0.f;
    if (FMT == CODED_INT8) {
        const uint32_t b = __float_as_uint(__fdiv_rn(a, 127.f));
        const uint32_t r = (b + 0x7Fu + ((b >> 8) & 1u)) & 0xFFFFFF00u;
        return __uint_as_float(127.f * __uint_as_float(r) < INFINITY ? r : r - 0x100u);
    }
    // a = m 2^e with 1 <= m < 2: 448 = 1.75 2^8
    const int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Four values as the bytes of a word.
template <int FMT>
__device__ __forceinline__ uint32_t code4(const float* x, float scale, float inv) {
    if (FMT == CODED_INT8) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= (uint32_t)((int)nearest_code(x[i], scale, inv) + 128) << (8 * i);
        return w;
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
}
template <int FMT>
__device__ __forceinline__ void value4(uint32_t w, float scale, float* x) {
    if (FMT == CODED_INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)((int)((w >> (8 * i)) & 255u) - 128) * scale;
    } else {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo[0] * scale; x[1] = lo[1] * scale; x[2] = hi[0] * scale; x[3] = hi[1] * scale;
    }
}

}  // namespace

// Threads hold pieces of 16 bytes of four neighbouring rows (the four keys that a lane of the decode takes of a channel).
template <int DT, int D> struct StoreShape {
    static constexpr int EPL = Elem<DT>::kPerLoad, ROW = D * Elem<DT>::kBytes, CPR = ROW / 16;
    static constexpr int GROUPS = 16 * CPR;                    // of four rows by 16 bytes
    static constexpr int PASSES = (GROUPS + 255) / 256;
};

// A workgroup per block of a key stream and kind (keys or values) that becomes full; the first one of a stream also keeps the open rows: those
// of the block that was open before it reads before it writes, the others it has from the source.
template <int DT, int D, int FMT>
__global__ void __launch_bounds__(256) coded_append_kernel(CodedAppendCall p) {
    using S = StoreShape<DT, D>;
    constexpr int EPL = S::EPL, ROW = S::ROW, CPR = S::CPR, PASSES = S::PASSES;
    __shared__ __align__(16) uint32_t bytes[coded_block_bytes(D) / 4];
    __shared__ uint32_t top[4];
    const int tid = (int)threadIdx.x;
    const int64_t per = 2 * p.wgs, unit = blockIdx.x / per, in = blockIdx.x - unit * per;
    const int which = (int)(in & 1);
    const int64_t i = in >> 1;
    const int s = (int)(unit / p.Hkv), h = (int)(unit - (int64_t)s * p.Hkv);
    const int64_t n0 = p.base[s], n1 = n0 + p.n, block = n0 / kCodedBlock + i;
    const char* const src = p.src[which] + s * p.seq + h * p.head;
    char* const open = p.a.open + (unit * 2 + which) * kCodedBlock * ROW;
    const bool full = (block + 1) * kCodedBlock <= n1;
    if (!full && i) return;
    if (full) {
        u32x4 raw[PASSES][4];
        uint32_t amax = 0;
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
            const int g = u * 256 + tid, c = g % CPR, r0 = g / CPR * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                raw[u][e] = u32x4{0, 0, 0, 0};
                if (g < S::GROUPS) {
                    const int64_t t = block * kCodedBlock + r0 + e;
                    const char* from = t < n0 ? open + (r0 + e) * ROW : src + (t - n0) * p.token;
                    raw[u][e] = *reinterpret_cast<const u32x4*>(from + c * 16);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x[EPL];
                Elem<DT>::widen(raw[u][e], x);
#pragma unroll
                for (int y = 0; y < EPL; ++y) {
                    const uint32_t b = __float_as_uint(x[y]) & 0x7FFFFFFFu;      // (as whole numbers: a NaN counts as more than an infinity)
                    amax = b > amax ? b : amax;
                }
            }
        }
        amax = wave_max_u32(amax);
        if (lane_id() == 0) top[tid >> 6] = amax;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) amax = top[w] > amax ? top[w] : amax;
        const float scale = block_scale<FMT>(amax);
        const bool live = scale > 0.f;                       // (not NaN either)
        const float by = live ? scale : 1.f, inv = 1.0f / by;
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
            const int g = u * 256 + tid, c = g % CPR * EPL, r0 = g / CPR * 4;
            if (g >= S::GROUPS) break;
            float x[4][EPL];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                Elem<DT>::widen(raw[u][e], x[e]);
#pragma unroll
                for (int y = 0; y < EPL; ++y) x[e][y] = live ? x[e][y] : 0.f;
            }
            if (which == 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
#pragma unroll
                    for (int y = 0; y < EPL; y += 4) bytes[coded_key_at(D, r0 + e, c + y) / 4] = code4<FMT>(&x[e][y], by, inv);
                }
            } else {
#pragma unroll
                for (int y = 0; y < EPL; ++y) {
                    const float col[4] = {x[0][y], x[1][y], x[2][y], x[3][y]};
                    bytes[coded_value_at(r0, c + y) / 4] = code4<FMT>(col, by, inv);
                }
            }
        }
        __syncthreads();
        const int64_t at = unit * p.a.blocks + block;
        char* const to = p.a.codes[which] + at * coded_block_bytes(D);
#pragma unroll
        for (int o = 0; o < coded_block_bytes(D) / 16; o += 256)
            if (o + tid < coded_block_bytes(D) / 16)
                *reinterpret_cast<u32x4*>(to + (o + tid) * 16) = *reinterpret_cast<const u32x4*>(&bytes[(o + tid) * 4]);
        if (tid == 0) p.a.scales[at * 2 + which] = scale;
    }
    if (i) return;
    // the rows behind the last full block (all threads have read the open rows: two barriers ago)
    const int64_t last = n1 / kCodedBlock * kCodedBlock, from = last > n0 ? last : n0;
    for (int64_t x = tid; x < (n1 - from) * CPR; x += 256) {
        const int64_t t = from + x / CPR;
        const int c = (int)(x % CPR);
        *reinterpret_cast<u32x4*>(open + (t - last) * ROW + c * 16) = *reinterpret_cast<const u32x4*>(src + (t - n0) * p.token + c * 16);
    }
    if (which == 0 && h == 0 && tid == 0) p.a.len[s] = (int32_t)n1;
}

// A workgroup per block that the rows asked for touch, key stream and kind.
template <int DT, int D, int FMT>
__global__ void __launch_bounds__(256) coded_read_kernel(CodedReadCall p, int64_t blocks) {
    using S = StoreShape<DT, D>;
    constexpr int EPL = S::EPL, ROW = S::ROW, CPR = S::CPR;
    __shared__ __align__(16) uint32_t bytes[coded_block_bytes(D) / 4];
    const int tid = (int)threadIdx.x;
    const int64_t per = 2 * blocks, unit = blockIdx.x / per, in = blockIdx.x - unit * per;
    const int which = (int)(in & 1);
    const int64_t block = p.first / kCodedBlock + (in >> 1);
    const int s = (int)(unit / p.Hkv), h = (int)(unit - (int64_t)s * p.Hkv);
    char* const dst = p.dst[which] + s * p.seq + h * p.head;
    const bool full = (block + 1) * kCodedBlock <= (int64_t)p.a.len[s];
    float scale = 0.f;
    if (full) {
        const int64_t at = unit * p.a.blocks + block;
        const char* const from = p.a.codes[which] + at * coded_block_bytes(D);
        scale = p.a.scales[at * 2 + which];
#pragma unroll
        for (int o = 0; o < coded_block_bytes(D) / 16; o += 256)
            if (o + tid < coded_block_bytes(D) / 16)
                *reinterpret_cast<u32x4*>(&bytes[(o + tid) * 4]) = *reinterpret_cast<const u32x4*>(from + (o + tid) * 16);
    }
    __syncthreads();
    const char* const open = p.a.open + (unit * 2 + which) * kCodedBlock * ROW;
#pragma unroll
    for (int g = tid; g < S::GROUPS; g += 256) {
        const int c = g % CPR * EPL, r0 = g / CPR * 4;
        float x[4][EPL];
        if (full) {
            if (which == 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
#pragma unroll
                    for (int y = 0; y < EPL; y += 4) value4<FMT>(bytes[coded_key_at(D, r0 + e, c + y) / 4], scale, &x[e][y]);
                }
            } else {
#pragma unroll
                for (int y = 0; y < EPL; ++y) {
                    float col[4];
                    value4<FMT>(bytes[coded_value_at(r0, c + y) / 4], scale, col);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e][y] = col[e];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t t = block * kCodedBlock + r0 + e;
            if (t < p.first || t >= p.first + p.n) continue;
            u32x4 row;
            if (full) {
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    if (DT == DT_F32) row[y] = __float_as_uint(x[e][y]);
                    else if (DT == DT_F16)
                        row[y] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[e][(2 * y) % EPL]) |
                                 (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[e][(2 * y + 1) % EPL]) << 16;
                    else
                        row[y] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[e][(2 * y) % EPL]) |
                                 (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[e][(2 * y + 1) % EPL]) << 16;
                }
            } else {
                row = *reinterpret_cast<const u32x4*>(open + (r0 + e) * ROW + c * Elem<DT>::kBytes);
            }
            *reinterpret_cast<u32x4*>(dst + (t - p.first) * p.token + c * Elem<DT>::kBytes) = row;
        }
    }
}

hipError_t launch_coded_append(const CodedAppendCall& a, hipStream_t st) {
    const int64_t wgs = (int64_t)a.B * a.Hkv * 2 * a.wgs;
    if (wgs > kMostWorkgroups) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wgs), wg(256);
#define TKA_APPEND(DT_, D_)                                                                                               \
    do {                                                                                                                  \
        if (a.format == CODED_INT8) hipLaunchKernelGGL((coded_append_kernel<DT_, D_, CODED_INT8>), grid, wg, 0, st, a);   \
        else hipLaunchKernelGGL((coded_append_kernel<DT_, D_, CODED_E4M3>), grid, wg, 0, st, a);                          \
    } while (0)
    TKA_BY_TYPE_AND_DIM(TKA_APPEND, a.dtype, a.D);
#undef TKA_APPEND
    return hipGetLastError();
}

hipError_t launch_coded_read(const CodedReadCall& a, hipStream_t st) {
    const int64_t blocks = (a.first + a.n - 1) / kCodedBlock - a.first / kCodedBlock + 1, wgs = (int64_t)a.B * a.Hkv * 2 * blocks;
    if (wgs > kMostWorkgroups) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wgs), wg(256);
#define TKA_READ(DT_, D_)                                                                                                 \
    do {                                                                                                                  \
        if (a.format == CODED_INT8) hipLaunchKernelGGL((coded_read_kernel<DT_, D_, CODED_INT8>), grid, wg, 0, st, a, blocks); \
        else hipLaunchKernelGGL((coded_read_kernel<DT_, D_, CODED_E4M3>), grid, wg, 0, st, a, blocks);                    \
    } while (0)
    TKA_BY_TYPE_AND_DIM(TKA_READ, a.dtype, a.D);
#undef TKA_READ
    return hipGetLastError();
}

}  // namespace tka
