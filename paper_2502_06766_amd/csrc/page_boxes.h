// Block index of the block-sparse decode: per page of 64 consecutive tokens the smallest and the largest key, channel by
// channel (lo, hi, both exact: a minimum rounds nothing).  With them sum_c max(q_c lo_c, q_c hi_c) bounds q . k for every key k of
// the page from above, whatever the signs.  Kept where keys are written (api.hip, rotary.hip, evict.hip).
#pragma once
#include "device_utils.h"
#include "internal.h"
#include "ops.h"

namespace tka {

// the value as the storage type holds it (an element of it, so nothing is rounded)
template <int DT>
__device__ __forceinline__ uint32_t stored_bits(float v) {
    if (DT == DT_F16) return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v);
    return __float_as_uint(v) >> (DT == DT_BF16 ? 16 : 0);
}

// Boxes of every page that rows [row0, row0 + n_new) touch, from all rows the page holds then (one read of at most 64 rows; the row0 of a
// batched append is the sequence's length).  n_new < 0: of all rows below the length.  One wave per page, bound by the read of the keys.
// A NaN in a key makes both edges of its channel NaN.
template <int DT, int D>
__global__ void __launch_bounds__(256)
page_box_kernel(const char* __restrict__ K, int64_t Ncap, int64_t Pcap, int Hkv, const int32_t* __restrict__ len_dev, int64_t row0_host,
                int64_t n_new, char* __restrict__ boxes) {
    constexpr int EPL = Elem<DT>::kPerLoad, LPR = D / EPL, RPW = kWave / LPR, U = 64 / RPW < 8 ? 64 / RPW : 8;
    constexpr int ROW = D * Elem<DT>::kBytes;
    const int lane = lane_id(), wave = threadIdx.x >> 6, kvh = blockIdx.y, b = blockIdx.z;
    const int64_t at = len_dev ? (int64_t)len_dev[b] : row0_host;
    const int64_t row0 = n_new < 0 ? 0 : at, n_total = n_new < 0 ? at : at + n_new;
    const int64_t page = row0 / 64 + (int64_t)blockIdx.x * 4 + wave;
    if (page * 64 >= n_total) return;
    const int n = (int)(n_total - page * 64 < 64 ? n_total - page * 64 : 64);
    const int rs = lane / LPR, c = lane % LPR;
    const int64_t head = (int64_t)b * Hkv + kvh;
    const char* rows = K + (head * Ncap + page * 64) * ROW + c * 16;
    float lo[EPL], hi[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
    for (int r0 = 0; r0 < n; r0 += U * RPW) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {                    // (past the end: the page's last row again)
            const int r = r0 + u * RPW + rs;
            raw[u] = *reinterpret_cast<const u32x4*>(rows + (int64_t)(r < n ? r : n - 1) * ROW);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float k[EPL];
            Elem<DT>::widen(raw[u], k);
#pragma unroll
            for (int e = 0; e < EPL; ++e) { lo[e] = __builtin_elementwise_minimum(lo[e], k[e]); hi[e] = __builtin_elementwise_maximum(hi[e], k[e]); }
        }
    }
#pragma unroll
    for (int o = LPR; o < kWave; o <<= 1) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            lo[e] = __builtin_elementwise_minimum(lo[e], wave_xor(lo[e], o));
            hi[e] = __builtin_elementwise_maximum(hi[e], wave_xor(hi[e], o));
        }
    }
    if (rs == 0) {
        char* out = boxes + (head * Pcap + page) * 2 * ROW + c * 16;
        uint32_t a[4], z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (DT == DT_F32) {
                a[i] = stored_bits<DT>(lo[i]); z[i] = stored_bits<DT>(hi[i]);
            } else {
                a[i] = stored_bits<DT>(lo[2 * i]) | (stored_bits<DT>(lo[(2 * i + 1) % EPL]) << 16);
                z[i] = stored_bits<DT>(hi[2 * i]) | (stored_bits<DT>(hi[(2 * i + 1) % EPL]) << 16);
            }
        }
        *reinterpret_cast<u32x4*>(out) = u32x4{a[0], a[1], a[2], a[3]};
        *reinterpret_cast<u32x4*>(out + ROW) = u32x4{z[0], z[1], z[2], z[3]};
    }
}

// n_new < 0: the boxes of `max_rows` = -n_new rows at most, as many as the device lengths say.
inline hipError_t launch_page_boxes(int dtype, int D, const void* K, int64_t Ncap, int64_t Pcap, int Hkv, int B, const int32_t* len_dev,
                                    int64_t row0, int64_t n_new, void* boxes, hipStream_t st) {
    if (n_new == 0) return hipSuccess;
    const int64_t pages = n_new < 0 ? (63 - n_new) / 64 : (n_new + 63) / 64 + 1;      // (the first page touched may be a partly filled one)
    const dim3 grid((unsigned)((pages + 3) / 4), (unsigned)Hkv, (unsigned)B);
#define TKA_BOX(DT_, D_)                                                                                                          \
    hipLaunchKernelGGL((page_box_kernel<DT_, D_>), grid, dim3(256), 0, st, static_cast<const char*>(K), Ncap, Pcap, Hkv, len_dev, \
                       row0, n_new, static_cast<char*>(boxes))
    TKA_BY_TYPE_AND_DIM(TKA_BOX, dtype, D);
#undef TKA_BOX
    return hipGetLastError();
}

}  // namespace tka
