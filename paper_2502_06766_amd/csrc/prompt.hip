// Attention of the tokens of a prompt over a cache in its own type (prompt.h has the kernel), and the joint of split keys.
#include "prompt.h"

namespace tka {

// out and lse of rows whose keys were split: D / 4 lanes a row, a wave a workgroup.  (Few rows have many splits: their factors are worked out at once, and 16 of their
// sums are on their way at a time.)
template <int DT>
__global__ void __launch_bounds__(64) prompt_join_kernel(PromptCall a) {
    __shared__ float factor[8][kPromptSplits];
    const int per = a.D / 4, slots = 64 / per, lane = lane_id(), slot = lane / per, c = 4 * (lane % per);
    const int64_t total = (int64_t)a.S * a.Hkv * a.row_blocks * a.block_rows;
    const int64_t i = (int64_t)blockIdx.x * slots + slot;
    const int64_t unit = (i < total ? i : total - 1) / a.block_rows;
    const int at = (int)((i < total ? i : total - 1) - unit * a.block_rows);
    const float* const lm = a.part_lm + 2 * (unit * a.n_split * a.block_rows + at);
    // the row's lanes take splits in turn
    constexpr int U = kPromptSplits / 8;                             // (of the fewest lanes a row has)
    float l[U], m[U], top = -INFINITY, sum_l = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int s = lane % per + u * per;
        l[u] = 0.f; m[u] = -INFINITY;
        if (u * per < a.n_split && s < a.n_split) {
            const float2 x = *reinterpret_cast<const float2*>(lm + 2 * (int64_t)s * a.block_rows);
            l[u] = x.x; m[u] = x.y;
        }
        top = fmaxf(top, m[u]);
    }
    for (int o = per / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int s = lane % per + u * per;
        const float f = m[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[u] - top);       // (no key that the row sees)
        if (f != 0.f) sum_l = fmaf(f, l[u], sum_l);
        if (s < a.n_split) factor[slot][s] = f;
    }
    for (int o = per / 2; o; o >>= 1) sum_l += __shfl_xor(sum_l, o, 64);
    __syncthreads();
    const float* const acc = a.part_acc + (unit * a.n_split * a.block_rows + at) * a.D + c;
    f32x4 sum[4] = {};
    for (int s0 = 0; s0 < a.n_split; s0 += 16) {
        f32x4 x[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) x[u] = *reinterpret_cast<const f32x4*>(acc + (int64_t)(s0 + u < a.n_split ? s0 + u : s0) * a.block_rows * a.D);
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const float f = s0 + u < a.n_split ? factor[slot][s0 + u] : 0.f;
            if (f != 0.f) {
#pragma unroll
                for (int y = 0; y < 4; ++y) sum[u & 3][y] = fmaf(f, x[u][y], sum[u & 3][y]);
            }
        }
    }
    const int rb = (int)(unit % a.row_blocks), stream = (int)(unit / a.row_blocks), row = rb * a.block_rows + at;
    if (i >= total || row >= (int)a.M * a.G) return;
    const int q = row / a.G, b = stream / a.Hkv, kvh = stream - b * a.Hkv;
    const int64_t to = ((int64_t)b * a.M + q) * a.Hq + kvh * a.G + (row - q * a.G);
    const f32x4 all = ((sum[0] + sum[1]) + (sum[2] + sum[3])) * (1.0f / sum_l);
    if (DT == DT_F32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to * a.D + c) = all;
    } else {
        using E = typename std::conditional<DT == DT_F16, _Float16, __bf16>::type;
        typedef E e4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<e4*>(static_cast<E*>(a.out) + to * a.D + c) = e4{(E)all[0], (E)all[1], (E)all[2], (E)all[3]};
    }
    if (c == 0 && a.lse) a.lse[to] = (top + log2f(sum_l)) * 0.69314718055994531f;
}

hipError_t launch_prompt_join(const PromptCall& a, hipStream_t st) {
    const int slots = 64 / (a.D / 4);
    const int64_t total = (int64_t)a.S * a.Hkv * a.row_blocks * a.block_rows;
    const dim3 grid((unsigned)((total + slots - 1) / slots)), wg(64);
    if (a.dtype == DT_F32) hipLaunchKernelGGL(prompt_join_kernel<DT_F32>, grid, wg, 0, st, a);
    else if (a.dtype == DT_F16) hipLaunchKernelGGL(prompt_join_kernel<DT_F16>, grid, wg, 0, st, a);
    else hipLaunchKernelGGL(prompt_join_kernel<DT_BF16>, grid, wg, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_prompt(const PromptCall& a, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.S * a.Hkv * a.n_split * a.row_blocks));
#define TKA_PROMPT_(DT_, D_, NW_)                                                                                         \
    do {                                                                                                                  \
        if (a.chunk > kFoldTiles<DT_, false>) hipLaunchKernelGGL((prompt_kernel<DT_, -1, D_, NW_, true>), grid, dim3(64 * NW_), 0, st, a); \
        else hipLaunchKernelGGL((prompt_kernel<DT_, -1, D_, NW_, false>), grid, dim3(64 * NW_), 0, st, a);                \
    } while (0)
#define TKA_PROMPT(DT_, D_)                                                                                               \
    do {                                                                                                                  \
        if constexpr (DT_ != DT_F32) {                                                                                    \
            if (a.block_rows == 32) {                                                                                     \
                TKA_PROMPT_(DT_, D_, 1);                                                                                  \
                break;                                                                                                    \
            }                                                                                                             \
        }                                                                                                                 \
        TKA_PROMPT_(DT_, D_, 4);                                                                                          \
    } while (0)
    TKA_BY_TYPE_AND_DIM(TKA_PROMPT, a.dtype, a.D);
#undef TKA_PROMPT
#undef TKA_PROMPT_
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || a.n_split == 1 ? e : launch_prompt_join(a, st);
}

}  // namespace tka
