// Attention of the tokens of a prompt over a cache in its own type (prompt.h has the kernel), and the joint of split keys.
#include "prompt.h"

namespace tka {

// out and lse of rows whose keys were split: D / 4 threads a row.
template <int DT>
__global__ void __launch_bounds__(256) prompt_join_kernel(PromptCall a) {
    const int per = a.D / 4, slots = 256 / per;
    const int64_t total = (int64_t)a.S * a.Hkv * a.row_blocks * a.block_rows;
    const int64_t i = (int64_t)blockIdx.x * slots + (int)threadIdx.x / per;
    const int c = 4 * ((int)threadIdx.x % per);
    if (i >= total) return;
    const int64_t unit = i / a.block_rows;
    const int at = (int)(i - unit * a.block_rows), rb = (int)(unit % a.row_blocks), stream = (int)(unit / a.row_blocks);
    const int row = rb * a.block_rows + at;
    if (row >= (int)a.M * a.G) return;
    const int m = row / a.G, b = stream / a.Hkv, kvh = stream - b * a.Hkv;
    const int64_t to = ((int64_t)b * a.M + m) * a.Hq + kvh * a.G + (row - m * a.G);
    const float* const lm = a.part_lm + 2 * (unit * a.n_split * a.block_rows + at);
    const float* const acc = a.part_acc + (unit * a.n_split * a.block_rows + at) * a.D + c;
    float top = -INFINITY;
    for (int s = 0; s < a.n_split; ++s) top = fmaxf(top, lm[2 * s * a.block_rows + 1]);
    float l = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.n_split; ++s) {
        const float ms = lm[2 * s * a.block_rows + 1];
        if (ms == -INFINITY) continue;                               // (no key that the row sees)
        const float f = __builtin_amdgcn_exp2f(ms - top);
        l = fmaf(f, lm[2 * s * a.block_rows], l);
        const f32x4 x = *reinterpret_cast<const f32x4*>(acc + (int64_t)s * a.block_rows * a.D);
#pragma unroll
        for (int y = 0; y < 4; ++y) sum[y] = fmaf(f, x[y], sum[y]);
    }
    const float inv = 1.0f / l;
    if (DT == DT_F32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to * a.D + c) = sum * inv;
    } else {
        using E = typename std::conditional<DT == DT_F16, _Float16, __bf16>::type;
        typedef E e4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<e4*>(static_cast<E*>(a.out) + to * a.D + c) =
            e4{(E)(sum[0] * inv), (E)(sum[1] * inv), (E)(sum[2] * inv), (E)(sum[3] * inv)};
    }
    if (c == 0 && a.lse) a.lse[to] = (top + log2f(l)) * 0.69314718055994531f;
}

hipError_t launch_prompt_join(const PromptCall& a, hipStream_t st) {
    const int slots = 256 / (a.D / 4);
    const int64_t total = (int64_t)a.S * a.Hkv * a.row_blocks * a.block_rows;
    const dim3 grid((unsigned)((total + slots - 1) / slots)), wg(256);
    if (a.dtype == DT_F32) hipLaunchKernelGGL(prompt_join_kernel<DT_F32>, grid, wg, 0, st, a);
    else if (a.dtype == DT_F16) hipLaunchKernelGGL(prompt_join_kernel<DT_F16>, grid, wg, 0, st, a);
    else hipLaunchKernelGGL(prompt_join_kernel<DT_BF16>, grid, wg, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_prompt(const PromptCall& a, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.S * a.Hkv * a.n_split * a.row_blocks));
#define TKA_PROMPT(DT_, D_)                                                                                               \
    do {                                                                                                                  \
        if (a.block_rows == 32) hipLaunchKernelGGL((prompt_kernel<DT_, -1, D_, 1>), grid, dim3(64), 0, st, a);              \
        else hipLaunchKernelGGL((prompt_kernel<DT_, -1, D_, 4>), grid, dim3(256), 0, st, a);                               \
    } while (0)
    TKA_BY_TYPE_AND_DIM(TKA_PROMPT, a.dtype, a.D);
#undef TKA_PROMPT
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || a.n_split == 1 ? e : launch_prompt_join(a, st);
}

}  // namespace tka
