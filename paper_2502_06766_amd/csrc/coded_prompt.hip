// Attention of the tokens of a prompt over the 8-bit cache (prompt.h has the kernel).
#include "prompt.h"

namespace tka {

hipError_t launch_prompt_coded(const PromptCall& a, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.S * a.Hkv * a.n_split * a.row_blocks));
#define TKA_PROMPT_(DT_, D_, FMT_)                                                                                        \
    do {                                                                                                                  \
        if (a.chunk > kFoldTiles<DT_, true>) hipLaunchKernelGGL((prompt_kernel<DT_, FMT_, D_, 4, true>), grid, dim3(256), 0, st, a); \
        else hipLaunchKernelGGL((prompt_kernel<DT_, FMT_, D_, 4, false>), grid, dim3(256), 0, st, a);                     \
    } while (0)
#define TKA_PROMPT(DT_, D_)                                                                                               \
    do {                                                                                                                  \
        if (a.format == CODED_INT8) TKA_PROMPT_(DT_, D_, CODED_INT8);                                                     \
        else TKA_PROMPT_(DT_, D_, CODED_E4M3);                                                                            \
    } while (0)
    TKA_BY_TYPE_AND_DIM(TKA_PROMPT, a.dtype, a.D);
#undef TKA_PROMPT
#undef TKA_PROMPT_
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || a.n_split == 1 ? e : launch_prompt_join(a, st);
}

}  // namespace tka
