// Host side of topk_attn_add_mass for the sanitizer run (tests/test_operator_edges_cpu.py): api_ops.hip linked with stand-ins for the kernel
// launchers, over a handle put together here.  A check that fails prints a line and makes the exit status 1.
#include <limits.h>
#include <stdio.h>

#include "../include/topk_attn.h"
#include "../paper_2502_06766_amd/csrc/handle.h"
#include "../paper_2502_06766_amd/csrc/internal.h"
#include "../paper_2502_06766_amd/csrc/ops.h"

static int failures = 0, largest = 0;
#define CHECK(cond)                                                      \
    do {                                                                 \
        if (!(cond)) {                                                   \
            printf("mass driver: line %d: %s\n", __LINE__, #cond);       \
            ++failures;                                                  \
        }                                                                \
    } while (0)

extern "C" hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }

namespace tka {
hipError_t launch_add_mass(const MassCall& a, hipStream_t) {
    // (the kernel counts to less than 8192 entries behind the last one)
    CHECK((int64_t)a.k + 8 * 1024 <= INT_MAX);
    if (a.k > largest) largest = a.k;
    return hipSuccess;
}
hipError_t launch_attend(const AttendCall&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_block_scores(const BlockCall&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_block_select(const BlockCall&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_rotary(const RotaryCall&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_evict(const EvictCall&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_balls_again(int, int, const void*, int64_t, int64_t, int, int, const int32_t*, int64_t, void*, float*, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_page_balls(int, int, const void*, int64_t, int64_t, int, int, const int32_t*, int64_t, int64_t, void*, float*, hipStream_t) { return hipErrorUnknown; }
}  // namespace tka

int main() {
    topk_attn h{};
    topk_attn_config& c = h.cfg;
    c.struct_size = sizeof c;
    c.n_layers = 1; c.n_seqs = 1; c.n_q_heads = 4; c.n_kv_heads = 1; c.head_dim = 64; c.max_tokens = 1000; c.max_k = 64; c.dtype = TOPK_ATTN_F16;
    h.len.assign(1, 100);
    int32_t* idx = reinterpret_cast<int32_t*>(0x40000);
    float* f = reinterpret_cast<float*>(0x50000);
    for (int k : {1, 64, 4096, 4097, 1 << 28}) CHECK(topk_attn_add_mass(&h, 0, idx, f, f, k, f, nullptr) == TOPK_ATTN_OK);
    for (int k : {0, -1, INT_MIN, (1 << 28) + 1, INT_MAX - 4096, INT_MAX}) CHECK(topk_attn_add_mass(&h, 0, idx, f, f, k, f, nullptr) == TOPK_ATTN_EINVAL);
    CHECK(largest == 1 << 28);
    if (failures == 0) printf("mass driver: all checks passed\n");
    return failures ? 1 : 0;
}
