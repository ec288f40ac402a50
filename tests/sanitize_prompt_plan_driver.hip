// Plans of prompts whose window is as wide as 64 bits, for the sanitizer run (tests/test_prompt_isa_cpu.py): the same as with a window of the whole sequence.
#include <stdio.h>

#include <algorithm>

#include "../paper_2502_06766_amd/csrc/prompt.h"

int main() {
    int failures = 0;
    for (const int64_t n : {(int64_t)1, (int64_t)31, (int64_t)64, (int64_t)1000, (int64_t)0x7FFFFF00})
        for (const int64_t M : {(int64_t)1, (int64_t)8, (int64_t)33})
            for (const int G : {1, 4, 128})
                for (const int dtype : {tka::DT_F32, tka::DT_F16}) {
                    if (M > n) continue;
                    int chunk[4], splits[4], i = 0;
                    for (const int64_t window : {n, (int64_t)1 << 62, INT64_MAX - 1, INT64_MAX}) {
                        tka::PromptCall a{};
                        const int64_t len[2] = {n, std::max<int64_t>(M, n / 2)};
                        a.M = M; a.S = 2; a.Hq = G; a.Hkv = 1; a.G = G; a.D = 64; a.dtype = dtype; a.format = -1; a.sinks = window; a.window = window;
                        tka::plan_prompt(&a, len, (size_t)1 << 30, 256);
                        chunk[i] = a.chunk;
                        splits[i++] = a.n_split;
                    }
                    for (int x = 1; x < 4; ++x)
                        if (chunk[x] != chunk[0] || splits[x] != splits[0]) {
                            printf("plan driver: %lld tokens, %lld queries, %d heads: %d tiles in place of %d\n", (long long)n, (long long)M, G, chunk[x], chunk[0]);
                            ++failures;
                        }
                }
    if (!failures) printf("plan driver: done\n");
    return failures != 0;
}
