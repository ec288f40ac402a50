// Host-side walk through the entry points of the 8-bit cache and of prompts for the sanitizer run (tests/test_coded_cpu.py): api_coded.hip and
// api_prompt.hip are linked with stand-ins for the kernel launchers, which check what they are handed and report success.
// Every check that fails prints a line and makes the exit status 1.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "../include/topk_attn.h"
#include "../paper_2502_06766_amd/csrc/coded.h"
#include "../paper_2502_06766_amd/csrc/handle.h"
#include "../paper_2502_06766_amd/csrc/internal.h"
#include "../paper_2502_06766_amd/csrc/prompt.h"

static int failures = 0, launches = 0;
#define CHECK(cond)                                                      \
    do {                                                                 \
        if (!(cond)) {                                                   \
            if (failures < 20) printf("coded driver: line %d: %s\n", __LINE__, #cond); \
            ++failures;                                                  \
        }                                                                \
    } while (0)

// stands in for the device: none, or one that is always current
static bool have_device = false;
extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return have_device ? hipSuccess : hipErrorNoDevice; }
hipError_t hipMemset(void*, int, size_t) { return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int) { memset(p, 0, sizeof *p); p->multiProcessorCount = 256; return hipSuccess; }
}

static char* const kv = reinterpret_cast<char*>((uintptr_t)1 << 46);         // (memory that nothing here touches)
static char* const ws = reinterpret_cast<char*>((uintptr_t)1 << 47);
static char* const rows = reinterpret_cast<char*>((uintptr_t)1 << 40);
static topk_attn_coded_config cfg;
static bool within(const void* p, double bytes, const char* base, size_t room) {
    const char* c = static_cast<const char*>(p);
    return c >= base && (double)(c - base) + bytes <= (double)room;
}
static size_t prompt_room;                   // bytes for a plain cache's partial sums, from `ws` on
static int64_t longest_tiles, most_blocks;
static int any_open;
static std::vector<int64_t> lens;            // of the layer
static int64_t walk_sinks;
static void find_longest(int64_t reach) {
    most_blocks = any_open = 0;
    for (int64_t n : lens) {
        const tka::CodedWalk w(n, walk_sinks, reach);
        most_blocks = std::max(most_blocks, w.blocks());
        any_open |= w.open();
    }
}

namespace tka {
static void check_arrays(const CodedArrays& a, int streams) {
    const double e = cfg.dtype == TOPK_ATTN_F32 ? 4 : 2;
    for (int i = 0; i < 2; ++i) CHECK(within(a.codes[i], (double)streams * a.blocks * 64 * cfg.head_dim, kv, cfg.kv_bytes));
    CHECK(within(a.scales, (double)streams * a.blocks * 8, kv, cfg.kv_bytes));
    CHECK(within(a.open, (double)streams * 128 * cfg.head_dim * e, kv, cfg.kv_bytes));
    CHECK(within(a.len, 4, ws, cfg.workspace_bytes) && a.blocks == cfg.max_tokens / 64);
}
hipError_t launch_coded_append(const CodedAppendCall& a, hipStream_t) {
    ++launches;
    check_arrays(a.a, a.B * a.Hkv);
    CHECK(a.B >= 1 && a.B <= kCodedSeqs && a.n >= 1 && a.wgs >= 1);
    for (int b = 0; b < a.B; ++b) {
        CHECK(a.base[b] >= 0 && a.base[b] + a.n <= cfg.max_tokens);
        CHECK((a.base[b] + a.n) / 64 - a.base[b] / 64 <= a.wgs);
    }
    CHECK((double)a.B * a.Hkv * 2 * a.wgs <= (double)kMostWorkgroups);
    return hipSuccess;
}
hipError_t launch_coded_read(const CodedReadCall& a, hipStream_t) {
    ++launches;
    check_arrays(a.a, a.B * a.Hkv);
    CHECK(a.first >= 0 && a.n >= 1 && a.first + a.n <= cfg.max_tokens);
    return hipSuccess;
}
hipError_t launch_coded_decode(const CodedDecodeCall& a, hipStream_t) {
    ++launches;
    check_arrays(a.a, a.B * a.Hkv);
    CHECK(a.chunk >= 1 && a.n_split >= 1 && a.n_split <= kMaxSplits && a.window >= 1);
    CHECK(a.rows == (a.M ? a.M * a.G : a.G) && a.row_blocks == (a.rows + 15) / 16 && a.reach >= a.window - (a.window > ((int64_t)1 << 40) ? a.window : 0));
    const double heads = (double)a.B * a.Hkv * a.rows * a.n_split;
    CHECK(within(a.part_acc, heads * a.D * 4, ws, cfg.workspace_bytes) && within(a.part_lm, heads * 8, ws, cfg.workspace_bytes));
    CHECK((char*)a.part_lm == (char*)a.part_acc + (size_t)a.B * a.Hkv * a.rows * a.n_split * a.D * 4);
    CHECK(within(a.arrive, (double)a.B * a.Hkv * a.row_blocks * 4, ws, (char*)a.part_acc - ws));
    if (a.M) find_longest(a.reach);
    CHECK((int64_t)(a.n_split - any_open) * a.chunk >= most_blocks && (int64_t)(a.n_split - any_open - 1) * a.chunk < std::max<int64_t>(most_blocks, 1));
    return hipSuccess;
}
static void check_prompt(const PromptCall& a, size_t room) {
    ++launches;
    const int64_t rows_ = a.M * a.G;
    CHECK(a.block_rows == 32 || a.block_rows == 128);
    CHECK((int64_t)a.row_blocks * a.block_rows >= rows_ && (int64_t)(a.row_blocks - 1) * a.block_rows < rows_);
    CHECK(a.n_split >= 1 && a.n_split <= kPromptSplits && a.chunk >= 1);
    if (a.n_split > 1) {
        CHECK((int64_t)a.n_split * a.chunk >= longest_tiles);
        const double slots = (double)a.S * a.Hkv * a.row_blocks * a.n_split * a.block_rows;
        CHECK(within(a.part_acc, slots * a.D * 4, ws, room) && within(a.part_lm, slots * 8, ws, room));
    }
}
hipError_t launch_attend(const AttendCall& a, hipStream_t) {
    ++launches;
    CHECK(a.M >= 1 && a.rows == a.M * a.G && a.rows <= kFewRowsF32 && a.dtype == TOPK_ATTN_F32 && a.row_blocks == (a.rows + 15) / 16 && a.chunk >= 1 && a.n_split >= 1 && a.n_split <= kMaxSplits);
    int64_t pages = 0;
    for (int64_t n : lens) pages = std::max(pages, tka::WindowWalk(n, walk_sinks, a.reach).pages());
    CHECK((int64_t)a.n_split * a.chunk >= pages && (int64_t)(a.n_split - 1) * a.chunk < pages);
    const double heads = (double)a.B * a.Hkv * a.rows * a.n_split;
    CHECK(within(a.part_acc, heads * a.D * 4, ws, prompt_room) && within(a.part_lm, heads * 8, ws, prompt_room));
    CHECK((char*)a.part_lm == (char*)a.part_acc + (size_t)a.B * a.Hkv * a.rows * a.n_split * a.D * 4);
    return hipSuccess;
}
hipError_t launch_prompt(const PromptCall& a, hipStream_t) { check_prompt(a, prompt_room); return hipSuccess; }
hipError_t launch_prompt_coded(const PromptCall& a, hipStream_t) { check_prompt(a, cfg.workspace_bytes); return hipSuccess; }
}  // namespace tka

static void config(int B, int Hq, int Hkv, int D, int64_t cap, int dtype, int format, int layers) {
    memset(&cfg, 0, sizeof cfg);
    cfg.struct_size = sizeof cfg;
    cfg.n_layers = layers; cfg.n_seqs = B; cfg.n_q_heads = Hq; cfg.n_kv_heads = Hkv; cfg.head_dim = D; cfg.max_tokens = cap; cfg.dtype = dtype; cfg.format = format;
    cfg.kv_storage = kv; cfg.workspace = ws;
    cfg.kv_bytes = topk_attn_coded_kv_bytes(&cfg);
    cfg.workspace_bytes = topk_attn_coded_workspace_bytes(&cfg);
}

int main() {
    float* const fp = reinterpret_cast<float*>(rows);
    topk_attn_coded_t* h = nullptr;
    // refusals of the configuration, before anything is touched
    config(2, 8, 2, 64, 1000, TOPK_ATTN_F16, TOPK_ATTN_CODED_INT8, 2);
    CHECK(cfg.kv_bytes && cfg.workspace_bytes);
    CHECK(topk_attn_coded_create(&cfg, nullptr) == TOPK_ATTN_EINVAL);
    CHECK(topk_attn_coded_create(&cfg, &h) == TOPK_ATTN_EDEVICE && !h);
    const auto refuse = [&](auto change, int code) {
        topk_attn_coded_config c = cfg;
        change(c);
        CHECK(topk_attn_coded_create(&c, &h) == code && !h);
    };
    refuse([](auto& c) { c.struct_size -= 4; }, TOPK_ATTN_EINVAL);
    refuse([](auto& c) { c.n_layers = 0; }, TOPK_ATTN_EINVAL);
    refuse([](auto& c) { c.max_tokens = 0; }, TOPK_ATTN_EINVAL);
    refuse([](auto& c) { c.max_tokens = (int64_t)1 << 31; }, TOPK_ATTN_EINVAL);
    refuse([](auto& c) { c.kv_storage = nullptr; }, TOPK_ATTN_EINVAL);
    refuse([](auto& c) { c.workspace = ws + 16; }, TOPK_ATTN_EINVAL);
    refuse([](auto& c) { c.head_dim = 96; }, TOPK_ATTN_EUNSUPPORTED);
    refuse([](auto& c) { c.dtype = 3; }, TOPK_ATTN_EUNSUPPORTED);
    refuse([](auto& c) { c.format = 2; }, TOPK_ATTN_EUNSUPPORTED);
    refuse([](auto& c) { c.n_q_heads = 7; }, TOPK_ATTN_EUNSUPPORTED);
    refuse([](auto& c) { c.n_q_heads = 2 * 129; }, TOPK_ATTN_EUNSUPPORTED);
    refuse([](auto& c) { c.n_seqs = 65535; c.n_kv_heads = c.n_q_heads = 65; }, TOPK_ATTN_EUNSUPPORTED);
    refuse([](auto& c) { c.kv_bytes -= 1; }, TOPK_ATTN_ENOMEM);
    refuse([](auto& c) { c.workspace_bytes -= 1; }, TOPK_ATTN_ENOMEM);
    have_device = true;
    CHECK(topk_attn_coded_create(&cfg, &h) == TOPK_ATTN_OK && h);
    // refusals of the calls leave the handle as it is
    CHECK(topk_attn_coded_append(h, 0, 0, rows, rows, 100, 0, 128, 64, nullptr) == TOPK_ATTN_OK);
    const int before = launches;
    for (int64_t n : {(int64_t)901, INT64_MAX, (int64_t)1 << 40}) {
        CHECK(topk_attn_coded_append(h, 0, 0, rows, rows, n, 0, 128, 64, nullptr) == TOPK_ATTN_ECAPACITY);
        CHECK(topk_attn_coded_read(h, 0, 0, 0, n, rows, rows, 0, 128, 64, nullptr) == TOPK_ATTN_EINVAL);
        CHECK(topk_attn_coded_read(h, 0, 0, n, n, rows, rows, 0, 128, 64, nullptr) == TOPK_ATTN_EINVAL);
        CHECK(topk_attn_coded_prompt(h, 0, 0, rows, n, 0, 1, rows, nullptr, nullptr) == TOPK_ATTN_EINVAL);
    }
    for (int64_t s : {INT64_MAX, INT64_MAX - 7, INT64_MIN, (int64_t)-8, (int64_t)4}) {
        CHECK(topk_attn_coded_append(h, 0, 0, rows, rows, 1, s, 128, 64, nullptr) == TOPK_ATTN_EINVAL);
        CHECK(topk_attn_coded_append(h, 0, 0, rows, rows, 1, 0, s, 64, nullptr) == TOPK_ATTN_EINVAL);
        CHECK(topk_attn_coded_append(h, 0, 0, rows, rows, 1, 0, 128, s, nullptr) == TOPK_ATTN_EINVAL);
        CHECK(topk_attn_coded_read(h, 0, 0, 0, 1, rows, rows, 0, s, 64, nullptr) == TOPK_ATTN_EINVAL);
    }
    CHECK(topk_attn_coded_decode(h, 0, rows, 0, 5, fp, nullptr, nullptr) == TOPK_ATTN_EINVAL);          // an empty sequence
    CHECK(topk_attn_coded_decode(h, 0, rows, 0, 0, fp, nullptr, nullptr) == TOPK_ATTN_EINVAL);
    CHECK(topk_attn_coded_decode(h, 0, rows, INT64_MIN, 1, fp, nullptr, nullptr) == TOPK_ATTN_EINVAL);
    CHECK(topk_attn_coded_decode(h, 2, rows, 0, 1, fp, nullptr, nullptr) == TOPK_ATTN_EINVAL);
    CHECK(topk_attn_coded_prompt(h, 0, -1, rows, 1, 0, 1, rows, nullptr, nullptr) == TOPK_ATTN_EINVAL);
    CHECK(topk_attn_coded_reset(h, 0, 2, nullptr) == TOPK_ATTN_EINVAL && topk_attn_coded_reset(h, 2, -1, nullptr) == TOPK_ATTN_EINVAL);
    CHECK(topk_attn_coded_length(h, 0, 0) == 100 && topk_attn_coded_length(h, 0, 1) == 0 && topk_attn_coded_length(h, 0, 2) == -1 && launches == before);
    CHECK(topk_attn_coded_destroy(h) == TOPK_ATTN_OK);
    // plans over shapes, lengths and windows: what is handed to the launchers is checked there
    uint32_t seed = 4711;
    const auto rnd = [&](uint32_t n) { seed = seed * 1664525u + 1013904223u; return (seed >> 8) % n; };
    const auto part = [&](int64_t n) { return (int64_t)(rnd(1 << 24) / 16777216.0 * (double)n); };
    for (int i = 0; i < 1500; ++i) {
        const int Hkv = 1 + (int)rnd(9), G = rnd(4) ? 1 + (int)rnd(16) : 1 + (int)rnd(128), B = rnd(3) ? 1 + (int)rnd(4) : 1 + (int)rnd(200), D = 32 << rnd(4);
        const int64_t cap = rnd(8) ? 1 + rnd(200000) : 1 + (int64_t)rnd(1 << 24) * 100;
        config(B, Hkv * G, Hkv, D, cap, (int)rnd(3), (int)rnd(2), 2);
        CHECK(topk_attn_coded_create(&cfg, &h) == TOPK_ATTN_OK);
        if (!h) continue;
        std::vector<int64_t> len(B);
        bool there = true;
        for (int b = 0; b < B; ++b) {
            const int64_t n = rnd(2) ? cap : 1 + part(cap);
            int rc = topk_attn_coded_append(h, 1, b, rows, rows, n, 0, D, D, nullptr);
            CHECK(rc == TOPK_ATTN_OK || (rc == TOPK_ATTN_EUNSUPPORTED && (double)Hkv * 2 * n / 64 > 15e6));
            there = there && rc == TOPK_ATTN_OK;
            len[b] = topk_attn_coded_length(h, 1, b);
        }
        int64_t least = INT64_MAX;
        for (int64_t n : len) least = std::min(least, n);
        const int64_t sinks = rnd(2) ? 0 : part(2 * cap), window = rnd(2) ? (int64_t)1 << 62 : 1 + part(cap);
        lens = len; walk_sinks = sinks;
        find_longest(window);
        if (there) {
            CHECK(topk_attn_coded_decode(h, 1, rows, sinks, window, fp, fp, nullptr) == TOPK_ATTN_OK);
            const int64_t M = rnd(2) ? 1 + part(std::min<int64_t>(least, 70)) : 1 + part(least);
            longest_tiles = 0;
            for (int64_t n : len) longest_tiles = std::max(longest_tiles, tka::prompt_tiles(n, 1, sinks, window));
            int rc = topk_attn_coded_prompt(h, 1, -1, rows, M, sinks, window, rows, nullptr, nullptr);
            CHECK(rc == TOPK_ATTN_OK || (rc == TOPK_ATTN_EUNSUPPORTED && (double)B * Hkv * M * G > 1e9));
            // the same over a plain cache
            topk_attn p{};
            p.cfg.n_layers = 2; p.cfg.n_seqs = B; p.cfg.n_q_heads = Hkv * G; p.cfg.n_kv_heads = Hkv; p.cfg.head_dim = D; p.cfg.max_tokens = cap; p.cfg.dtype = cfg.dtype;
            p.cfg.kv_storage = kv; p.cfg.workspace = ws;
            p.ws.cand_cap = 16384 << rnd(3);
            p.n_cu = 256;
            p.len.assign(2 * B, 0);
            std::copy(len.begin(), len.end(), p.len.begin() + B);
            prompt_room = (size_t)B * Hkv * G * p.ws.cand_cap * 8;
            rc = topk_attn_prompt(&p, 1, -1, rows, M, sinks, window, rows, nullptr, nullptr);
            CHECK(rc == TOPK_ATTN_OK || (rc == TOPK_ATTN_EUNSUPPORTED && (double)B * Hkv * M * G > 1e9));
            const int64_t first = part(least), n = 1 + part(least - first);
            rc = topk_attn_coded_read(h, 1, -1, first, n, rows, rows, 0, D, D, nullptr);
            CHECK(rc == TOPK_ATTN_OK || (rc == TOPK_ATTN_EUNSUPPORTED && (double)B * Hkv * 2 * n / 64 > 14e6));
        }
        CHECK(topk_attn_coded_destroy(h) == TOPK_ATTN_OK);
    }
    CHECK(launches > 5000);
    if (failures == 0) printf("coded driver: all checks passed\n");
    return failures ? 1 : 0;
}
