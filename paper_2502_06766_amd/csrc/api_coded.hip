// C entries of the cache held in 8 bits (topk_attn_coded_*): handle, argument checks, launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "../../include/topk_attn.h"
#include "coded.h"
#include "handle.h"
#include "internal.h"
#include "prompt.h"
#include "split_plan.h"

using namespace tka;

struct topk_attn_coded {
    topk_attn_coded_config cfg;
    std::vector<int64_t> len;   // host mirror of the device lengths, [L][B]
    int n_cu;
};

namespace {

bool config_ok(const topk_attn_coded_config* c, int* why) {
    *why = TOPK_ATTN_EINVAL;
    if (!c || c->struct_size != sizeof(topk_attn_coded_config)) return false;
    if (c->n_layers < 1 || c->n_seqs < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1) return false;
    if (c->max_tokens < 1 || c->max_tokens > (int64_t)0x7FFFFF00 || c->device < 0) return false;
    if (c->n_seqs > 65535 || c->n_kv_heads > 65535) return false;
    *why = TOPK_ATTN_EUNSUPPORTED;
    if (c->dtype != TOPK_ATTN_F32 && c->dtype != TOPK_ATTN_F16 && c->dtype != TOPK_ATTN_BF16) return false;
    if (c->format != TOPK_ATTN_CODED_INT8 && c->format != TOPK_ATTN_CODED_E4M3) return false;
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return false;
    if (c->n_q_heads % c->n_kv_heads || c->n_q_heads / c->n_kv_heads > 128) return false;
    if ((int64_t)c->n_seqs * c->n_kv_heads > kMostStreams) return false;
    *why = TOPK_ATTN_OK;
    return true;
}

// Storage: key codes, value codes, scales, open rows, of all layers each.
struct Storage {
    size_t codes[2], scales, open, total;
    int64_t streams, blocks, layer_streams;
};
Storage storage_of(const topk_attn_coded_config* c) {
    Storage s;
    s.layer_streams = (int64_t)c->n_seqs * c->n_kv_heads;
    s.streams = c->n_layers * s.layer_streams;
    s.blocks = c->max_tokens / kCodedBlock;
    size_t o = 0;
    const auto take = [&](size_t bytes) { const size_t at = o; o = align_up(o + bytes); return at; };
    for (size_t& at : s.codes) at = take((size_t)s.streams * s.blocks * coded_block_bytes(c->head_dim));
    s.scales = take((size_t)s.streams * s.blocks * 2 * sizeof(float));
    s.open = take((size_t)s.streams * 2 * kCodedBlock * c->head_dim * elem_bytes(c->dtype));
    s.total = o;
    return s;
}

// Workspace: lengths, counters of the decode, partial sums.
struct Workspace {
    size_t len, arrive, parts, parts_bytes, total;
    int64_t max_splits;
};
Workspace workspace_of(const topk_attn_coded_config* c) {
    Workspace w;
    const int64_t G = c->n_q_heads / c->n_kv_heads, units = (int64_t)c->n_seqs * c->n_kv_heads * ((G + 15) / 16);
    const int64_t blocks = c->max_tokens / kCodedBlock;
    size_t o = 0;
    const auto take = [&](size_t bytes) { const size_t at = o; o = align_up(o + bytes); return at; };
    w.len = take((size_t)c->n_layers * c->n_seqs * sizeof(int32_t));
    w.arrive = take((size_t)c->n_seqs * c->n_kv_heads * (size_t)std::max<int64_t>((G + 15) / 16, kFewRows / 16) * sizeof(uint32_t));
    // splits that fill the chip, and no more than 256 blocks a split (64 a wave, whose sums follow each other); one of open rows
    w.max_splits = std::min<int64_t>(kMaxSplits, 1 + std::min<int64_t>(std::max<int64_t>(blocks, 1), std::max<int64_t>(4096 / units, blocks / 256) + 1));
    size_t parts = (size_t)c->n_seqs * c->n_q_heads * (size_t)w.max_splits * (c->head_dim + 2) * sizeof(float);
    // few rows of every stream of a long cache: splits of at most 1024 blocks (256 a wave, whose sums follow each other), and one of open rows; a hundredth of the cache at most
    if (blocks >= 1024)
        parts = std::max(parts, (size_t)c->n_seqs * c->n_kv_heads * (size_t)few_rows(c->dtype, c->head_dim) * (size_t)(blocks / 1024 + 2) * (c->head_dim + 2) * sizeof(float));
    // chunks of few rows whose keys are split: two workgroups of 128 rows on each of 256 compute units
    if (blocks >= 8) parts = std::max(parts, (size_t)512 * 128 * (c->head_dim + 2) * sizeof(float));
    w.parts = take(w.parts_bytes = parts);
    w.total = o;
    return w;
}

CodedArrays arrays_of(const topk_attn_coded* h, int layer, int seq) {
    const topk_attn_coded_config& c = h->cfg;
    const Storage s = storage_of(&c);
    const int64_t stream = layer * s.layer_streams + (int64_t)seq * c.n_kv_heads;
    char* const base = static_cast<char*>(c.kv_storage);
    CodedArrays a;
    for (int i = 0; i < 2; ++i) a.codes[i] = base + s.codes[i] + (size_t)stream * s.blocks * coded_block_bytes(c.head_dim);
    a.scales = reinterpret_cast<float*>(base + s.scales) + stream * s.blocks * 2;
    a.open = base + s.open + (size_t)stream * 2 * kCodedBlock * c.head_dim * elem_bytes(c.dtype);
    a.len = reinterpret_cast<int32_t*>(static_cast<char*>(c.workspace) + workspace_of(&c).len) + (size_t)layer * c.n_seqs + seq;
    a.blocks = s.blocks;
    return a;
}

bool range_ok(const topk_attn_coded_t* h, int layer, int seq) {
    return h && layer >= 0 && layer < h->cfg.n_layers && seq >= -1 && seq < h->cfg.n_seqs;
}
// strides in elements that a call's rows may have: pieces of 16 bytes, below 2^40 (times 65535 sequences they fit 64 bits)
bool strides_ok(int64_t seq, int64_t token, int64_t head, int e) {
    for (const int64_t x : {seq, token, head})
        if (x < 0 || x >= (int64_t)1 << 40 || ((x * e) & 15)) return false;
    return true;
}

// Splits of `rows` rows of each key stream that there is room for.
int64_t split_room(const topk_attn_coded_config& c, const Workspace& ws, int seqs, int64_t rows) {
    return (int64_t)(ws.parts_bytes / ((size_t)seqs * c.n_kv_heads * (size_t)rows * (c.head_dim + 2) * sizeof(float)));
}

// The kernel over few rows of each of B sequences from b0 on.
int decode_rows(topk_attn_coded* h, int layer, int b0, CodedDecodeCall a, void* hip_stream) {
    const topk_attn_coded_config& c = h->cfg;
    const int64_t* const len = &h->len[(size_t)layer * c.n_seqs + b0];
    int64_t longest = 0;
    int open = 0;
    for (int b = 0; b < a.B; ++b) {
        const CodedWalk w(len[b], a.sinks, a.reach);
        longest = std::max(longest, w.blocks());
        open |= w.open();
    }
    const Workspace ws = workspace_of(&c);
    a.a = arrays_of(h, layer, b0);
    a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype; a.format = c.format;
    a.row_blocks = (a.rows + 15) / 16;
    int64_t sample[16];                          // (of a larger batch some sequences stand for all)
    const int n_sample = std::min(a.B, 16);
    for (int i = 0; i < n_sample; ++i) sample[i] = std::max<int64_t>(1, CodedWalk(len[(int64_t)i * a.B / n_sample], a.sinks, a.reach).blocks());
    // splits that there is room for, one of them of open rows
    const int64_t most = std::min<int64_t>(a.M ? kMaxSplits : ws.max_splits, split_room(c, ws, a.B, a.rows)) - 1;
    a.chunk = longest ? (int)pages_per_split(sample, n_sample, (double)a.B / n_sample * a.Hkv * a.row_blocks, longest, most, h->n_cu, (double)c.head_dim) : 1;
    a.chunk = (int)std::min<int64_t>(a.chunk, std::max<int64_t>(256, (longest + most - 1) / most));
    a.n_split = (int)((longest + a.chunk - 1) / a.chunk) + open;
    char* const base = static_cast<char*>(c.workspace);
    a.part_acc = reinterpret_cast<float*>(base + ws.parts);
    a.part_lm = a.part_acc + (size_t)a.B * a.Hkv * a.rows * a.n_split * a.D;
    a.arrive = reinterpret_cast<uint32_t*>(base + ws.arrive);
    a.join_later = (int64_t)a.n_split * std::min(a.rows, 16) * a.D * 4 > kJoinBytes;
    if (coded_decode_wgs(a) > kMostWorkgroups || (int64_t)a.B * a.Hkv * a.rows > kMostWorkgroups) return TOPK_ATTN_EUNSUPPORTED;
    const DeviceOf device(c.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    return launch_coded_decode(a, (hipStream_t)hip_stream) == hipSuccess ? TOPK_ATTN_OK : TOPK_ATTN_EDEVICE;
}

__global__ void set_lens_kernel(int32_t* len, int n) {
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) len[i] = 0;
}

}  // namespace

extern "C" {

size_t topk_attn_coded_kv_bytes(const topk_attn_coded_config* cfg) {
    int why;
    return config_ok(cfg, &why) ? storage_of(cfg).total : 0;
}

size_t topk_attn_coded_workspace_bytes(const topk_attn_coded_config* cfg) {
    int why;
    return config_ok(cfg, &why) ? workspace_of(cfg).total : 0;
}

int topk_attn_coded_create(const topk_attn_coded_config* cfg, topk_attn_coded_t** out) {
    if (!out) return TOPK_ATTN_EINVAL;
    *out = nullptr;
    int why;
    if (!config_ok(cfg, &why)) return why;
    if (!cfg->kv_storage || !cfg->workspace) return TOPK_ATTN_EINVAL;
    if (((uintptr_t)cfg->kv_storage | (uintptr_t)cfg->workspace) & (kAlign - 1)) return TOPK_ATTN_EINVAL;
    const Workspace w = workspace_of(cfg);
    if (cfg->kv_bytes < storage_of(cfg).total || cfg->workspace_bytes < w.total) return TOPK_ATTN_ENOMEM;
    topk_attn_coded* h = nullptr;
    try {
        h = new topk_attn_coded;
        h->cfg = *cfg;
        h->len.assign((size_t)cfg->n_layers * cfg->n_seqs, 0);
    } catch (const std::bad_alloc&) {
        delete h;
        return TOPK_ATTN_ENOMEM;
    }
    const DeviceOf device(cfg->device);
    hipDeviceProp_t prop;
    // lengths and counters start at zero
    if (!device.ok() || hipGetDeviceProperties(&prop, cfg->device) != hipSuccess ||
        hipMemset(cfg->workspace, 0, w.parts) != hipSuccess || hipDeviceSynchronize() != hipSuccess) {
        delete h;
        return TOPK_ATTN_EDEVICE;
    }
    h->n_cu = prop.multiProcessorCount > 0 ? prop.multiProcessorCount : 256;
    *out = h;
    return TOPK_ATTN_OK;
}

int topk_attn_coded_destroy(topk_attn_coded_t* h) {
    if (!h) return TOPK_ATTN_EINVAL;
    delete h;
    return TOPK_ATTN_OK;
}

int64_t topk_attn_coded_length(const topk_attn_coded_t* h, int layer, int seq) {
    if (!h || layer < 0 || layer >= h->cfg.n_layers || seq < 0 || seq >= h->cfg.n_seqs) return -1;
    return h->len[(size_t)layer * h->cfg.n_seqs + seq];
}

int topk_attn_coded_reset(topk_attn_coded_t* h, int layer, int seq, void* hip_stream) {
    if (!range_ok(h, layer, seq)) return TOPK_ATTN_EINVAL;
    const DeviceOf device(h->cfg.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    const int B = seq < 0 ? h->cfg.n_seqs : 1, b0 = seq < 0 ? 0 : seq;
    hipLaunchKernelGGL(set_lens_kernel, dim3((unsigned)((B + 255) / 256)), dim3(256), 0, (hipStream_t)hip_stream, arrays_of(h, layer, b0).len, B);
    if (hipGetLastError() != hipSuccess) return TOPK_ATTN_EDEVICE;
    std::fill_n(h->len.begin() + (size_t)layer * h->cfg.n_seqs + b0, B, 0);
    return TOPK_ATTN_OK;
}

int topk_attn_coded_append(topk_attn_coded_t* h, int layer, int seq, const void* k_new, const void* v_new, int64_t n_new,
                           int64_t seq_stride, int64_t token_stride, int64_t head_stride, void* hip_stream) {
    if (!range_ok(h, layer, seq) || n_new < 0) return TOPK_ATTN_EINVAL;
    if (n_new == 0) return TOPK_ATTN_OK;
    const topk_attn_coded_config& c = h->cfg;
    const int e = elem_bytes(c.dtype);
    if (!k_new || !v_new || (((uintptr_t)k_new | (uintptr_t)v_new) & 15) || !strides_ok(seq_stride, token_stride, head_stride, e)) return TOPK_ATTN_EINVAL;
    const int B = seq < 0 ? c.n_seqs : 1, b0 = seq < 0 ? 0 : seq;
    int64_t* const len = &h->len[(size_t)layer * c.n_seqs + b0];
    for (int b = 0; b < B; ++b)
        if (n_new > c.max_tokens - len[b]) return TOPK_ATTN_ECAPACITY;
    // (a launch holds at most n_new / 64 + 1 full blocks a stream)
    if (std::min(B, kCodedSeqs) * (int64_t)c.n_kv_heads * 2 * (n_new / kCodedBlock + 1) > kMostWorkgroups) return TOPK_ATTN_EUNSUPPORTED;
    const DeviceOf device(c.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    for (int s0 = 0; s0 < B; s0 += kCodedSeqs) {
        CodedAppendCall a{};
        a.a = arrays_of(h, layer, b0 + s0);
        a.B = std::min(kCodedSeqs, B - s0);
        a.src[0] = static_cast<const char*>(k_new) + s0 * seq_stride * e;
        a.src[1] = static_cast<const char*>(v_new) + s0 * seq_stride * e;
        a.seq = seq_stride * e; a.token = token_stride * e; a.head = head_stride * e;
        a.n = n_new; a.wgs = 1;
        for (int b = 0; b < a.B; ++b) {
            a.base[b] = (int32_t)len[s0 + b];
            a.wgs = std::max(a.wgs, (len[s0 + b] + n_new) / kCodedBlock - len[s0 + b] / kCodedBlock);
        }
        a.Hkv = c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype; a.format = c.format;
        if (launch_coded_append(a, (hipStream_t)hip_stream) != hipSuccess) return TOPK_ATTN_EDEVICE;
        for (int b = 0; b < a.B; ++b) len[s0 + b] += n_new;
    }
    return TOPK_ATTN_OK;
}

int topk_attn_coded_read(topk_attn_coded_t* h, int layer, int seq, int64_t first, int64_t n, void* k_out, void* v_out,
                         int64_t seq_stride, int64_t token_stride, int64_t head_stride, void* hip_stream) {
    if (!range_ok(h, layer, seq) || first < 0 || n < 0) return TOPK_ATTN_EINVAL;
    const topk_attn_coded_config& c = h->cfg;
    const int e = elem_bytes(c.dtype), B = seq < 0 ? c.n_seqs : 1, b0 = seq < 0 ? 0 : seq;
    for (int b = 0; b < B; ++b) {
        const int64_t N = h->len[(size_t)layer * c.n_seqs + b0 + b];
        if (first > N || n > N - first) return TOPK_ATTN_EINVAL;
    }
    if (n == 0) return TOPK_ATTN_OK;
    if (!k_out || !v_out || (((uintptr_t)k_out | (uintptr_t)v_out) & 15) || !strides_ok(seq_stride, token_stride, head_stride, e)) return TOPK_ATTN_EINVAL;
    if (B * (int64_t)c.n_kv_heads * 2 * (n / kCodedBlock + 2) > kMostWorkgroups) return TOPK_ATTN_EUNSUPPORTED;
    const DeviceOf device(c.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    CodedReadCall a{};
    a.a = arrays_of(h, layer, b0);
    a.dst[0] = static_cast<char*>(k_out); a.dst[1] = static_cast<char*>(v_out);
    a.seq = seq_stride * e; a.token = token_stride * e; a.head = head_stride * e;
    a.first = first; a.n = n; a.B = B; a.Hkv = c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype; a.format = c.format;
    return launch_coded_read(a, (hipStream_t)hip_stream) == hipSuccess ? TOPK_ATTN_OK : TOPK_ATTN_EDEVICE;
}

int topk_attn_coded_decode(topk_attn_coded_t* h, int layer, const void* q, int64_t sinks, int64_t window, float* out, float* lse, void* hip_stream) {
    if (!h || !q || !out || layer < 0 || layer >= h->cfg.n_layers || ((uintptr_t)q & 15) || sinks < 0 || window < 1) return TOPK_ATTN_EINVAL;
    for (int b = 0; b < h->cfg.n_seqs; ++b)
        if (h->len[(size_t)layer * h->cfg.n_seqs + b] < 1) return TOPK_ATTN_EINVAL;
    CodedDecodeCall a{};
    a.q = q; a.out = out; a.lse = lse; a.sinks = sinks; a.window = a.reach = window;
    a.B = h->cfg.n_seqs; a.rows = h->cfg.n_q_heads / h->cfg.n_kv_heads;
    return decode_rows(h, layer, 0, a, hip_stream);
}

int topk_attn_coded_prompt(topk_attn_coded_t* h, int layer, int seq, const void* q, int64_t n_queries, int64_t sinks, int64_t window, void* out,
                           float* lse, void* hip_stream) {
    if (!range_ok(h, layer, seq) || n_queries < 0 || sinks < 0 || window < 1) return TOPK_ATTN_EINVAL;
    const topk_attn_coded_config& c = h->cfg;
    const int S = seq < 0 ? c.n_seqs : 1, b0 = seq < 0 ? 0 : seq;
    const int64_t* const len = &h->len[(size_t)layer * c.n_seqs + b0];
    for (int b = 0; b < S; ++b)
        if (n_queries > len[b]) return TOPK_ATTN_EINVAL;
    if (n_queries == 0) return TOPK_ATTN_OK;
    if (!q || !out || (((uintptr_t)q | (uintptr_t)out) & 15)) return TOPK_ATTN_EINVAL;
    const Workspace ws = workspace_of(&c);
    const int64_t rows = n_queries * (c.n_q_heads / c.n_kv_heads);
    if (rows <= few_rows(c.dtype, c.head_dim) && split_room(c, ws, S, rows) >= 2) {      // (blocks and open rows)
        CodedDecodeCall a{};
        a.q = q; a.out_rows = out; a.lse = lse; a.sinks = sinks; a.window = window;
        a.reach = std::min(window, (int64_t)1 << 40) + n_queries - 1;
        a.B = S; a.M = (int)n_queries; a.rows = (int)rows;
        return decode_rows(h, layer, b0, a, hip_stream);
    }
    PromptCall a{};
    a.c = arrays_of(h, layer, b0);
    a.q = q; a.out = out; a.lse = lse; a.len = a.c.len;
    a.M = n_queries; a.sinks = sinks; a.window = window;
    a.S = S; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype; a.format = c.format;
    if (a.M * a.G > kMostPromptRows) return TOPK_ATTN_EUNSUPPORTED;
    plan_prompt(&a, len, ws.parts_bytes, h->n_cu);
    place_prompt_parts(&a, static_cast<char*>(c.workspace) + ws.parts);
    if ((int64_t)S * a.Hkv * a.row_blocks * a.n_split > kMostWorkgroups) return TOPK_ATTN_EUNSUPPORTED;
    const DeviceOf device(c.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    return launch_prompt_coded(a, (hipStream_t)hip_stream) == hipSuccess ? TOPK_ATTN_OK : TOPK_ATTN_EDEVICE;
}

}  // extern "C"
