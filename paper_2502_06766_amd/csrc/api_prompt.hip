// C entry of the attention of a prompt's tokens over a cache in its own type.
#include <hip/hip_runtime.h>

#include "../../include/topk_attn.h"
#include "handle.h"
#include "layer.h"
#include "ops.h"
#include "prompt.h"
#include "split_plan.h"

using namespace tka;

namespace {

// Bytes for partial sums: the candidate lists' place.
size_t parts_bytes(const topk_attn* h) { return (size_t)h->cfg.n_seqs * h->cfg.n_q_heads * h->ws.cand_cap * sizeof(uint64_t); }
// Splits of `rows` rows of each key stream that there is room for: at least one of kFewRowsF32 (a candidate list has 2^14 entries or more).
int64_t split_room(const topk_attn* h, int seqs, int64_t rows) {
    return (int64_t)(parts_bytes(h) / ((size_t)seqs * h->cfg.n_kv_heads * (size_t)rows * (h->cfg.head_dim + 2) * sizeof(float)));
}

// Few rows of each of S sequences from b0 on: the walk of single tokens (dense.hip).
int decode_rows(topk_attn* h, int layer, int b0, int S, const void* q, int64_t M, int64_t sinks, int64_t window, void* out, float* lse, void* hip_stream) {
    const topk_attn_config& c = h->cfg;
    const int64_t* const len = &h->len[(size_t)layer * c.n_seqs + b0];
    const Layer l = layer_of(h, layer);
    AttendCall a{};
    a.K = l.K + (int64_t)b0 * c.n_kv_heads * l.head; a.V = l.V + (int64_t)b0 * c.n_kv_heads * l.head;
    a.q = q; a.out_rows = out; a.lse = lse; a.len = l.len + b0;
    a.B = S; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype;
    a.M = (int)M; a.rows = a.M * a.G; a.row_blocks = (a.rows + 15) / 16;
    a.Ncap = c.max_tokens; a.sinks = sinks; a.window = window;
    a.reach = std::min(window, (int64_t)1 << 40) + M - 1;
    int64_t pages = 1, sample[16];               // (of a larger batch some sequences stand for all)
    const int n_sample = std::min(S, 16);
    for (int b = 0; b < S; ++b) pages = std::max(pages, WindowWalk(len[b], sinks, a.reach).pages());
    for (int i = 0; i < n_sample; ++i) sample[i] = WindowWalk(len[(int64_t)i * S / n_sample], sinks, a.reach).pages();
    a.chunk = (int)pages_per_split(sample, n_sample, (double)S / n_sample * a.Hkv * a.row_blocks, pages, std::min<int64_t>(kMaxSplits, split_room(h, S, a.rows)),
                                   h->n_cu, (double)l.row);
    a.n_split = (int)((pages + a.chunk - 1) / a.chunk);
    a.walk = pages * 64;
    a.join_later = (int64_t)a.n_split * std::min(a.rows, 16) * a.D * 4 > kJoinBytes;
    a.join_heads = 1;
    a.part_acc = scratch_at<float>(h, h->ws.cand);
    a.part_lm = a.part_acc + (size_t)S * a.Hkv * a.rows * a.n_split * a.D;
    a.arrive = scratch_at<uint32_t>(h, h->ws.arrive);
    a.scale_log2e = 1.4426950408889634f / sqrtf((float)a.D);
    if (attend_walk_wgs(a) > kMostWorkgroups || attend_join_wgs(a) > kMostWorkgroups) return TOPK_ATTN_EUNSUPPORTED;
    const DeviceOf device(c.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    return launch_attend(a, (hipStream_t)hip_stream) == hipSuccess ? TOPK_ATTN_OK : TOPK_ATTN_EDEVICE;
}

}  // namespace

extern "C" {

int topk_attn_prompt(topk_attn_t* h, int layer, int seq, const void* q, int64_t n_queries, int64_t sinks, int64_t window, void* out, float* lse,
                     void* hip_stream) {
    if (!h || layer < 0 || layer >= h->cfg.n_layers || seq < -1 || seq >= h->cfg.n_seqs || n_queries < 0 || sinks < 0 || window < 1) return TOPK_ATTN_EINVAL;
    const topk_attn_config& c = h->cfg;
    const int S = seq < 0 ? c.n_seqs : 1, b0 = seq < 0 ? 0 : seq;
    const int64_t* const len = &h->len[(size_t)layer * c.n_seqs + b0];
    for (int b = 0; b < S; ++b)
        if (n_queries > len[b]) return TOPK_ATTN_EINVAL;
    if (n_queries == 0) return TOPK_ATTN_OK;
    if (!q || !out || (((uintptr_t)q | (uintptr_t)out) & 15)) return TOPK_ATTN_EINVAL;
    const Layer l = layer_of(h, layer);
    const int64_t rows = n_queries * (c.n_q_heads / c.n_kv_heads);
    if (c.dtype == TOPK_ATTN_F32 && rows <= kFewRowsF32) return decode_rows(h, layer, b0, S, q, n_queries, sinks, window, out, lse, hip_stream);
    PromptCall a{};
    a.K = l.K + (int64_t)b0 * c.n_kv_heads * l.head; a.V = l.V + (int64_t)b0 * c.n_kv_heads * l.head;
    a.q = q; a.out = out; a.lse = lse; a.len = l.len + b0;
    a.Ncap = c.max_tokens; a.M = n_queries; a.sinks = sinks; a.window = window;
    a.S = S; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype; a.format = -1;
    if (a.M * a.G > kMostPromptRows) return TOPK_ATTN_EUNSUPPORTED;
    plan_prompt(&a, len, parts_bytes(h), h->n_cu);
    place_prompt_parts(&a, scratch_at<float>(h, h->ws.cand));
    if ((int64_t)S * a.Hkv * a.row_blocks * a.n_split > kMostWorkgroups) return TOPK_ATTN_EUNSUPPORTED;
    const DeviceOf device(c.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    return launch_prompt(a, (hipStream_t)hip_stream) == hipSuccess ? TOPK_ATTN_OK : TOPK_ATTN_EDEVICE;
}

}  // extern "C"
