// The handle behind topk_attn_t, and where its arrays lie: shared by the translation units with C entry points.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <vector>

#include "../../include/topk_attn.h"
#include "internal.h"

namespace tka {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline int elem_bytes(int dtype) { return dtype == TOPK_ATTN_F32 ? 4 : 2; }

struct WsLayout {
    size_t len, arrive, thr, bins, samp, seg_cnt, seg_max, seg_cnt2, flags, hmax, fallback, tailrec, page_mask, page_cnt, page_list, hist, cand, bnd, scores, sel_idx, sel_val, part_acc, part_l, part_m, block_score, block_list, total;
    int cand_cap, bnd_cap, n_chunk_cap, hist_cap, page_words, batch_layers;
};

inline size_t kv_half_bytes(const topk_attn_config* c) {
    return align_up((size_t)c->n_layers * c->n_seqs * c->n_kv_heads * (size_t)c->max_tokens * c->head_dim *
                    elem_bytes(c->dtype));
}

// int8 index behind K and V: codes, then scales
inline size_t index_codes_bytes(const topk_attn_config* c) {
    if (c->index_kind != TOPK_ATTN_INDEX_INT8) return 0;
    return align_up((size_t)c->n_layers * c->n_seqs * c->n_kv_heads * (size_t)c->max_tokens * c->head_dim);
}
inline size_t index_scales_bytes(const topk_attn_config* c) {
    if (c->index_kind != TOPK_ATTN_INDEX_INT8) return 0;
    return align_up((size_t)c->n_layers * c->n_seqs * c->n_kv_heads * (size_t)c->max_tokens * sizeof(float));
}
// page index behind K and V: centres, then (radius, centre norm) pairs
inline int64_t page_cap_of(const topk_attn_config* c) { return (c->max_tokens + 63) / 64; }
inline size_t page_centres_bytes(const topk_attn_config* c) {
    if (c->index_kind != TOPK_ATTN_INDEX_PAGES) return 0;
    return align_up((size_t)c->n_layers * c->n_seqs * c->n_kv_heads * (size_t)page_cap_of(c) * c->head_dim * elem_bytes(c->dtype));
}
inline size_t page_balls_bytes(const topk_attn_config* c) {
    if (c->index_kind != TOPK_ATTN_INDEX_PAGES) return 0;
    return align_up((size_t)c->n_layers * c->n_seqs * c->n_kv_heads * (size_t)page_cap_of(c) * 2 * sizeof(float));
}
// block index behind K and V: per page the smallest, then the largest key, channel by channel
inline size_t page_boxes_bytes(const topk_attn_config* c) {
    if (c->index_kind != TOPK_ATTN_INDEX_BOXES) return 0;
    return align_up((size_t)c->n_layers * c->n_seqs * c->n_kv_heads * (size_t)page_cap_of(c) * 2 * c->head_dim * elem_bytes(c->dtype));
}
inline size_t kv_total_bytes(const topk_attn_config* c) {
    return 2 * kv_half_bytes(c) + index_codes_bytes(c) + index_scales_bytes(c) + page_centres_bytes(c) + page_balls_bytes(c) +
           page_boxes_bytes(c);
}

}  // namespace tka

struct topk_attn {
    topk_attn_config cfg;
    tka::WsLayout ws;
    tka::WsLayout ws_one;            // the layout without room for further layers (the built-in scratch)
    size_t kv_half;
    std::vector<int64_t> len;   // host mirror of the device lengths, [L][B]
    int path;
    bool last_fast;
    bool last_static;           // the last decode used the built-in scratch
    int force_redo;             // measurement aid, see topk_attn_debug_force_redo: 0, 1, or 2 (chip-wide selection)
    float page_beta;            // scale of the page radius in the page bound (1 = exact)
    bool last_paged;            // the last decode went through the page index
    bool last_tail;             // the last decode used the chip-wide selection (its per-head records are in the workspace)
    int last_queries;           // queries per sequence of the last decode
    int last_n_seg, last_seg_cap;   // the split of the last filtered decode's candidate lists (0: not filtered)
    int last_layer;
    int last_slot;              // layers of the last call before its last one in the per-call buffers
    char* scratch_dev;          // this device's copy of the built-in scratch
    int n_cu;                   // compute units of the device
    // optional event pairs around the key scan of each decode (measurement only)
    bool timing;
    std::vector<hipEvent_t> ev;  // 2 * kTimingSlots once enabled
    int ev_used;
};
