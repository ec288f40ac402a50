// C entry of the attention of a prompt's tokens over a cache in its own type.
#include <hip/hip_runtime.h>

#include "../../include/topk_attn.h"
#include "handle.h"
#include "layer.h"
#include "prompt.h"
#include "split_plan.h"

using namespace tka;

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
    PromptCall a{};
    a.K = l.K + (int64_t)b0 * c.n_kv_heads * l.head; a.V = l.V + (int64_t)b0 * c.n_kv_heads * l.head;
    a.q = q; a.out = out; a.lse = lse; a.len = l.len + b0;
    a.Ncap = c.max_tokens; a.M = n_queries; a.sinks = sinks; a.window = window;
    a.S = S; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype; a.format = -1;
    if (a.M * a.G > kMostPromptRows) return TOPK_ATTN_EUNSUPPORTED;
    // partial sums in the candidate lists' place
    plan_prompt(&a, len, (size_t)c.n_seqs * c.n_q_heads * h->ws.cand_cap * sizeof(uint64_t), h->n_cu);
    place_prompt_parts(&a, scratch_at<float>(h, h->ws.cand));
    if ((int64_t)S * a.Hkv * a.row_blocks * a.n_split > kMostWorkgroups) return TOPK_ATTN_EUNSUPPORTED;
    const DeviceOf device(c.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    return launch_prompt(a, (hipStream_t)hip_stream) == hipSuccess ? TOPK_ATTN_OK : TOPK_ATTN_EDEVICE;
}

}  // extern "C"
