// Where the arrays of a handle's layer lie: shared by the translation units with C entry points beside the top-k decode.
#pragma once
#include "handle.h"
#include "internal.h"

namespace tka {

struct Layer {
    int64_t row, head;              // bytes of a row, and of a key stream's rows
    char *K, *V;
    int32_t* len;
    char* index;                    // behind K and V, all layers
    int64_t stream0;                // key streams of the layers before
};
inline Layer layer_of(const topk_attn* h, int layer) {
    const topk_attn_config& c = h->cfg;
    Layer l;
    l.row = (int64_t)c.head_dim * elem_bytes(c.dtype);
    l.head = c.max_tokens * l.row;
    l.stream0 = (int64_t)layer * c.n_seqs * c.n_kv_heads;
    l.K = static_cast<char*>(c.kv_storage) + l.stream0 * l.head;
    l.V = l.K + h->kv_half;
    l.len = reinterpret_cast<int32_t*>(static_cast<char*>(c.workspace) + h->ws.len) + (size_t)layer * c.n_seqs;
    l.index = static_cast<char*>(c.kv_storage) + 2 * h->kv_half;
    return l;
}
template <class T>
T* scratch_at(const topk_attn* h, size_t offset) { return reinterpret_cast<T*>(static_cast<char*>(h->cfg.workspace) + offset); }

}  // namespace tka
