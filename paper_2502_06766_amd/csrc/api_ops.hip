// C entries of the operators beside the top-k decode: appends that normalise and rotate, dense and block-sparse decode, accumulated
// attention weight and eviction by it.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "../../include/topk_attn.h"
#include "handle.h"
#include "internal.h"
#include "layer.h"
#include "ops.h"
#include "page_boxes.h"
#include "split_plan.h"

using namespace tka;

namespace {

int decode_all(topk_attn_t* h, int layer, const void* q, int n_blocks, float* out, int32_t* blocks, float* lse, float* mass,
               void* hip_stream, int64_t sinks = 0, int64_t window = 0) {
    const topk_attn_config& c = h->cfg;
    if ((int64_t)c.n_seqs * c.n_kv_heads > kMostStreams) return TOPK_ATTN_EUNSUPPORTED;
    const Layer l = layer_of(h, layer);
    int64_t longest = 0;
    for (int b = 0; b < c.n_seqs; ++b) {
        const int64_t n = h->len[(size_t)layer * c.n_seqs + b];
        if (n < 1) return TOPK_ATTN_EINVAL;
        longest = std::max(longest, n);
    }
    const DeviceOf device(h->cfg.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    hipStream_t st = (hipStream_t)hip_stream;
    int64_t pages = (longest + 63) / 64;
    AttendCall a{};
    a.K = l.K; a.V = l.V; a.q = q; a.len = l.len;
    a.B = c.n_seqs; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype;
    a.Ncap = c.max_tokens;
    const bool some = n_blocks && pages > n_blocks;              // (a sequence of at most n_blocks pages is attended whole)
    if (some) pages = n_blocks;
    // (sequences that are seen whole: as the dense decode)
    if (window && WindowWalk(longest, sinks, window).first > 0) {
        a.sinks = sinks; a.window = a.reach = window;
        pages = WindowWalk(longest, sinks, window).pages();
        for (int b = 0; b < c.n_seqs; ++b)               // (a shorter sequence may have more pages: its sinks and its window meet)
            pages = std::max(pages, WindowWalk(h->len[(size_t)layer * c.n_seqs + b], sinks, window).pages());
    }
    a.walk = pages * 64;
    a.score_stride = c.max_tokens;               // (of a list: whole pages, one less than the cache has at least)
    a.scores = scratch_at<float>(h, h->ws.scores);
    a.rows = a.G;
    a.row_blocks = (a.G + 15) / 16;
    // partial sums in the candidate lists' place
    const size_t room = (size_t)h->ws.cand_cap * sizeof(uint64_t) / ((size_t)c.head_dim * sizeof(float) + 2 * sizeof(float));
    const int64_t max_splits = std::min<int64_t>(kMaxSplits, (int64_t)room);
    int64_t sample[16];                          // (of a larger batch some sequences stand for all)
    const int n_sample = std::min(c.n_seqs, 16);
    for (int i = 0; i < n_sample; ++i) {
        const int64_t n = h->len[(size_t)layer * c.n_seqs + (size_t)((int64_t)i * c.n_seqs / n_sample)];
        sample[i] = std::min(a.window ? WindowWalk(n, sinks, window).pages() : (n + 63) / 64, pages);
    }
    a.chunk = (int)pages_per_split(sample, n_sample, (double)c.n_seqs / n_sample * a.Hkv * a.row_blocks, pages, max_splits, h->n_cu,
                                   (double)l.row);
    a.n_split = (int)((pages + a.chunk - 1) / a.chunk);
    const bool many = (int64_t)a.n_split * std::min(a.G, 16) * a.D * 4 > kJoinBytes;
    a.join_later = mass || many;
    a.join_heads = many ? 1 : 16;
    a.part_acc = scratch_at<float>(h, h->ws.cand);
    a.part_lm = a.part_acc + (size_t)a.B * a.Hq * a.n_split * a.D;
    a.arrive = scratch_at<uint32_t>(h, h->ws.arrive);
    a.out = out; a.lse = lse; a.mass = mass;
    a.scale_log2e = 1.4426950408889634f / sqrtf((float)c.head_dim);
    if (attend_walk_wgs(a) > kMostWorkgroups || attend_join_wgs(a) + attend_mass_wgs(a) > kMostWorkgroups) return TOPK_ATTN_EUNSUPPORTED;
    if (n_blocks) {
        BlockCall p{};
        p.boxes = l.index + l.stream0 * page_cap_of(&c) * 2 * l.row;
        p.q = q; p.len = l.len;
        p.score = scratch_at<double>(h, h->ws.block_score);
        p.list = blocks ? blocks : scratch_at<int32_t>(h, h->ws.block_list);
        // (a longer list than the cache has pages: only the caller's own array has room for it)
        p.n_blocks = blocks ? n_blocks : (int)std::min<int64_t>(n_blocks, page_cap_of(&c));
        p.list_stride = p.n_blocks;
        p.Pcap = page_cap_of(&c); p.pages = (longest + 63) / 64;
        p.B = a.B; p.Hq = a.Hq; p.Hkv = a.Hkv; p.G = a.G; p.D = a.D; p.dtype = a.dtype;
        if (some) { a.list = p.list; a.list_stride = p.list_stride; a.n_list = n_blocks; }
        if (some && launch_block_scores(p, st) != hipSuccess) return TOPK_ATTN_EDEVICE;
        if ((blocks || some) && launch_block_select(p, st) != hipSuccess) return TOPK_ATTN_EDEVICE;
    }
    return launch_attend(a, st) == hipSuccess ? TOPK_ATTN_OK : TOPK_ATTN_EDEVICE;
}

}  // namespace

extern "C" {

int topk_attn_decode_dense(topk_attn_t* h, int layer, const void* q, float* out, float* lse, float* mass, void* hip_stream) {
    if (!h || !q || !out || layer < 0 || layer >= h->cfg.n_layers || ((uintptr_t)q & 15)) return TOPK_ATTN_EINVAL;
    return decode_all(h, layer, q, 0, out, nullptr, lse, mass, hip_stream);
}

int topk_attn_decode_sinks(topk_attn_t* h, int layer, const void* q, int64_t sinks, int64_t window, float* out, float* lse, void* hip_stream) {
    if (!h || !q || !out || layer < 0 || layer >= h->cfg.n_layers || ((uintptr_t)q & 15)) return TOPK_ATTN_EINVAL;
    if (sinks < 0 || window < 1) return TOPK_ATTN_EINVAL;
    return decode_all(h, layer, q, 0, out, nullptr, lse, nullptr, hip_stream, sinks, window);
}

int topk_attn_decode_blocks(topk_attn_t* h, int layer, const void* q, int n_blocks, float* out, int32_t* blocks, float* lse, float* mass,
                            void* hip_stream) {
    if (!h || !q || !out || layer < 0 || layer >= h->cfg.n_layers || ((uintptr_t)q & 15)) return TOPK_ATTN_EINVAL;
    if (h->cfg.index_kind != TOPK_ATTN_INDEX_BOXES || n_blocks < 1) return TOPK_ATTN_EINVAL;
    return decode_all(h, layer, q, n_blocks, out, blocks, lse, mass, hip_stream);
}

int topk_attn_add_mass(topk_attn_t* h, int layer, const int32_t* idx, const float* vals, const float* lse, int k, float* mass,
                       void* hip_stream) {
    if (!h || !idx || !vals || !lse || !mass || layer < 0 || layer >= h->cfg.n_layers || k < 1) return TOPK_ATTN_EINVAL;
    if (k > kMostSelected) return TOPK_ATTN_EINVAL;                  // (no decode has more; the kernel counts up to k + 4096 in 32 bits)
    const topk_attn_config& c = h->cfg;
    if ((int64_t)c.n_seqs * c.n_kv_heads > kMostStreams) return TOPK_ATTN_EUNSUPPORTED;
    const DeviceOf device(h->cfg.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    MassCall a{};
    a.idx = idx; a.vals = vals; a.lse = lse; a.mass = mass; a.Ncap = c.max_tokens;
    a.B = c.n_seqs; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads; a.k = k;
    a.scale_log2e = 1.4426950408889634f / sqrtf((float)c.head_dim);
    return launch_add_mass(a, (hipStream_t)hip_stream) == hipSuccess ? TOPK_ATTN_OK : TOPK_ATTN_EDEVICE;
}

int topk_attn_evict(topk_attn_t* h, int layer, float* mass, int64_t budget, int64_t recent, int32_t* kept, void* hip_stream) {
    if (!h || !mass || layer < 0 || layer >= h->cfg.n_layers) return TOPK_ATTN_EINVAL;
    const topk_attn_config& c = h->cfg;
    if (budget < 1 || budget > c.max_tokens || recent < 0 || recent > budget) return TOPK_ATTN_EINVAL;
    int64_t longest = 0;
    for (int b = 0; b < c.n_seqs; ++b) longest = std::max(longest, h->len[(size_t)layer * c.n_seqs + b]);
    if (longest <= budget && !kept) return TOPK_ATTN_OK;
    if ((int64_t)c.n_seqs * c.n_kv_heads > kMostStreams) return TOPK_ATTN_EUNSUPPORTED;
    const Layer l = layer_of(h, layer);
    EvictCall a{};
    a.mass = mass; a.len = l.len; a.Ncap = c.max_tokens; a.budget = budget; a.recent = recent; a.B = c.n_seqs; a.Hkv = c.n_kv_heads;
    a.kept = kept ? kept : scratch_at<int32_t>(h, h->ws.scores);
    auto add = [&](void* base, int row, bool cleared) {
        EvictArray& x = a.array[a.n_arrays++];
        x.base = static_cast<char*>(base); x.row = row; x.cleared = cleared;
        x.unit_rows = row >= 16 ? kEvictUnitBytes / row : 256 * kEvictPieces;
        x.units = (int)(((cleared ? longest : budget) + x.unit_rows - 1) / x.unit_rows);
        a.units += x.units;
    };
    add(l.K, (int)l.row, false);
    add(l.V, (int)l.row, false);
    if (c.index_kind == TOPK_ATTN_INDEX_INT8) {
        add(l.index + l.stream0 * c.max_tokens * c.head_dim, c.head_dim, false);
        add(l.index + index_codes_bytes(&c) + l.stream0 * c.max_tokens * sizeof(float), sizeof(float), false);
    }
    add(mass, sizeof(float), true);
    a.longest = longest - recent;
    a.chunk = std::max<int64_t>(kEvictHeldTokens, (a.longest + kEvictChunks - 1) / kEvictChunks);
    // scratch in the candidate lists' place
    const size_t streams = (size_t)c.n_seqs * c.n_kv_heads;
    size_t words = 0;
    const auto take = [&](size_t n) { uint32_t* p = scratch_at<uint32_t>(h, h->ws.cand) + words; words += (n + 3) / 4 * 4; return p; };
    if (a.longest > kEvictHeldTokens) {
        a.hist = take(streams * 2 * kEvictChunks * kEvictBins);
        a.pick = take(streams * kEvictPick);
    }
    a.state = take(streams * (a.units + 1));
    a.old_len = reinterpret_cast<int32_t*>(take(c.n_seqs));
    if (words * 4 > (size_t)c.n_seqs * c.n_q_heads * h->ws.cand_cap * sizeof(uint64_t)) return TOPK_ATTN_ENOMEM;
    const DeviceOf device(h->cfg.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = launch_evict(a, st);
    if (e != hipSuccess) return e == hipErrorInvalidValue ? TOPK_ATTN_ENOMEM : TOPK_ATTN_EDEVICE;
    if (longest <= budget) return TOPK_ATTN_OK;
    for (int b = 0; b < c.n_seqs; ++b) {
        int64_t& n = h->len[(size_t)layer * c.n_seqs + b];
        n = std::min(n, budget);
    }
    const int64_t pcap = page_cap_of(&c);
    if (c.index_kind == TOPK_ATTN_INDEX_PAGES &&
        launch_balls_again(c.dtype, c.head_dim, l.K, c.max_tokens, pcap, c.n_kv_heads, c.n_seqs, l.len, budget,
                           l.index + l.stream0 * pcap * l.row,
                           reinterpret_cast<float*>(l.index + page_centres_bytes(&c)) + l.stream0 * pcap * 2, st) != hipSuccess)
        return TOPK_ATTN_EDEVICE;
    if (c.index_kind == TOPK_ATTN_INDEX_BOXES &&
        launch_page_boxes(c.dtype, c.head_dim, l.K, c.max_tokens, pcap, c.n_kv_heads, c.n_seqs, l.len, 0, -budget,
                          l.index + l.stream0 * pcap * 2 * l.row, st) != hipSuccess)
        return TOPK_ATTN_EDEVICE;
    return TOPK_ATTN_OK;
}

__global__ static void advance_len_kernel(int32_t* len, int B, int32_t n_new) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < B) len[b] += n_new;
}

int topk_attn_append_rotary(topk_attn_t* h, int layer, int seq, const topk_attn_rotary* r, void* hip_stream) {
    if (!h || !r || r->struct_size != sizeof(topk_attn_rotary)) return TOPK_ATTN_EINVAL;
    const topk_attn_config& c = h->cfg;
    if (layer < 0 || layer >= c.n_layers || seq < -1 || seq >= c.n_seqs || r->n_new < 0) return TOPK_ATTN_EINVAL;
    if (r->rotary_dim < 0 || r->rotary_dim > c.head_dim || (r->rotary_dim & 1) || !(r->norm_eps >= 0.f) || isinf(r->norm_eps)) return TOPK_ATTN_EINVAL;
    if (r->n_new == 0) return TOPK_ATTN_OK;
    if (!r->k || !r->v || !r->q != !r->q_out || (r->rotary_dim && !r->inv_freq)) return TOPK_ATTN_EINVAL;
    const int e = elem_bytes(c.dtype);
    const int64_t strides[6] = {r->q_seq_stride, r->q_token_stride, r->k_seq_stride, r->k_token_stride, r->v_seq_stride, r->v_token_stride};
    for (int i = r->q ? 0 : 2; i < 6; ++i)
        if (strides[i] < 0 || strides[i] > INT64_MAX / 8 || ((strides[i] * e) & 15)) return TOPK_ATTN_EINVAL;
    if (((uintptr_t)r->q | (uintptr_t)r->k | (uintptr_t)r->v | (uintptr_t)r->q_out | (uintptr_t)r->q_norm | (uintptr_t)r->k_norm) & 15)
        return TOPK_ATTN_EINVAL;
    const int B = seq < 0 ? c.n_seqs : 1, b0 = seq < 0 ? 0 : seq;
    const size_t slot = (size_t)layer * c.n_seqs + b0;
    for (int b = 0; b < B; ++b)
        if (r->n_new > c.max_tokens - h->len[slot + b]) return TOPK_ATTN_ECAPACITY;
    if ((int64_t)B * r->n_new > kMostWorkgroups) return TOPK_ATTN_EUNSUPPORTED;
    const DeviceOf device(h->cfg.device);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    hipStream_t st = (hipStream_t)hip_stream;
    const Layer l = layer_of(h, layer);
    const int64_t stream0 = l.stream0 + (int64_t)b0 * c.n_kv_heads, pcap = page_cap_of(&c);
    RotaryCall a{};
    a.q = static_cast<const char*>(r->q); a.k = static_cast<const char*>(r->k); a.v = static_cast<const char*>(r->v);
    a.q_seq = r->q_seq_stride * e; a.q_token = r->q_token_stride * e;
    a.k_seq = r->k_seq_stride * e; a.k_token = r->k_token_stride * e;
    a.v_seq = r->v_seq_stride * e; a.v_token = r->v_token_stride * e;
    a.q_out = static_cast<char*>(r->q_out);
    a.K = l.K + (int64_t)b0 * c.n_kv_heads * l.head;
    a.V = l.V + (int64_t)b0 * c.n_kv_heads * l.head;
    a.q_norm = r->q_norm; a.k_norm = r->k_norm; a.inv_freq = r->inv_freq; a.positions = r->positions;
    a.len = l.len + b0;
    if (c.index_kind == TOPK_ATTN_INDEX_INT8) {
        a.codes = reinterpret_cast<int8_t*>(l.index) + stream0 * c.max_tokens * c.head_dim;
        a.scales = reinterpret_cast<float*>(l.index + index_codes_bytes(&c)) + stream0 * c.max_tokens;
    }
    a.Ncap = c.max_tokens; a.n = r->n_new; a.B = B; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype;
    a.rotary = r->rotary_dim; a.interleaved = r->interleaved != 0; a.eps = r->norm_eps;
    // Sequences of one length: passed by value, so that no workgroup reads what another one advances.  (A launch that advances the lengths
    // costs 5 us of a prompt's 56, a counter of the tokens done 50.)
    a.base = h->len[slot];
    for (int b = 1; b < B; ++b)
        if (h->len[slot + b] != a.base) a.base = -1;
    // the kernel advances the lengths unless an index kernel after it needs the old ones
    a.advance = c.index_kind != TOPK_ATTN_INDEX_PAGES && c.index_kind != TOPK_ATTN_INDEX_BOXES && (a.base >= 0 || r->n_new == 1);
    if (launch_rotary(a, st) != hipSuccess) return TOPK_ATTN_EDEVICE;
    if (c.index_kind == TOPK_ATTN_INDEX_PAGES &&
        launch_page_balls(c.dtype, c.head_dim, a.K, c.max_tokens, pcap, c.n_kv_heads, B, a.len, 0, r->n_new, l.index + stream0 * pcap * l.row,
                          reinterpret_cast<float*>(l.index + page_centres_bytes(&c)) + stream0 * pcap * 2, st) != hipSuccess)
        return TOPK_ATTN_EDEVICE;
    if (c.index_kind == TOPK_ATTN_INDEX_BOXES &&
        launch_page_boxes(c.dtype, c.head_dim, a.K, c.max_tokens, pcap, c.n_kv_heads, B, a.len, 0, r->n_new,
                          l.index + stream0 * pcap * 2 * l.row, st) != hipSuccess)
        return TOPK_ATTN_EDEVICE;
    if (!a.advance) hipLaunchKernelGGL(advance_len_kernel, dim3((unsigned)((B + 255) / 256)), dim3(256), 0, st, a.len, B, (int32_t)r->n_new);
    if (hipGetLastError() != hipSuccess) return TOPK_ATTN_EDEVICE;
    for (int b = 0; b < B; ++b) h->len[slot + b] += r->n_new;
    return TOPK_ATTN_OK;
}

}  // extern "C"
