// C entries of the operators beside the top-k decode: appends that normalise and rotate, dense and block-sparse decode, accumulated
// attention weight and eviction by it.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "../../include/topk_attn.h"
#include "handle.h"
#include "internal.h"
#include "ops.h"
#include "page_boxes.h"

using namespace tka;

namespace {

// The handle's device, current while the call enqueues.
class DeviceOf {
  public:
    explicit DeviceOf(const topk_attn* h) {
        ok_ = hipGetDevice(&before_) == hipSuccess && (before_ == h->cfg.device || hipSetDevice(h->cfg.device) == hipSuccess);
        changed_ = ok_ && before_ != h->cfg.device;
    }
    ~DeviceOf() { if (changed_) (void)hipSetDevice(before_); }
    bool ok() const { return ok_; }
  private:
    int before_ = 0;
    bool ok_ = false, changed_ = false;
};

// Where a layer's arrays lie.
struct Layer {
    int64_t row, head;              // bytes of a row, and of a key stream's rows
    char *K, *V;
    int32_t* len;
    char* index;                    // behind K and V, all layers
    int64_t stream0;                // key streams of the layers before
};
Layer layer_of(const topk_attn* h, int layer) {
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

// Pages that one workgroup of the walk takes: the split with the least estimated time.  The estimate, in microseconds, for key streams of
// pages[i] pages (each standing for `weight` streams), from measurements with 8 KV heads of d = 128 in 16 bits (32 KB a page):
//   - a page takes a workgroup 0.5 on an empty chip and 1.42 with one on every compute unit (5.9 TB/s), between them as the root of their number;
//   - more workgroups than compute units take whole rounds if all are alike, else their share of the work and a part of one at the end;
//   - a workgroup costs 1 in itself, 1.7 where others follow it, putting splits together 3.2, and 0.05 a split.
// One sequence of 500 / 1000 / 2000 / 16384 / 131072 tokens takes 8.5 / 9.0 / 9.8 / 18.0 / 93.6 us with 8 (one split), 2, 2, 8 and 64 pages a
// workgroup; with 2, 16 (one split), 16, 2 and 32 pages 8.8 / 12.7 / 16.0 / 21.8 / 97.3.  24 sequences of 400 to 8192 tokens, 64 heads: 105 / 92 / 92
// / 84 / 113 with 4 / 8 / 16 / 32 / 64 pages; 5 of 1600 to 32768: 80 / 75 / 73 / 76 / 107.
// Rows of 512 and 1024 bytes (d = 256, single-buffered) against the best of 2, 8, 16, 32 and 64 pages: 16 bits, 500 / 4000 / 16000 / 128000 tokens 10.5 /
// 14.7 / 28.4 / 181 and 10.5 / 14.7 / 28.4 / 178, 12 sequences of 400 to 8192 91 and 85; fp32, 500 / 4000 / 16000 / 64000 17.1 / 22.6 / 72.7 / 182
// and the same, 6 sequences 141 and 120.
int64_t pages_per_split(const int64_t* pages, int n, double weight, int64_t longest, int64_t max_splits, int n_cu, double row_bytes) {
    double best = 1e30, all = 0.0;
    int64_t chunk = longest;                                 // (max_splits >= 1)
    const double scale = row_bytes / 256.0;
    for (int i = 0; i < n; ++i) all += (double)pages[i];
    all *= weight / n_cu;
    const auto consider = [&](int64_t splits) {              // of the longest sequence
        const int64_t c = std::max<int64_t>(2, (longest + splits - 1) / splits);
        double wgs = 0.0;
        const float inv = 1.0f / (float)c;
        for (int i = 0; i < n; ++i) wgs += (double)(int64_t)((float)(pages[i] + c - 1) * inv);
        wgs *= weight / n_cu;                                // to a compute unit
        double cost = splits > 1 ? 3.2 + 0.05 * (double)splits : 0.0;
        if (wgs <= 1.0) cost += 1.0 + scale * (double)c * std::max(0.5, 1.42 * sqrt(wgs));
        else cost += 1.7 * wgs + scale * 1.42 * std::min(ceil(wgs) * (double)c, all + 0.25 * (double)c);
        if (cost < best) { best = cost; chunk = c; }
    };
    // powers of two, one number between each two of them, and what fills whole rounds if all sequences are as long
    for (int64_t k = 1; k <= max_splits && k <= longest; k *= 2) {
        consider(k);
        if (k >= 2 && k + k / 2 <= max_splits) consider(k + k / 2);
    }
    for (int r = 1; r <= 4; ++r) {
        const int64_t k = (int64_t)(r * n_cu / (n * weight));
        if (k >= 1 && k <= max_splits) consider(k);
    }
    return chunk;
}
// Beyond this many bytes of a head block's partial sums the one workgroup that would put them together takes longer than a launch that has a
// workgroup per head.  One sequence of 4k / 16k / 64k tokens, d = 128, joined in the walk's launch and after it, in us:
//   64 KB (32 splits of the 4 heads of 8 KV heads)  11.3 / 17.9 / 58.0 and 10.3 / 18.1 / 60.3
//   80 KB (5 heads)                                 12.7 / 19.2 / 66.7 and 10.4 / 18.5 / 67.2
//   128 KB (8 heads)                                13.5 / 19.8 / 66.3 and 10.9 / 18.9 / 62.8
//   256 to 728 KB (16 heads, one KV head)           16.3 / 19.4 / 30.1 and 11.7 / 14.8 / 18.5
// (32 KB, four sequences, 8 heads to each of 8 KV heads, 8 splits: 18.1 and 18.8 of 4k tokens, 52.6 and 53.7 of 16k.)
constexpr int64_t kJoinBytes = 64 << 10;

int decode_all(topk_attn_t* h, int layer, const void* q, int n_blocks, float* out, int32_t* blocks, float* lse, float* mass,
               void* hip_stream) {
    const topk_attn_config& c = h->cfg;
    if ((int64_t)c.n_seqs * c.n_kv_heads > kMostStreams) return TOPK_ATTN_EUNSUPPORTED;
    const Layer l = layer_of(h, layer);
    int64_t longest = 0;
    for (int b = 0; b < c.n_seqs; ++b) {
        const int64_t n = h->len[(size_t)layer * c.n_seqs + b];
        if (n < 1) return TOPK_ATTN_EINVAL;
        longest = std::max(longest, n);
    }
    const DeviceOf device(h);
    if (!device.ok()) return TOPK_ATTN_EDEVICE;
    hipStream_t st = (hipStream_t)hip_stream;
    int64_t pages = (longest + 63) / 64;
    AttendCall a{};
    a.K = l.K; a.V = l.V; a.q = q; a.len = l.len;
    a.B = c.n_seqs; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = c.n_q_heads / c.n_kv_heads; a.D = c.head_dim; a.dtype = c.dtype;
    a.Ncap = c.max_tokens;
    const bool some = n_blocks && pages > n_blocks;              // (a sequence of at most n_blocks pages is attended whole)
    if (some) pages = n_blocks;
    a.walk = pages * 64;
    a.score_stride = c.max_tokens;               // (of a list: whole pages, one less than the cache has at least)
    a.scores = scratch_at<float>(h, h->ws.scores);
    a.row_blocks = (a.G + 15) / 16;
    // partial sums in the candidate lists' place
    const size_t room = (size_t)h->ws.cand_cap * sizeof(uint64_t) / ((size_t)c.head_dim * sizeof(float) + 2 * sizeof(float));
    const int64_t max_splits = std::min<int64_t>(kMaxSplits, (int64_t)room);
    int64_t sample[16];                          // (of a larger batch some sequences stand for all)
    const int n_sample = std::min(c.n_seqs, 16);
    for (int i = 0; i < n_sample; ++i) {
        const int64_t n = h->len[(size_t)layer * c.n_seqs + (size_t)((int64_t)i * c.n_seqs / n_sample)];
        sample[i] = std::min((n + 63) / 64, pages);
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
    const DeviceOf device(h);
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
    const DeviceOf device(h);
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
    const DeviceOf device(h);
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
