// Launchers of the operators beside the top-k decode (dense.hip, blocks.hip, rotary.hip, evict.hip), called by api_ops.hip.
#pragma once
#include "internal.h"

namespace tka {

// CALL(DT, D) for the handle's type and head dimension.
#define TKA_BY_TYPE_AND_DIM(CALL, dtype, D)                                                                                \
    do {                                                                                                                   \
        if ((dtype) == DT_F16) { if ((D) == 32) CALL(DT_F16, 32); else if ((D) == 64) CALL(DT_F16, 64);                     \
                                 else if ((D) == 128) CALL(DT_F16, 128); else CALL(DT_F16, 256); }                         \
        else if ((dtype) == DT_BF16) { if ((D) == 32) CALL(DT_BF16, 32); else if ((D) == 64) CALL(DT_BF16, 64);             \
                                       else if ((D) == 128) CALL(DT_BF16, 128); else CALL(DT_BF16, 256); }                 \
        else { if ((D) == 32) CALL(DT_F32, 32); else if ((D) == 64) CALL(DT_F32, 64);                                       \
               else if ((D) == 128) CALL(DT_F32, 128); else CALL(DT_F32, 256); }                                           \
    } while (0)

// A launch has fewer than 2^32 threads.
constexpr int64_t kMostWorkgroups = (1 << 24) - 1;     // of 256
constexpr int64_t kMostStreams = (1 << 22) - 1;        // one workgroup of 1024 each

constexpr int kMostSelected = 1 << 28;                 // the largest max_k of a handle

constexpr int kMaxSplits = 256;  // splits of a sequence (their factors sit in LDS when they are joined)

// The first `sinks` and the newest `window` (>= 1) of N tokens, in pages of 64 rows: those of the first ones from the front, those of the
// newest ones from the first token of the window on, so that a page has rows to leave out at its end only.
struct WindowWalk {
    int64_t N, first, sinks, sink_pages;     // (first token of the window; sinks in front of it)
    __host__ __device__ WindowWalk(int64_t n, int64_t sinks_, int64_t window) : N(n) {
        first = window < n ? n - window : 0;
        if (sinks_ >= first) { first = 0; sinks_ = 0; }
        sinks = sinks_;
        sink_pages = (sinks + 63) / 64;
    }
    __host__ __device__ int64_t pages() const { return sink_pages + (N - first + 63) / 64; }
    __host__ __device__ int64_t row(int64_t page) const { return page < sink_pages ? page * 64 : first + (page - sink_pages) * 64; }
    __host__ __device__ int64_t end(int64_t page) const { return page < sink_pages ? sinks : N; }     // row that the page's stretch ends before
};

// Splits of the keys of [heads] and what they leave.
struct SplitParts {
    float* part_acc;            // [heads][n_split][D] weighted sums of the splits
    float* part_lm;             // [heads][n_split][2] their sums of weights, and the score the weights are relative to (times log2(e) / sqrt(D))
    float* out;                 // [heads][D]
    float* lse;                 // [heads] or null
    int n_split;                // splits of the longest sequence
    int D;
};

// Attention of one query per sequence and head over all cached tokens, the newest and the first ones, or a list of pages of 64 tokens; or of the last
// M tokens' queries (few of them, 32 bits), each over what it sees: then a row is a query and a head of the group, m G + g, as in prompt.h.
struct AttendCall : SplitParts {
    const char* K;              // this layer's keys and values [B][Hkv][Ncap][D]
    const char* V;
    const void* q;              // [B][Hq][D]
    const int32_t* len;         // [B]
    const int32_t* list;        // [B][Hkv][list_stride] pages to attend, ascending, or null: all
    int64_t list_stride;
    int n_list;                 // pages of a list (a sequence of fewer pages: all of its own)
    uint32_t* arrive;           // [B][Hkv][row_blocks] splits that are done; zero between calls
    float* scores;              // [B*Hq][score_stride] raw scores in the order of the walk, kept for `mass`
    int64_t score_stride;
    float* mass;                // [B][Hkv][Ncap] or null
    int64_t Ncap;
    int64_t walk;               // most keys a sequence's walk covers, whole pages
    int64_t sinks, window;      // window > 0: the first `sinks` and the newest `window` tokens alone
    int64_t reach;              // tokens some query's window has: window + M - 1
    void* out_rows;             // M > 0: [B][M][Hq][D] in the type of q (lse [B][M][Hq])
    int M;                      // 0: one query per sequence
    int rows;                   // of a key stream: G, or M G
    int B, Hq, Hkv, G, dtype;
    int chunk;                  // pages per split
    int join_later;             // the splits are put together in a launch of its own,
    int join_heads;             // by a workgroup per head (1) or per block of heads (16)
    int row_blocks;             // blocks of 16 rows
    float scale_log2e;          // log2(e) / sqrt(D)
};
constexpr int kMassPerBlock = 1024;      // keys whose weights one workgroup adds up
// Workgroups of the walk, of the joins after it and of the sums of weights.
inline int64_t attend_walk_wgs(const AttendCall& a) {
    const int64_t units = (int64_t)a.B * a.Hkv * a.n_split;
    return a.row_blocks > 1 ? (units + 7) / 8 * 8 * a.row_blocks : units;
}
inline int64_t attend_join_wgs(const AttendCall& a) {
    return a.join_later && a.n_split > 1 ? (int64_t)a.B * a.Hkv * (a.join_heads == 1 ? a.rows : a.row_blocks) : 0;
}
inline int64_t attend_mass_wgs(const AttendCall& a) {
    return a.mass ? (int64_t)a.B * a.Hkv * ((a.walk + kMassPerBlock - 1) / kMassPerBlock) : 0;
}
hipError_t launch_attend(const AttendCall& a, hipStream_t st);
constexpr int kFewRows = 128;            // rows of a key stream that the kernels of single tokens take at most

// Pages of the block-sparse decode.
struct BlockCall {
    const char* boxes;          // this layer's [B][Hkv][Pcap][2][D]
    const void* q;              // [B][Hq][D]
    const int32_t* len;         // [B]
    double* score;              // [B][Hkv][Pcap]
    int32_t* list;              // [B][Hkv][list_stride]
    int64_t list_stride, Pcap;
    int64_t pages;              // of the longest sequence
    int n_blocks;
    int B, Hq, Hkv, G, D, dtype;
};
hipError_t launch_block_scores(const BlockCall& a, hipStream_t st);
hipError_t launch_block_select(const BlockCall& a, hipStream_t st);

// Projections of new tokens into the cache, keys (and queries) normalised and rotated on the way.
struct RotaryCall {
    const char* q;              // element (b, t, h, c) at b * q_seq + t * q_token + h * D + c (bytes); null: keys and values only
    const char* k;
    const char* v;
    int64_t q_seq, q_token, k_seq, k_token, v_seq, v_token;
    char* q_out;                // [B][n][Hq][D]
    char* K;                    // first sequence's keys and values [B][Hkv][Ncap][D]
    char* V;
    const void* q_norm;         // [D] or null
    const void* k_norm;
    const float* inv_freq;      // [rotary / 2]
    const int32_t* positions;   // [B][n] or null: the row the token goes to
    int32_t* len;               // [B]
    int8_t* codes;              // int8 index of the first sequence [B][Hkv][Ncap][D], or null
    float* scales;
    int64_t Ncap, n;
    int64_t base;               // length of all sequences before the call, or -1: as the device has it
    int advance;                // the kernel advances the lengths itself (for base >= 0, or n = 1)
    int B, Hq, Hkv, D, dtype, rotary, interleaved;
    float eps;
};
hipError_t launch_rotary(const RotaryCall& a, hipStream_t st);

// Eviction: the survivors' old positions, then the rows moved to the front.
struct EvictArray {
    char* base;                 // [B * Hkv][Ncap] rows
    int row;                    // bytes of a row: 4, or a multiple of 16
    int unit_rows;              // rows a workgroup holds at a time
    int units;                  // units per key stream
    int cleared;                // rows behind the survivors are cleared
};
constexpr int kEvictArrays = 5; // keys, values, mass, codes, scales
constexpr int kEvictBins = 2048, kEvictChunks = 8;     // bins of a step of the selection, chunks of a key stream
constexpr int64_t kEvictHeldTokens = 16384;            // tokens one workgroup holds
constexpr int kEvictPick = 16;
struct EvictCall {
    EvictArray array[kEvictArrays];
    int n_arrays, units;        // units per key stream over all arrays
    float* mass;                // [B][Hkv][Ncap]
    int32_t* len;               // [B]
    int32_t* kept;              // [B][Hkv][budget], or scratch of the same shape
    uint32_t* state;            // scratch [B * Hkv][1 + units]: the next unit, then a flag per unit
    int32_t* old_len;           // scratch [B]
    uint32_t* hist;             // scratch [B * Hkv][2][kEvictChunks][kEvictBins], for streams of more than kEvictHeldTokens
    uint32_t* pick;             // scratch [B * Hkv][kEvictPick]
    int64_t Ncap, budget, recent;
    int64_t longest;            // older tokens of the longest sequence
    int64_t chunk;              // tokens of a chunk
    int B, Hkv;
};
constexpr int kEvictPieces = 16;                       // 16-byte pieces a thread of a unit holds
constexpr int kEvictUnitBytes = 256 * 16 * kEvictPieces;
hipError_t launch_evict(const EvictCall& a, hipStream_t st);
hipError_t launch_balls_again(int dtype, int D, const void* K, int64_t Ncap, int64_t Pcap, int Hkv, int B, const int32_t* len_dev,
                              int64_t rows, void* centres, float* balls, hipStream_t st);

// Weights of a top-k selection added to the accumulators.
struct MassCall {
    const int32_t* idx;         // [B][Hq][k]
    const float* vals;
    const float* lse;           // [B][Hq]
    float* mass;                // [B][Hkv][Ncap]
    int64_t Ncap;
    int B, Hq, Hkv, G, k;
    float scale_log2e;
};
hipError_t launch_add_mass(const MassCall& a, hipStream_t st);

}  // namespace tka
