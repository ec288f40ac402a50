// Pages of the block-sparse decode: which pages of 64 tokens a KV head attends to.
//
//   page_score_kernel   score of a page = max over the group's heads of sum_c max(q_c lo_c, q_c hi_c), the largest raw score any key of the
//                       page can have with any of the heads (page_boxes.h)
//   block_select_kernel the n_blocks - 1 best pages of a key stream and its newest one, ascending
//
// Which pages are read is a definite answer: products of two numbers of 32 bits or fewer are exact in 64, whatever their exponents (those of bf16
// leave the range of 32 bits), and they are added up there, so that only pages equal to 15 digits could change places.
#include "device_utils.h"
#include "internal.h"
#include "ops.h"
#include "team.h"

namespace tka {

// 16 pages per wave, four lanes a page (lane / 16), each with every fourth 16-byte piece of the boxes; the queries of up to 16 heads at a
// time in LDS, in 64 bits.  Bound by d fused products and sums in 64 bits (with a choice and a conversion each; with products of 16-bit types in 32 bits,
// which bf16's leave, it took as long) per page and head, and the read of the boxes (2 / 64 of the keys) close behind: 16384 pages, 8 KV heads, 4 heads
// each 20 us for 67 MB (3.4 TB/s), 751 pages 6.3.
constexpr int kScoreHeads = 16;
template <int DT, int D>
__global__ void __launch_bounds__(256) page_score_kernel(BlockCall a) {
    constexpr int EPL = Elem<DT>::kPerLoad, S = D / (4 * EPL), ROW = D * Elem<DT>::kBytes;
    __shared__ double qs[kScoreHeads][D];
    const int lane = lane_id(), j = lane >> 4, m = lane & 15, wave = threadIdx.x >> 6;
    const int kvh = blockIdx.y, b = blockIdx.z;
    const int64_t P = ((int64_t)a.len[b] + 63) / 64;
    const int64_t p0 = (int64_t)blockIdx.x * 64;
    if (p0 >= P) return;
    const int64_t page = p0 + wave * 16 + m, stream = (int64_t)b * a.Hkv + kvh;
    const char* box = a.boxes + (stream * a.Pcap + (page < P ? page : P - 1)) * 2 * ROW + j * 16;
    u32x4 lo[S], hi[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        lo[s] = *reinterpret_cast<const u32x4*>(box + 64 * s);
        hi[s] = *reinterpret_cast<const u32x4*>(box + ROW + 64 * s);
    }
    const char* q = static_cast<const char*>(a.q) + ((int64_t)b * a.Hq + (int64_t)kvh * a.G) * ROW;
    double best = -INFINITY;
    for (int g0 = 0; g0 < a.G; g0 += kScoreHeads) {
        const int heads = a.G - g0 < kScoreHeads ? a.G - g0 : kScoreHeads;
        if (g0) __syncthreads();
        for (int i = (int)threadIdx.x; i < heads * D / EPL; i += 256) {
            float f[EPL];
            Elem<DT>::widen(*reinterpret_cast<const u32x4*>(q + (int64_t)g0 * ROW + i * 16), f);
#pragma unroll
            for (int e = 0; e < EPL; ++e) (&qs[0][0])[i * EPL + e] = f[e];
        }
        __syncthreads();
        for (int g = 0; g < heads; ++g) {
            double sum = 0.0;
#pragma unroll
            for (int s = 0; s < S; ++s) {
                float l[EPL], h[EPL];
                Elem<DT>::widen(lo[s], l);
                Elem<DT>::widen(hi[s], h);
                const double* qc = &qs[g][(4 * s + j) * EPL];
#pragma unroll
                for (int e = 0; e < EPL; ++e) sum = fma(qc[e], (double)(qc[e] >= 0.0 ? h[e] : l[e]), sum);
            }
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (sum > best || sum != sum) best = sum;              // (a NaN stays)
        }
    }
    if (j == 0 && page < P) a.score[stream * a.Pcap + page] = best;
}

// Monotone map double -> uint64 (NaN above all: the page is attended and the NaN seen; -0 with +0).
__device__ __forceinline__ uint64_t ord_of(double v) {
    if (!(v == v)) return ~0ull;
    const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
    return u ^ ((u >> 63) ? ~0ull : 0x8000000000000000ull);
}

// One workgroup per key stream.  The page that ends the selection (its score, and among equal scores its number: lower ones first) is
// found from a linear histogram between the smallest and the largest score, whose one bin in question is ranked by direct comparison,
// or, where that bin is crowded or the scores are not finite, byte by byte of their ordered bits.  Then the pages up to it are written in
// their order.  A wave has a stretch of the pages, 64 neighbouring ones at a time; up to 16 a thread stay in registers (16384 pages, a million tokens: 14 us; 37 us
// when each of the five passes reads them again), and beyond they are read again.
constexpr int kPickThreads = 1024, kPickBins = 1024, kPickList = 2048, kPickHeld = 16;
struct PickShared {
    uint32_t tot[2][16];
    float red[2][2][16];
    uint32_t hist[kPickBins];
    uint64_t key[kPickList];
    uint32_t page[kPickList];
    uint32_t n_list, bin, need;
    uint32_t wave[kPickThreads / kWave];
    uint64_t edge_key, prefix;
    uint32_t edge_page;
};
// sum of the counts of the waves before this one (of at most 16)
__device__ __forceinline__ uint32_t row_scan_add_below(const uint32_t* count, int wave) {
    const uint32_t t = row_scan_add(count[lane_id() & 15]);
    return wave ? (uint32_t)__builtin_amdgcn_readlane((int)t, wave - 1) : 0u;
}
// HELD: pages a thread holds, or 0.
template <int HELD>
__device__ __forceinline__ void pick_pages(const double* score, int32_t* list, int64_t n, uint32_t want, PickShared& sm) {
    using Team = WorkgroupTeam<kPickThreads>;
    const int tid = (int)threadIdx.x;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t steps = (uint32_t)((n + kPickThreads - 1) / kPickThreads), end = (uint32_t)n;
    const uint32_t s0 = (uint32_t)wave * steps * kWave + (uint32_t)lane;
    double held[HELD ? HELD : 1];
    if (HELD) {
#pragma unroll
        for (uint32_t u = 0; u < HELD; ++u) held[u] = u < steps ? score[s0 + u * kWave < end ? s0 + u * kWave : end - 1] : 0.0;
    }
    // f(page, its score, there is such a page) for 64 neighbouring pages at a time, in order
    auto all = [&](auto f) {
        if (HELD) {
#pragma unroll
            for (uint32_t u = 0; u < HELD; ++u)
                if (u < steps) f(s0 + u * kWave, held[u], s0 + u * kWave < end);
        } else {
            for (uint32_t u = 0; u < steps; ++u) f(s0 + u * kWave, score[s0 + u * kWave < end ? s0 + u * kWave : end - 1], s0 + u * kWave < end);
        }
    };
    auto each = [&](auto f) {                                  // f(page, its score) for the thread's pages
        all([&](uint32_t i, double s, bool there) { if (there) f(i, s); });
    };
    // range of the scores, in 32 bits (a histogram edge needs no more)
    float lo = INFINITY, hi = -INFINITY;
    bool bad = false;
    each([&](uint32_t, double s) {
        const float v = (float)s;
        bad |= !(fabsf(v) < INFINITY);
        lo = fminf(lo, v); hi = fmaxf(hi, v);
    });
    if (bad) { lo = -INFINITY; hi = INFINITY; }
    for (int i = tid; i < kPickBins; i += kPickThreads) sm.hist[i] = 0;
    if (tid == 0) sm.n_list = 0;
    team_range<Team>(lo, hi, sm, 0);
    const float inv = (float)kPickBins / (hi - lo);
    bool listed = hi < INFINITY && lo > -INFINITY && hi > lo && inv < INFINITY;
    // (monotone: a rounding, a difference and a product with a positive number)
    auto bin_of = [&](double s) { const int x = (int)(((float)s - lo) * inv); return x < kPickBins - 1 ? x : kPickBins - 1; };
    if (listed) {
        each([&](uint32_t, double s) { atomicAdd(&sm.hist[bin_of(s)], 1u); });
        __syncthreads();
        // thread t looks at bin 1023 - t: the bin in which the want-th score from above lies
        const uint32_t c = sm.hist[kPickBins - 1 - tid];
        uint32_t total;
        const uint32_t above = team_prefix<Team>(c, total, sm, 0);
        if (above < want && above + c >= want) { sm.bin = (uint32_t)(kPickBins - 1 - tid); sm.need = want - above; }
        __syncthreads();
        const int bin = (int)sm.bin;
        listed = sm.hist[bin] <= kPickList;
        if (listed) {
            each([&](uint32_t i, double s) {
                if (bin_of(s) == bin) {
                    const uint32_t at = atomicAdd(&sm.n_list, 1u);      // (in any order: they are ranked by score and number)
                    sm.key[at] = ord_of(s); sm.page[at] = i;
                }
            });
            __syncthreads();
            const uint32_t have = sm.n_list, need = sm.need;
            for (uint32_t x = (uint32_t)tid; x < have; x += kPickThreads) {
                const uint64_t kx = sm.key[x];
                const uint32_t px = sm.page[x];
                uint32_t rank = 0;
                for (uint32_t y = 0; y < have; ++y) rank += sm.key[y] > kx || (sm.key[y] == kx && sm.page[y] < px);
                if (rank == need - 1) { sm.edge_key = kx; sm.edge_page = px; }
            }
        }
    }
    if (!listed) {
        // byte by byte: the key of the want-th page, then among the pages of that key the want-th of what is left
        uint64_t prefix = 0;
        uint32_t need = want;
        for (int shift = 56; shift >= 0; shift -= 8) {
            __syncthreads();
            for (int i = tid; i < 256; i += kPickThreads) sm.hist[i] = 0;
            __syncthreads();
            const uint64_t mask = shift == 56 ? 0ull : ~0ull << (shift + 8);
            each([&](uint32_t, double s) {
                const uint64_t k = ord_of(s);
                if ((k & mask) == prefix) atomicAdd(&sm.hist[(k >> shift) & 255], 1u);
            });
            __syncthreads();
            const uint32_t c = tid < 256 ? sm.hist[255 - tid] : 0u;
            uint32_t total;
            const uint32_t above = team_prefix<Team>(c, total, sm, 0);
            if (above < need && above + c >= need) { sm.prefix = prefix | ((uint64_t)(255 - tid) << shift); sm.need = need - above; }
            __syncthreads();
            prefix = sm.prefix; need = sm.need;
        }
        uint32_t same = 0;
        each([&](uint32_t, double s) { same += ord_of(s) == prefix; });
        same = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_add(same), kWave - 1);
        if (lane == 0) sm.wave[wave] = same;
        __syncthreads();
        uint32_t before = row_scan_add_below(sm.wave, wave);
        all([&](uint32_t i, double s, bool there) {
            const bool eq = there && ord_of(s) == prefix;
            const uint64_t m = __ballot(eq);
            if (eq && before + (uint32_t)mask_rank(m) == need - 1) { sm.edge_key = prefix; sm.edge_page = i; }
            before += (uint32_t)__popcll(m);
        });
    }
    __syncthreads();
    const uint64_t edge_key = sm.edge_key;                     // selected: key > edge_key, or equal and page <= edge_page
    const uint32_t edge_page = sm.edge_page;
    auto picked = [&](uint32_t i, double s) {
        const uint64_t k = ord_of(s);
        return k > edge_key || (k == edge_key && i <= edge_page);
    };
    uint32_t mine = 0;
    each([&](uint32_t i, double s) { mine += picked(i, s); });
    mine = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_add(mine), kWave - 1);
    __syncthreads();                                           // (sm.wave has been read)
    if (lane == 0) sm.wave[wave] = mine;
    __syncthreads();
    int32_t* to = list + (row_scan_add_below(sm.wave, wave));
    if (mine == 0) return;
    all([&](uint32_t i, double s, bool there) {
        const bool in = there && picked(i, s);
        const uint64_t m = __ballot(in);
        if (in) to[mask_rank(m)] = (int32_t)i;
        to += __popcll(m);
    });
}
__global__ void __launch_bounds__(kPickThreads) block_select_kernel(BlockCall a) {
    __shared__ PickShared sm;
    const int tid = (int)threadIdx.x;
    const int64_t stream = blockIdx.x;
    const int64_t P = ((int64_t)a.len[stream / a.Hkv] + 63) / 64;
    int32_t* const list = a.list + stream * a.list_stride;
    if (P <= a.n_blocks) {                                     // all of them
        for (int64_t i = tid; i < a.n_blocks; i += kPickThreads) list[i] = i < P ? (int32_t)i : -1;
        return;
    }
    const double* const score = a.score + stream * a.Pcap;
    const uint32_t want = (uint32_t)a.n_blocks - 1;            // 0 <= want < P - 1: the newest page is in without a search
    if (tid == 0) list[want] = (int32_t)(P - 1);
    if (want == 0) return;
    if (P - 1 <= kPickThreads) pick_pages<1>(score, list, P - 1, want, sm);
    else if (P - 1 <= 4 * kPickThreads) pick_pages<4>(score, list, P - 1, want, sm);
    else if (P - 1 <= kPickHeld * kPickThreads) pick_pages<kPickHeld>(score, list, P - 1, want, sm);
    else pick_pages<0>(score, list, P - 1, want, sm);
}

hipError_t launch_block_scores(const BlockCall& a, hipStream_t st) {
    const dim3 grid((unsigned)((a.pages + 63) / 64), (unsigned)a.Hkv, (unsigned)a.B);
#define TKA_SCORES(DT_, D_) hipLaunchKernelGGL((page_score_kernel<DT_, D_>), grid, dim3(256), 0, st, a)
    TKA_BY_TYPE_AND_DIM(TKA_SCORES, a.dtype, a.D);
#undef TKA_SCORES
    return hipGetLastError();
}

hipError_t launch_block_select(const BlockCall& a, hipStream_t st) {
    hipLaunchKernelGGL(block_select_kernel, dim3((unsigned)(a.B * a.Hkv)), dim3(kPickThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace tka
