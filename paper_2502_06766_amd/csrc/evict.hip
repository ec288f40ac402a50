// Accumulated attention weight of the cached tokens: eviction by it (topk_attn_evict), and its accumulation from a top-k selection
// (topk_attn_add_mass; dense.hip adds it up in the dense and block-sparse decodes).
//
//   evict_select_kernel, evict_step_kernel
//                        survivors of each key stream, ascending: the newest tokens and the heaviest of the older ones
//   evict_move_kernel    their rows to the front of the cache, in place: keys, values, accumulators, int8 codes and scales
//   add_mass_kernel      mass[position] += exp(score / sqrt(d) - lse)
#include "device_utils.h"
#include "internal.h"
#include "ops.h"
#include "team.h"

namespace tka {

// Monotone map of an accumulated weight to 32 bits (NaN below all numbers, -0 with +0).
__device__ __forceinline__ uint32_t mass_key(float v) { return v == v ? ord_from_bits(__float_as_uint(v + 0.0f)) : 0u; }
constexpr uint32_t kZeroMass = 0x80000000u;      // of zero: tokens no query has attended to, often most of a cache

// The weight of the last survivor is found from the top of the keys' bits: 11 of them by a histogram in LDS, then 11 and 10 more among the keys
// that share the ones before (or, where at most 512 keys do after the first, those compared with each other); then the survivors are written
// in order, a stretch of the cache per wave.  One workgroup has up to 16384 tokens of a key stream in its registers and does it all
// (8065 tokens 13 us).  Longer streams are cut into up to eight chunks and take a launch per step, each workgroup adding up the chunks'
// histograms of the step before for itself (32 streams of 19k to 100k tokens: 84 us in one
// workgroup each, 32 in four launches); chunks of more than 16384 tokens are read again by each step.
constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave, kEvictList = 512, kEvictHeld = 16;
constexpr int kEvictCopies = 4;       // of a histogram, for every fourth lane one (16384 tokens of 80 different bins 9.2 -> 6.5 us), 16 banks apart
struct EvictShared {
    uint32_t tot[2][16];
    uint32_t hist_[kEvictCopies][kEvictBins + 16];
    __device__ __forceinline__ uint32_t count(int bin) const { return (hist_[0][bin] + hist_[1][bin]) + (hist_[2][bin] + hist_[3][bin]); }
    uint32_t list[kEvictList];
    uint32_t n_list, prefix, need;
    uint32_t above[kEvictWaves], equal[kEvictWaves];
};
using EvictTeam = WorkgroupTeam<kEvictThreads>;
// position of step `pass` among a key's bits
__device__ __forceinline__ constexpr int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ constexpr int digit_bits(int pass) { return pass == 2 ? 10 : 11; }

// The keys of tokens [c0, c1), c1 > c0: each wave has a stretch of `steps` times 64 neighbouring ones.
template <bool HELD> struct KeyWalk {
    const float* mass;
    uint32_t c1, s0, steps;                                    // (a cache has fewer than 2^31 tokens, by 256 at least: no sum here reaches 2^32)
    uint32_t held[HELD ? kEvictHeld : 1];
    __device__ __forceinline__ KeyWalk(const float* m, int64_t c0, int64_t end) : mass(m), c1((uint32_t)end) {
        steps = (uint32_t)((end - c0 + kEvictThreads - 1) / kEvictThreads);
        s0 = (uint32_t)c0 + (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * steps * kWave + (uint32_t)lane_id();
        if (HELD) {
            float v[HELD ? kEvictHeld : 1];
#pragma unroll
            for (uint32_t u = 0; u < (HELD ? kEvictHeld : 1); ++u) v[u] = u < steps ? mass[s0 + u * kWave < c1 ? s0 + u * kWave : c1 - 1] : 0.f;
#pragma unroll
            for (int u = 0; u < (HELD ? kEvictHeld : 1); ++u) held[u] = mass_key(v[u]);
        }
    }
    // f(position, key, there is such a token) for 64 neighbouring tokens at a time, in order
    template <class F> __device__ __forceinline__ void each(F f) const {
        if (HELD) {
#pragma unroll
            for (uint32_t u = 0; u < (HELD ? kEvictHeld : 1); ++u)
                if (u < steps) f(s0 + u * kWave, held[u], s0 + u * kWave < c1);
        } else {
            constexpr uint32_t U = 16;
            for (uint32_t u0 = 0; u0 < steps; u0 += U) {
                const uint32_t i = s0 + u0 * kWave;
                float v[U];
#pragma unroll
                for (uint32_t u = 0; u < U; ++u) v[u] = mass[i + u * kWave < c1 ? i + u * kWave : c1 - 1];
#pragma unroll
                for (uint32_t u = 0; u < U; ++u)
                    if (u0 + u < steps) f(i + u * kWave, mass_key(v[u]), i + u * kWave < c1);
            }
        }
    }
};
// Histogram of step `pass` of the keys whose higher bits are those of `prefix`, in sm.count() (the caller waits).
template <class Walk>
__device__ __forceinline__ void digit_histogram(const Walk& keys, int pass, uint32_t prefix, EvictShared& sm) {
    const int shift = digit_shift(pass), bits = digit_bits(pass);
    const uint32_t mask = pass == 0 ? 0u : ~0u << (shift + bits);
    for (int i = (int)threadIdx.x; i < kEvictCopies * (kEvictBins + 16); i += kEvictThreads) (&sm.hist_[0][0])[i] = 0;
    __syncthreads();
    uint32_t* const hist = sm.hist_[threadIdx.x % kEvictCopies];
    uint32_t zeros = 0;                                        // (counted apart: thousands of additions to one counter otherwise)
    keys.each([&](uint32_t, uint32_t k, bool there) {
        if (!there) return;
        if (k == kZeroMass) ++zeros;
        else if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
    });
    if (zeros && (kZeroMass & mask) == prefix) atomicAdd(&hist[(kZeroMass >> shift) & ((1u << bits) - 1)], zeros);
}
// Thread t brings the counts of bins 2047 - 2 t and 2046 - 2 t.  `prefix` grows by the bin that the need-th key from above lies in, `need` becomes
// its rank there.  (The caller waits before sm.prefix and sm.need are used again.)
__device__ __forceinline__ void digit_pick(uint32_t c1, uint32_t c0, int pass, uint32_t& prefix, uint32_t& need, EvictShared& sm) {
    const int tid = (int)threadIdx.x;
    uint32_t total;
    const uint32_t above = team_prefix<EvictTeam>(c1 + c0, total, sm, pass & 1);
    if (above < need && above + c1 + c0 >= need) {
        const bool upper = above + c1 >= need;
        sm.prefix = prefix | ((uint32_t)(kEvictBins - 1 - 2 * tid - (upper ? 0 : 1)) << digit_shift(pass));
        sm.need = need - above - (upper ? 0 : c1);
    }
    __syncthreads();
    prefix = sm.prefix; need = sm.need;
}
// Survivors among the walk's tokens: a key above `edge`, or one of the first `need` equal to it, counting `equal_before` of them before; the first
// one goes to kept[at].
template <class Walk>
__device__ __forceinline__ void write_survivors(const Walk& keys, uint32_t edge, uint32_t need, uint32_t at, uint32_t equal_before, int32_t* kept,
                                                EvictShared& sm) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    uint32_t above = 0, equal = 0;
    keys.each([&](uint32_t, uint32_t k, bool there) { above += there && k > edge; equal += there && k == edge; });
    above = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_add(above), kWave - 1);
    equal = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_add(equal), kWave - 1);
    if (lane_id() == 0) { sm.above[wave] = above; sm.equal[wave] = equal; }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        const uint32_t left = equal_before < need ? need - equal_before : 0u;
        at += sm.above[w] + (sm.equal[w] < left ? sm.equal[w] : left);
        equal_before += sm.equal[w];
    }
    int32_t* to = kept + at;
    if (equal == 0 || equal_before >= need) {                  // (of the wave's tokens none that is equal survives, as in most waves)
        keys.each([&](uint32_t i, uint32_t k, bool there) {
            const uint64_t m = __ballot(there && k > edge);
            if (there && k > edge) to[mask_rank(m)] = (int32_t)i;
            to += __popcll(m);
        });
        return;
    }
    keys.each([&](uint32_t i, uint32_t k, bool there) {
        const uint64_t eq = __ballot(there && k == edge);
        const bool keep = there && (k > edge || (k == edge && equal_before + (uint32_t)mask_rank(eq) < need));
        const uint64_t m = __ballot(keep);
        if (keep) to[mask_rank(m)] = (int32_t)i;
        to += __popcll(m);
        equal_before += (uint32_t)__popcll(eq);
    });
}

// What there is to select of a stream: `want` of the first n tokens (0: nothing).  With `first` also what needs no selection: the newest tokens,
// or all, and the scratch of the move.
__device__ __forceinline__ uint32_t evict_task(const EvictCall& a, int64_t stream, bool first, int64_t& n) {
    const int tid = (int)threadIdx.x, b = (int)(stream / a.Hkv);
    const int64_t N = a.len[b];
    int32_t* const kept = a.kept + stream * a.budget;
    if (first) {
        for (int i = tid; i <= a.units; i += kEvictThreads) a.state[stream * (a.units + 1) + i] = 0u;
        if (tid == 0 && stream == (int64_t)b * a.Hkv) a.old_len[b] = (int32_t)N;
    }
    if (N <= a.budget) {                                       // all stay
        if (first)
            for (int64_t i = tid; i < a.budget; i += kEvictThreads) kept[i] = i < N ? (int32_t)i : -1;
        return 0;
    }
    n = N - a.recent;                                          // older tokens
    const uint32_t want = (uint32_t)(a.budget - a.recent);     // of them survive; want < n
    if (first)
        for (int64_t i = tid; i < a.recent; i += kEvictThreads) kept[want + i] = (int32_t)(n + i);
    return want;
}

__global__ void __launch_bounds__(kEvictThreads) evict_select_kernel(EvictCall a) {
    __shared__ EvictShared sm;
    const int64_t stream = blockIdx.x;
    const int tid = (int)threadIdx.x;
    int64_t n = 0;
    uint32_t need = evict_task(a, stream, true, n), prefix = 0;
    if (need == 0) return;
    const KeyWalk<true> keys(a.mass + stream * a.Ncap, 0, n);
    for (int pass = 0; pass < 3; ++pass) {
        digit_histogram(keys, pass, prefix, sm);
        if (tid == 0) sm.n_list = 0;
        __syncthreads();
        digit_pick(sm.count(kEvictBins - 1 - 2 * tid), sm.count(kEvictBins - 2 - 2 * tid), pass, prefix, need, sm);
        const uint32_t have = sm.count((int)(prefix >> digit_shift(0)));
        if (pass == 0 && have <= kEvictList) {
            keys.each([&](uint32_t, uint32_t k, bool there) {
                if (there && (k >> digit_shift(0)) == (prefix >> digit_shift(0))) sm.list[atomicAdd(&sm.n_list, 1u)] = k;
            });
            __syncthreads();
            if (tid < (int)have) {
                const uint32_t k = sm.list[tid];
                uint32_t more = 0, same = 0;
                for (uint32_t y = 0; y < have; ++y) { more += sm.list[y] > k; same += sm.list[y] == k; }
                if (more < need && more + same >= need) { sm.prefix = k; sm.need = need - more; }      // (all that are equal say the same)
            }
            __syncthreads();
            prefix = sm.prefix; need = sm.need;
            break;
        }
        __syncthreads();
    }
    write_survivors(keys, prefix, need, 0, 0, a.kept + stream * a.budget, sm);
}

// The same in steps, a launch each; grid (streams, chunks).  pick: per stream the prefix and rank after the steps so far, and per chunk the keys
// above the second step's prefix.  The histograms of a step lie in one of two places, those of the step before in the other.
template <int PASS, bool HELD>
__global__ void __launch_bounds__(kEvictThreads) evict_step_kernel(EvictCall a) {
    __shared__ EvictShared sm;
    const int64_t stream = blockIdx.x;
    const int tid = (int)threadIdx.x, chunk = (int)blockIdx.y, lane = lane_id();
    int64_t n = 0;
    uint32_t need = evict_task(a, stream, PASS == 0 && chunk == 0, n), prefix = 0;
    const int64_t c0 = chunk * a.chunk;
    if (need == 0 || c0 >= n) return;
    const int n_chunks = (int)((n + a.chunk - 1) / a.chunk);
    const KeyWalk<HELD> keys(a.mass + stream * a.Ncap, c0, c0 + a.chunk < n ? c0 + a.chunk : n);
    uint32_t* const pick = a.pick + stream * kEvictPick;
    if (PASS > 0) {
        if (PASS > 1) { prefix = pick[2 * (PASS - 2)]; need = pick[2 * (PASS - 2) + 1]; }
        const uint32_t* before = a.hist + (stream * 2 + ((PASS - 1) & 1)) * kEvictChunks * kEvictBins;
        uint32_t c1 = 0, c0_ = 0;
        uint2 v[kEvictChunks];                                 // (all asked for at once)
#pragma unroll
        for (int x = 0; x < kEvictChunks; ++x)
            v[x] = x < n_chunks ? *reinterpret_cast<const uint2*>(before + x * kEvictBins + kEvictBins - 2 - 2 * tid) : make_uint2(0u, 0u);
#pragma unroll
        for (int x = 0; x < kEvictChunks; ++x) { c0_ += v[x].x; c1 += v[x].y; }
        digit_pick(c1, c0_, PASS - 1, prefix, need, sm);
        if (chunk == 0 && tid == 0) { pick[2 * (PASS - 1)] = prefix; pick[2 * (PASS - 1) + 1] = need; }
    }
    if (PASS < 3) {
        digit_histogram(keys, PASS, prefix, sm);
        if (PASS == 2) {
            uint32_t above = 0;
            keys.each([&](uint32_t, uint32_t k, bool there) { above += there && (k >> digit_shift(1)) > (prefix >> digit_shift(1)); });
            above = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_add(above), kWave - 1);
            if (lane == 0) sm.above[tid >> 6] = above;
        }
        __syncthreads();
        uint32_t* mine = a.hist + ((stream * 2 + (PASS & 1)) * kEvictChunks + chunk) * kEvictBins;
        for (int i = tid; i < kEvictBins; i += kEvictThreads) mine[i] = sm.count(i);
        if (PASS == 2 && tid == 0) {
            uint32_t above = 0;
            for (int w = 0; w < kEvictWaves; ++w) above += sm.above[w];
            pick[6 + chunk] = above;
        }
        return;
    }
    // survivors in the chunks before: above the second step's prefix, above it in the third digit, equal to it
    const uint32_t* last = a.hist + (stream * 2) * kEvictChunks * kEvictBins;
    const uint32_t digit = prefix & ((1u << digit_bits(2)) - 1);
    const int wave = tid >> 6;
    if (wave < chunk) {
        uint32_t more = 0;
        for (uint32_t i = digit + 1 + (uint32_t)lane; i < (1u << digit_bits(2)); i += kWave) more += last[wave * kEvictBins + i];
        more = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_add(more), kWave - 1);
        if (lane == 0) { sm.list[2 * wave] = pick[6 + wave] + more; sm.list[2 * wave + 1] = last[wave * kEvictBins + digit]; }
    }
    __syncthreads();
    uint32_t at = 0, equal_before = 0;
    for (int x = 0; x < chunk; ++x) {
        const uint32_t left = equal_before < need ? need - equal_before : 0u, same = sm.list[2 * x + 1];
        at += sm.list[2 * x] + (same < left ? same : left);
        equal_before += same;
    }
    write_survivors(keys, prefix, need, at, equal_before, a.kept + stream * a.budget, sm);
}

// Row j of the cache becomes row kept[j] >= j, for all j of a stream, in place.  A workgroup holds a unit of neighbouring rows j in
// registers; it may overwrite them once every unit whose sources lie among them has read its own.  Those are units before it (kept[j] >= j),
// each of which raises a flag when its loads have come back and waits for nothing before that.  The units of a stream are handed out by a
// counter, so those before a unit are always in the hands of a workgroup that runs or has run: every wait ends.  (A counter a stream, and the
// streams in turn, so that the units before one were handed out some time ago: one counter, stream after stream, took 131 us where this takes
// 117.)  Flags carry no data (the rows themselves were written by earlier launches), so they need no more than the loads' return in front of them.
// One read and one write of the rows that move; through a buffer it would be two of each.  32 streams cut to 16384 tokens (537 MB): 117 to 121
// us, 4.4 to 4.6 TB/s (a large copy reaches 4.8).
__global__ void __launch_bounds__(256) evict_move_kernel(EvictCall a) {
    __shared__ uint32_t ticket;
    const int64_t stream = blockIdx.x % (uint32_t)(a.B * a.Hkv);
    uint32_t* flags = a.state + stream * (a.units + 1);
    if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add(flags, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    int unit = (int)ticket;                                     // (as many workgroups as units have the stream)
    ++flags;
    const int b = (int)(stream / a.Hkv);
    const int64_t N = a.old_len[b];
    if (N <= a.budget) return;                                  // (the whole stream: nobody waits for it)
    if (unit == 0 && stream == (int64_t)b * a.Hkv && threadIdx.x == 0) a.len[b] = (int32_t)a.budget;
    int x = 0;
    while (unit >= a.array[x].units) { unit -= a.array[x].units; flags += a.array[x].units; ++x; }
    const EvictArray arr = a.array[x];
    const int64_t end = arr.cleared ? N : a.budget;
    const int64_t j0 = (int64_t)unit * arr.unit_rows;
    if (j0 >= end) return;
    const int64_t j1 = j0 + arr.unit_rows < end ? j0 + arr.unit_rows : end;
    const int32_t* const kept = a.kept + stream * a.budget;
    if (j1 <= a.budget && kept[j1 - 1] == (int32_t)(j1 - 1)) return;      // all in place (and not a source of other rows)
    char* const base = arr.base + stream * a.Ncap * arr.row;
    const bool wide = arr.row >= 16;
    const int per_row = wide ? arr.row / 16 : 1, log2_per = 31 - __builtin_clz((uint32_t)per_row);
    const int pieces = (int)(j1 - j0) * per_row;
    u32x4 held[kEvictPieces];
    int32_t from[kEvictPieces];
#pragma unroll
    for (int u = 0; u < kEvictPieces; ++u) {
        const int p = u * 256 + (int)threadIdx.x;
        const int64_t j = j0 + ((p < pieces ? p : pieces - 1) >> log2_per);
        from[u] = j < a.budget ? kept[j] : -1;
    }
#pragma unroll
    for (int u = 0; u < kEvictPieces; ++u) {
        const int p = u * 256 + (int)threadIdx.x, part = (p < pieces ? p : pieces - 1) & (per_row - 1);
        held[u] = u32x4{0u, 0u, 0u, 0u};
        if (from[u] >= 0) {
            const char* src = base + (int64_t)from[u] * arr.row + part * 16;
            if (wide) held[u] = *reinterpret_cast<const u32x4*>(src);
            else held[u].x = *reinterpret_cast<const uint32_t*>(src);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // the rows are here
    __syncthreads();
    if (threadIdx.x == 0) __hip_atomic_store(&flags[unit], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int64_t w = (int64_t)threadIdx.x; w < unit; w += 256) {
        const int64_t last = (w + 1) * arr.unit_rows < a.budget ? (w + 1) * arr.unit_rows : a.budget;
        if (w * arr.unit_rows >= a.budget || kept[last - 1] < (int32_t)j0) continue;      // reads nothing from here on
        while (__hip_atomic_load(&flags[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0u) __builtin_amdgcn_s_sleep(2);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kEvictPieces; ++u) {
        const int p = u * 256 + (int)threadIdx.x;
        if (p < pieces) {
            char* dst = base + (j0 + (p >> log2_per)) * arr.row + (p & (per_row - 1)) * 16;
            if (wide) *reinterpret_cast<u32x4*>(dst) = held[u];
            else *reinterpret_cast<uint32_t*>(dst) = held[u].x;
        }
    }
}

// One workgroup per key stream takes its heads one after the other (the positions of a head are distinct), so the sums come out the
// same in every run: a chain of trips to memory, two a head.  256 positions of 32 heads 5.9 us, 16 sequences of 1024 positions 11; 16384
// positions of 32 heads over 8, of a million tokens, 145 a call: 8 workgroups, 4 heads one after the other.
constexpr int kMassThreads = 1024;
__global__ void __launch_bounds__(kMassThreads) add_mass_kernel(MassCall a) {
    const int64_t stream = blockIdx.x;
    const int64_t b = stream / a.Hkv, kvh = stream - b * a.Hkv;
    float* const mass = a.mass + stream * a.Ncap;
    for (int g = 0; g < a.G; ++g) {
        const int64_t bh = b * a.Hq + kvh * a.G + g;
        const float lse2 = a.lse[bh] * 1.4426950408889634f;
        const int32_t* idx = a.idx + bh * a.k;
        const float* vals = a.vals + bh * a.k;
        constexpr int U = 4;
        for (int i0 = (int)threadIdx.x; i0 < a.k; i0 += U * kMassThreads) {
            int32_t at[U];
            float w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kMassThreads;
                at[u] = i < a.k ? idx[i] : -1;
                w[u] = i < a.k ? vals[i] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (at[u] < 0 || at[u] >= a.Ncap) continue;
                mass[at[u]] += exp2f(fmaf(w[u], a.scale_log2e, -lse2));
            }
        }
        __syncthreads();
    }
}

hipError_t launch_evict(const EvictCall& a, hipStream_t st) {
    const int64_t streams = (int64_t)a.B * a.Hkv;
    if (streams * a.units > kMostWorkgroups) return hipErrorInvalidValue;
    if (a.longest <= kEvictHeldTokens) {
        hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)streams), dim3(kEvictThreads), 0, st, a);
    } else {
        const dim3 grid((unsigned)streams, (unsigned)((a.longest + a.chunk - 1) / a.chunk));
#define TKA_STEP(PASS_)                                                                                                            \
    do {                                                                                                                          \
        if (a.chunk <= kEvictHeldTokens) hipLaunchKernelGGL((evict_step_kernel<PASS_, true>), grid, dim3(kEvictThreads), 0, st, a); \
        else hipLaunchKernelGGL((evict_step_kernel<PASS_, false>), grid, dim3(kEvictThreads), 0, st, a);                            \
    } while (0)
        TKA_STEP(0); TKA_STEP(1); TKA_STEP(2); TKA_STEP(3);
#undef TKA_STEP
    }
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(streams * a.units)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_add_mass(const MassCall& a, hipStream_t st) {
    hipLaunchKernelGGL(add_mass_kernel, dim3((unsigned)(a.B * a.Hkv)), dim3(kMassThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace tka
