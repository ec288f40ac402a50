// Accumulated attention weight of the cached tokens: eviction by it (topk_attn_evict), and its accumulation from a top-k selection
// (topk_attn_add_mass; dense.hip adds it up in the dense and block-sparse decodes).
//
//   evict_select_kernel  survivors of each key stream, ascending: the newest tokens and the heaviest of the older ones
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

// One workgroup per key stream: the weight of the last survivor by 11, 11 and 10 bits of its key from the top, then the survivors in
// order, a stretch of the cache per wave.  Reads the weights five times, from L2 but for the first (4 bytes a token; a moved token is
// 4 d e of them): one compute unit's share of L2, 64 bytes a clock, is what bounds it.
constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave, kEvictBins = 2048;
__global__ void __launch_bounds__(kEvictThreads) evict_select_kernel(EvictCall a) {
    using Team = WorkgroupTeam<kEvictThreads>;
    struct SM {
        uint32_t tot[2][16];
        uint32_t hist[kEvictBins];
        uint32_t prefix, need;
        uint32_t above[kEvictWaves], equal[kEvictWaves];
    };
    __shared__ SM sm;
    const int tid = (int)threadIdx.x, lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t stream = blockIdx.x;
    const int b = (int)(stream / a.Hkv);
    const int64_t N = a.len[b];
    int32_t* const kept = a.kept + stream * a.budget;
    for (int i = tid; i < a.units; i += kEvictThreads) a.state[1 + stream * a.units + i] = 0u;
    if (tid == 0) {
        if (stream == 0) a.state[0] = 0u;
        if (stream == (int64_t)b * a.Hkv) a.old_len[b] = (int32_t)N;
    }
    if (N <= a.budget) {                                       // all stay
        for (int64_t i = tid; i < a.budget; i += kEvictThreads) kept[i] = i < N ? (int32_t)i : -1;
        return;
    }
    const float* const mass = a.mass + stream * a.Ncap;
    const int64_t n = N - a.recent;                            // older tokens
    const uint32_t want = (uint32_t)(a.budget - a.recent);     // of them survive; want < n
    for (int64_t i = tid; i < a.recent; i += kEvictThreads) kept[want + i] = (int32_t)(n + i);
    if (want == 0) return;
    uint32_t prefix = 0, need = want;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        const uint32_t mask = pass == 0 ? 0u : ~0u << (shift + bits);
        for (int i = tid; i < kEvictBins; i += kEvictThreads) sm.hist[i] = 0;
        __syncthreads();
        uint32_t zeros = 0;                                    // (counted apart: thousands of additions to one counter otherwise)
        auto count = [&](uint32_t k) {
            if (k == kZeroMass) ++zeros;
            else if ((k & mask) == prefix) atomicAdd(&sm.hist[(k >> shift) & ((1u << bits) - 1)], 1u);
        };
        int64_t i = tid;
        for (; i + 7 * kEvictThreads < n; i += 8 * kEvictThreads) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = mass[i + u * kEvictThreads];
#pragma unroll
            for (int u = 0; u < 8; ++u) count(mass_key(v[u]));
        }
        for (; i < n; i += kEvictThreads) count(mass_key(mass[i]));
        if (zeros && (kZeroMass & mask) == prefix) atomicAdd(&sm.hist[(kZeroMass >> shift) & ((1u << bits) - 1)], zeros);
        __syncthreads();
        // thread t looks at the two bins from 2047 - 2 t down
        const uint32_t c1 = sm.hist[kEvictBins - 1 - 2 * tid], c0 = sm.hist[kEvictBins - 2 - 2 * tid];
        uint32_t total;
        const uint32_t above = team_prefix<Team>(c1 + c0, total, sm, pass & 1);
        if (above < need && above + c1 + c0 >= need) {
            const bool upper = above + c1 >= need;
            sm.prefix = prefix | ((uint32_t)(kEvictBins - 1 - 2 * tid - (upper ? 0 : 1)) << shift);
            sm.need = need - above - (upper ? 0 : c1);
        }
        __syncthreads();
        prefix = sm.prefix; need = sm.need;
    }
    // survivors: a key above `prefix`, or the first `need` equal to it
    const int64_t stretch = ((n + kEvictWaves - 1) / kEvictWaves + kWave - 1) / kWave * kWave;
    const int64_t s0 = wave * stretch < n ? wave * stretch : n, s1 = s0 + stretch < n ? s0 + stretch : n;
    uint32_t above = 0, equal = 0;
    constexpr int U = 8;
    for (int64_t i = s0; i < s1; i += U * kWave) {
        float v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = mass[i + u * kWave + lane < s1 ? i + u * kWave + lane : s1 - 1];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = i + u * kWave + lane < s1;
            const uint32_t k = mass_key(v[u]);
            above += (uint32_t)__popcll(__ballot(in && k > prefix));
            equal += (uint32_t)__popcll(__ballot(in && k == prefix));
        }
    }
    if (lane == 0) { sm.above[wave] = above; sm.equal[wave] = equal; }
    __syncthreads();
    uint32_t at = 0, equal_before = 0;
    for (int w = 0; w < wave; ++w) {
        const uint32_t left = equal_before < need ? need - equal_before : 0u;
        at += sm.above[w] + (sm.equal[w] < left ? sm.equal[w] : left);
        equal_before += sm.equal[w];
    }
    for (int64_t i = s0; i < s1; i += U * kWave) {
        float v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = mass[i + u * kWave + lane < s1 ? i + u * kWave + lane : s1 - 1];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = i + u * kWave + lane < s1;
            const uint32_t k = mass_key(v[u]);
            const uint64_t eq = __ballot(in && k == prefix);
            const bool keep = in && (k > prefix || (k == prefix && equal_before + (uint32_t)mask_rank(eq) < need));
            const uint64_t m = __ballot(keep);
            if (keep) kept[at + (uint32_t)mask_rank(m)] = (int32_t)(i + u * kWave + lane);
            at += (uint32_t)__popcll(m);
            equal_before += (uint32_t)__popcll(eq);
        }
    }
}

// Row j of the cache becomes row kept[j] >= j, for all j of a stream, in place.  A workgroup holds a unit of neighbouring rows j in
// registers; it may overwrite them once every unit whose sources lie among them has read its own.  Those are units before it (kept[j] >= j),
// each of which raises a flag when its loads have come back and waits for nothing before that.  Units are handed out by a counter, so the
// units before a unit are always in the hands of a workgroup that runs or has run: every wait ends.  Flags carry no data (the rows
// themselves were written by earlier launches), so they need no more than the loads' return in front of them.
// One read and one write of the rows that move; through a buffer it would be two of each.
__global__ void __launch_bounds__(256) evict_move_kernel(EvictCall a) {
    __shared__ uint32_t ticket;
    if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add(&a.state[0], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const int64_t stream = ticket / (uint32_t)a.units;
    int unit = (int)(ticket - (uint32_t)stream * (uint32_t)a.units);
    uint32_t* flags = a.state + 1 + stream * a.units;
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
// same in every run.  A head's positions and weights are loaded ahead of the barrier in front of it.
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
    if (streams * a.units > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)streams), dim3(kEvictThreads), 0, st, a);
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(streams * a.units)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_add_mass(const MassCall& a, hipStream_t st) {
    hipLaunchKernelGGL(add_mass_kernel, dim3((unsigned)(a.B * a.Hkv)), dim3(kMassThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace tka
