// Attention of one query per sequence and head over the 8-bit cache (topk_attn_coded_decode): out = sum_t p_t V_t / sum_t p_t with
// p_t = exp(q . K_t / sqrt(d)), K_t = k_b c_t and V_t = v_b c'_t for codes c, c' and the scales k_b, v_b of their block, over the first `sinks` and the newest
// `window` tokens, in one pass over the codes.
//
// Codes are exact in fp16, so both products are fp16 MFMA whatever the type of the queries: k_b multiplies a block's scores, v_b goes into the weights.
// A split is a run of blocks, a wave has a block at a time; one more split has the open rows, in their own type.  The last split of a key stream
// to finish joins them.
//
// A prompt's last tokens, where they are few, are rows here as the heads of a group are (ROWS), each with its own mask.
//
// Bound by the read of the codes: 16 KB per 64 keys and KV head (d = 128).  A million tokens, 8 KV heads, int8, fp16 queries: 373 us (5.8 TB/s; plain
// reads reach 6.0 to 6.1); 16 sequences of up to 32768, e4m3: 127 (4.5 TB/s: their splits end unevenly); 500 tokens 11.2, all latency; eight tokens of 4 sequences
// of 1000 to 20000 (32 rows) 46.  Two tiles a wave in registers, two workgroups to a compute unit: the next block is on its way during this one's products.
#include "coded.h"
#include "scan_tiles.h"
#include "split_join.h"

namespace tka {

namespace {

__device__ __forceinline__ float top_of_rows(float v) {        // largest of lanes l, l ^ 16, l ^ 32, l ^ 48
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// A whole number that is not below x, and that the product which x is the rounding of is not above: from 2^23 on it is off by ones.
__device__ __forceinline__ float whole_above(float x) { return ceilf(x) + floorf(fminf(fabsf(x), 0x1p120f) * 0x1p-23f); }      // (-inf stays)
// 2^x for a whole number x (0 for -inf)
__device__ __forceinline__ float power2(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace

// ROWS: of the last M tokens.
template <int DT, int D, int FMT, bool ROWS>
__global__ void __launch_bounds__(256, (DT == DT_F32 && D == 256 ? 1 : 2)) coded_decode_kernel(CodedDecodeCall a) {
    constexpr int T = D / 16, C = D / 32, UK = D / 16, ROW = D * Elem<DT>::kBytes, EPL = Elem<DT>::kPerLoad, PARTS = QueryParts<DT>::value;
    constexpr int NW = 4, NT = NW * kWave, RED = NW * 16 * (D + 4), JOIN = 16 * kMaxSplits + 8 * NT;
    constexpr bool kTwoTiles = D <= 128;
    __shared__ __align__(16) float lds[RED > JOIN ? RED : JOIN];
    float (*const red)[16][D + 4] = reinterpret_cast<float (*)[16][D + 4]>(lds);
    __shared__ float red_m[NW][16], red_l[NW][16], red_e[NW][16];
    __shared__ uint32_t arrived;
    const int lane = lane_id(), j = lane >> 4, n = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    // (units as in the dense decode: head blocks of a split eight workgroups apart, splits of one rank after each other, a stream later each)
    int unit = (int)blockIdx.x, rb = 0;
    if (a.row_blocks > 1) {
        const int group = unit / (8 * a.row_blocks), in = unit - group * 8 * a.row_blocks;
        rb = in >> 3;
        unit = group * 8 + (in & 7);
    }
    const int streams = a.B * a.Hkv, split = unit / streams;
    if (split >= a.n_split) return;
    int stream = unit - split * streams - split % streams;
    if (stream < 0) stream += streams;
    const int b = stream / a.Hkv, kvh = stream - b * a.Hkv;
    const CodedWalk seen(a.a.len[b], a.sinks, ROWS ? a.reach : a.window);
    const int open = seen.open() ? 1 : 0;
    const int64_t blocks = seen.blocks();
    int ns = (int)((blocks + a.chunk - 1) / a.chunk);
    ns = (ns < a.n_split - open ? ns : a.n_split - open) + open;
    if (split >= ns) return;
    const int heads = a.rows - 16 * rb < 16 ? a.rows - 16 * rb : 16;
    const int64_t head0 = (int64_t)stream * a.rows + 16 * rb;
    const JoinedRows<DT, CodedDecodeCall> to_rows{a, stream, 16 * rb};
    const char* const query = static_cast<const char*>(a.q) + (ROWS ? to_rows.at(n < heads ? n : 0) : head0 + (n < heads ? n : 0)) * ROW;
    // what the lane's row sees, and what all rows do
    const int64_t pos = ROWS ? seen.N - a.M + (16 * rb + (n < heads ? n : 0)) / a.G : 0;
    const auto sees = [&](int64_t t) { return ROWS ? t <= pos && (t < a.sinks || t > pos - a.window) : seen.sees(t); };
    const auto all_see = [&](int64_t block) {
        const int64_t t0 = block * kCodedBlock, t1 = t0 + kCodedBlock;
        return ROWS ? t1 <= seen.N - a.M + 1 && (t0 > seen.N - 1 - a.window || t1 <= a.sinks) : seen.whole(block);
    };
    // log2(e) / sqrt(D) as two numbers: the rounding of one would be a part of every score
    constexpr double kScale = 1.4426950408889634 / (D == 32 ? 5.656854249492381 : D == 64 ? 8.0 : D == 128 ? 11.313708498984761 : 16.0);
    constexpr float kScaleHi = (float)kScale, kScaleLo = (float)(kScale - (double)kScaleHi);

    float m = -INFINITY, l = 0.f, e_w = -INFINITY;     // running maximum (rounded up to a whole number), sum of weights, power of two of the weighted sum
    if (split < open) {
        // ---- open rows: 16 keys a wave ----
        const int rows = (int)(seen.N - seen.full * kCodedBlock);
        const char* const base = a.a.open + (int64_t)stream * 2 * kCodedBlock * ROW;
        const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, rows * ROW, 0x00020000);
        const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base) + kCodedBlock * ROW, 0, rows * ROW, 0x00020000);
        constexpr int KCH = ROW / 64;
        f32x4 s = {0.f, 0.f, 0.f, 0.f}, part[4] = {};
#pragma unroll
        for (int x = 0; x < KCH; ++x) {
            u32x4 qv = *reinterpret_cast<const u32x4*>(query + 64 * x + 16 * j);
            if (n >= heads) qv = u32x4{0, 0, 0, 0};
            const u32x4 kv = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, (16 * wave + n) * ROW + 64 * x + 16 * j, 0, 0));
            if constexpr (DT == DT_F32) {
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    part[y] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kv[y]), __uint_as_float(qv[y]), part[y], 0, 0, 0);
            } else {
                using v8 = typename Mfma<DT>::v8;
                s = Mfma<DT>::mac(__builtin_bit_cast(v8, kv), __builtin_bit_cast(v8, qv), s);
            }
        }
        if (DT == DT_F32) s = (part[0] + part[1]) + (part[2] + part[3]);
        const int64_t t0 = seen.full * kCodedBlock + 16 * wave + 4 * j;
        float top = -INFINITY, p[4];
        bool there[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            there[i] = 16 * wave + 4 * j + i < rows && sees(t0 + i);
            if (there[i]) top = fmaxf(top, s[i] * kScaleHi);
        }
        m = whole_above(top_of_rows(top));
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = there[i] && s[i] != -INFINITY ? __builtin_amdgcn_exp2f(fmaf(s[i], kScaleHi, fmaf(s[i], kScaleLo, -ref))) : 0.f;
            l += p[i];
        }
        e_w = m;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            // (a row that is not seen is taken as zeros: no weight of zero meets an infinity.  Where rows see different tokens, what is no number is, and
            // goes to those that see it, one token at a time.)
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            const auto value = [&](int key, int c) {
                const int off = (16 * wave + key) * ROW + c * Elem<DT>::kBytes;
                if constexpr (DT == DT_F32) {
                    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rv, off, 0, 0));
                } else {
                    const uint16_t bits = __builtin_amdgcn_raw_buffer_load_b16(rv, off, 0, 0);
                    return DT == DT_F16 ? (float)__builtin_bit_cast(_Float16, bits) : __uint_as_float((uint32_t)bits << 16);
                }
            };
            bool odd = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = value(4 * j + i, 16 * t + n);
                const bool number = fabsf(v) < INFINITY;
                odd |= !number;
                if (ROWS ? !number : !there[i]) v = 0.f;
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[i], acc, 0, 0, 0);
            }
            if (ROWS && __any(odd)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    for (int y = 0; y < 4; ++y) {
                        const float w = __shfl(p[i], 16 * y + n, 64);
                        const bool sees_it = __shfl((int)there[i], 16 * y + n, 64);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float v = value(4 * y + i, 16 * t + 4 * j + r);
                            if (sees_it && !(fabsf(v) < INFINITY)) acc[r] = fmaf(w, v, acc[r]);
                        }
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) red[wave][n][16 * t + 4 * j + r] = acc[r];
        }
    } else {
        // ---- blocks ----
        f16x8 q[PARTS][C];
        float unit_q;                                  // what a score is times for its power of two
        {
            float x[C][8], amax = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
#pragma unroll
                for (int y = 0; y < 8; y += EPL)
                    Elem<DT>::widen(*reinterpret_cast<const u32x4*>(query + (32 * c + 8 * j + y) * Elem<DT>::kBytes), &x[c][y]);
#pragma unroll
                for (int y = 0; y < 8; ++y) amax = fmaxf(amax, fabsf(x[c][y]));
            }
            amax = top_of_rows(amax);
            // amax times 2^up lies in [2^13, 2^14)
            int up = 13 - ((int)(__float_as_uint(amax) >> 23) - 127);
            up = amax == 0.f || up > 120 ? 120 : up < -114 ? -114 : up;
            const float by = __uint_as_float((uint32_t)(up + 127) << 23);
            unit_q = __uint_as_float((uint32_t)(127 - up) << 23) * CodeUnit<FMT>::value;
#pragma unroll
            for (int c = 0; c < C; ++c) {
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    float rest = n < heads ? x[c][y] * by : 0.f;
#pragma unroll
                    for (int z = 0; z < PARTS; ++z) {
                        q[z][c][y] = (_Float16)rest;
                        rest -= (float)q[z][c][y];
                    }
                }
            }
        }
        const int64_t p0 = (int64_t)(split - open) * a.chunk, p1 = split + 1 < ns ? p0 + a.chunk : blocks;
        const int mine = (int)(p1 - p0) > wave ? ((int)(p1 - p0) - wave + NW - 1) / NW : 0;
        struct Tile { u32x4 k[UK], v[UK]; float2 scale; };
        const char* const Kb = a.a.codes[0] + (int64_t)stream * a.a.blocks * coded_block_bytes(D) + lane * 16;
        const char* const Vb = a.a.codes[1] + (int64_t)stream * a.a.blocks * coded_block_bytes(D) + lane * 16;
        const float* const Sb = a.a.scales + (int64_t)stream * a.a.blocks * 2;
        auto block_of = [&](int i) { return seen.block(p0 + wave + NW * (int64_t)(i < mine ? i : mine - 1)); };
        auto load = [&](Tile& t, int i) {
            const int64_t block = block_of(i);
            const char* const k = Kb + block * coded_block_bytes(D);
            const char* const v = Vb + block * coded_block_bytes(D);
#pragma unroll
            for (int u = 0; u < UK; ++u) t.k[u] = *reinterpret_cast<const u32x4*>(k + u * 1024);
#pragma unroll
            for (int u = 0; u < UK; ++u) t.v[u] = *reinterpret_cast<const u32x4*>(v + u * 1024);
            t.scale = *reinterpret_cast<const float2*>(Sb + block * 2);
        };
        f32x4 acc[T];
#pragma unroll
        for (int t = 0; t < T; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        float carry = 0.f;                             // what the additions to l rounded off
        auto use = [&](const Tile& t, int i) {
            const int64_t block = block_of(i);
            f32x4 s[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                s[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int u = g * C + c;
                    const f16x8 k = code_values<FMT>(t.k[u / 2][u % 2 * 2], t.k[u / 2][u % 2 * 2 + 1]);
#pragma unroll
                    for (int z = 0; z < PARTS; ++z) s[g] = Mfma<DT_F16>::mac(k, q[z][c], s[g]);
                }
            }
            // score times log2(e) / sqrt(D), in two parts: f + f_lo is the factor to 2^-48
            const float by = t.scale.x * unit_q, f = by * kScaleHi, f_lo = fmaf(by, kScaleHi, -f) + by * kScaleLo;
            const bool whole = all_see(block);
            float top = -INFINITY, p[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                float v = s[x / 4][x % 4] * f;
                if (!whole && !sees(block * kCodedBlock + 16 * (x / 4) + 4 * j + x % 4)) v = -INFINITY;
                p[x] = v;
                top = fmaxf(top, v);
            }
            const float bm = whole_above(top_of_rows(top));
            const float m_new = fmaxf(m, bm), ref = m_new == -INFINITY ? 0.f : m_new;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const float raw = s[x / 4][x % 4], w = __builtin_amdgcn_exp2f(fmaf(raw, f, fmaf(raw, f_lo, -ref)));
                p[x] = !whole && p[x] == -INFINITY ? 0.f : w;
            }
            float sum = 0.f;
#pragma unroll
            for (int x = 0; x < 16; x += 4) sum += (p[x] + p[x + 1]) + (p[x + 2] + p[x + 3]);
            const float down = power2(m - ref);
            l *= down;
            carry *= down;
            const float add = sum - carry, grown = l + add;          // (32 bits that grow without end round every small weight the same way)
            carry = (grown - l) - add;
            l = grown;
            m = m_new;
            // The weighted sum has a power of two of its own, e_w: the largest weight so far times its block's value scale, rounded up.  (Relative to m, blocks
            // whose values are small would lose their weights' low parts to those of a block whose values are large.)
            const float sv = t.scale.y;
            const int ke = (int)(__float_as_uint(sv) >> 23) - 126;   // sv < 2^ke
            const float e_new = sv > 0.f ? fmaxf(e_w, bm + (float)ke) : e_w;
            float g = sv;
            if (sv > 0.f) {
                const float up = fminf(ref - e_new + kShift, (float)(127 - ke));
                g = ldexpf(sv, (int)fmaxf(up, -300.f));
            }
            if (ROWS && bm == -INFINITY) g = 0.f;                    // (a block of NaN that the row does not see)
            if (__any(e_new != e_w)) {
                const float f_w = e_w == -INFINITY ? 1.f : power2(e_w - e_new);
#pragma unroll
                for (int c = 0; c < T; ++c) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[c][r] *= f_w;
                }
            }
            e_w = e_new;
            f16x8 hi[2], lo[2];
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                // (the product is a number of its own: rounded to 16 bits together with the multiplication in one place and after it in the other, the two
                // parts did not make up the weight now and then, 2^-11 of one key's)
                float w = p[x] * g;
                asm("" : "+v"(w));
                hi[x / 8][x % 8] = (_Float16)w;
                lo[x / 8][x % 8] = (_Float16)(w - (float)hi[x / 8][x % 8]);      // (two parts: 2^-22 of a weight)
            }
#pragma unroll
            for (int c = 0; c < T; ++c) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int u = 2 * c + x;
                    const f16x8 v = code_values<FMT>(t.v[u / 2][u % 2 * 2], t.v[u / 2][u % 2 * 2 + 1]);
                    acc[c] = Mfma<DT_F16>::mac(v, hi[x], acc[c]);
                    acc[c] = Mfma<DT_F16>::mac(v, lo[x], acc[c]);
                }
            }
        };
        if (mine > 0) {
            if constexpr (kTwoTiles) {
                Tile ta, tb;
                load(ta, 0);
                for (int i = 0; i < mine; i += 2) {
                    load(tb, i + 1);
                    __builtin_amdgcn_sched_barrier(0);
                    use(ta, i);
                    if (i + 1 >= mine) break;
                    load(ta, i + 2);
                    __builtin_amdgcn_sched_barrier(0);
                    use(tb, i + 1);
                }
            } else {
                Tile t;
                for (int i = 0; i < mine; ++i) {
                    load(t, i);
                    __builtin_amdgcn_sched_barrier(0);
                    use(t, i);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < T; ++c) {
#pragma unroll
            for (int r = 0; r < 4; ++r) red[wave][n][16 * c + 4 * j + r] = acc[c][r] * CodeUnit<FMT>::value;
        }
    }
    l = add_lanes_32(add_lanes_16(l));
    // A maximum passes over NaN: a wave of nothing but NaN would count as one without a key.  (With a maximum of +inf its factor is NaN.)
    if (l != l) m = INFINITY;
    if (j == 0) { red_m[wave][n] = m; red_l[wave][n] = l; red_e[wave][n] = e_w; }
    __syncthreads();
    const bool alone = ns == 1;
    const float shift = split < open ? 0.f : kShift;                 // (of blocks' weighted sums; beyond 2^24 a power less 13 is no number)
    for (int i = (int)threadIdx.x; i < heads * D; i += NT) {
        const int h = i / D, c = i - h * D;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, red_m[w][h]);
        float sum = 0.f, total = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = red_m[w][h] == -INFINITY ? 0.f : power2(red_m[w][h] - top);
            const float f_w = red_e[w][h] == -INFINITY ? 0.f : power2(red_e[w][h] - top - shift);
            sum = fmaf(f_w, red[w][h][c], sum);
            if (f != 0.f) total = fmaf(f, red_l[w][h], total);
        }
        const int64_t bh = head0 + h;
        if (alone && !a.join_later) {
            const float o = sum * (1.0f / total), lse = (top + log2f(total)) * 0.69314718055994531f;
            if (ROWS) {
                to_rows.one(h, c, o);
                if (c == 0) to_rows.lse(h, lse);
            } else {
                a.out[bh * D + c] = o;
                if (c == 0 && a.lse) a.lse[bh] = lse;
            }
        } else {
            put(&a.part_acc[(bh * a.n_split + split) * D + c], sum);
            if (c == 0) {
                put(&a.part_lm[(bh * a.n_split + split) * 2], total);
                put(&a.part_lm[(bh * a.n_split + split) * 2 + 1], top);
            }
        }
    }
    if (a.join_later || alone) return;
    // the last split of the stream's head block to get here joins them (and leaves the counter at zero for the next call)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    uint32_t* const counter = a.arrive + (int64_t)stream * a.row_blocks + rb;
    if (threadIdx.x == 0) arrived = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (arrived + 1u != (uint32_t)ns) return;
    if (threadIdx.x == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    f32x4* const room = reinterpret_cast<f32x4*>(lds + 16 * kMaxSplits);
    if constexpr (ROWS) join_splits<NT>(a, head0, to_rows, heads, ns, 0.f, lds, room);
    else join_splits<NT>(a, head0, heads, ns, 0.f, lds, room);
}

// A workgroup per head: many splits of many heads.  ROWS: of the last tokens' rows, of type DT.
template <int DT, bool ROWS>
__global__ void __launch_bounds__(256) coded_join_kernel(CodedDecodeCall a) {
    __shared__ float f[kMaxSplits];
    __shared__ f32x4 sums[512];
    const int64_t head = blockIdx.x;
    const int stream = (int)(head / a.rows);
    const CodedWalk seen(a.a.len[stream / a.Hkv], a.sinks, ROWS ? a.reach : a.window);
    const int open = seen.open() ? 1 : 0;
    int ns = (int)((seen.blocks() + a.chunk - 1) / a.chunk);
    ns = (ns < a.n_split - open ? ns : a.n_split - open) + open;
    if constexpr (ROWS) join_splits<256>(a, head, JoinedRows<DT, CodedDecodeCall>{a, stream, (int)(head - (int64_t)stream * a.rows)}, 1, ns, 0.f, f, sums);
    else join_splits<256>(a, head, 1, ns, 0.f, f, sums);
}

hipError_t launch_coded_decode(const CodedDecodeCall& a, hipStream_t st) {
    const dim3 grid((unsigned)coded_decode_wgs(a)), wg(256);
#define TKA_DECODE_(DT_, D_, FMT_)                                                                                        \
    do {                                                                                                                  \
        if (a.M) hipLaunchKernelGGL((coded_decode_kernel<DT_, D_, FMT_, true>), grid, wg, 0, st, a);                      \
        else hipLaunchKernelGGL((coded_decode_kernel<DT_, D_, FMT_, false>), grid, wg, 0, st, a);                         \
    } while (0)
#define TKA_DECODE(DT_, D_)                                                                                               \
    do {                                                                                                                  \
        if (a.format == CODED_INT8) TKA_DECODE_(DT_, D_, CODED_INT8);                                                     \
        else TKA_DECODE_(DT_, D_, CODED_E4M3);                                                                            \
    } while (0)
    TKA_BY_TYPE_AND_DIM(TKA_DECODE, a.dtype, a.D);
#undef TKA_DECODE
#undef TKA_DECODE_
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.join_later) return e;
    const dim3 heads((unsigned)((int64_t)a.B * a.Hkv * a.rows));
    if (!a.M) hipLaunchKernelGGL((coded_join_kernel<DT_F32, false>), heads, wg, 0, st, a);
    else if (a.dtype == DT_F32) hipLaunchKernelGGL((coded_join_kernel<DT_F32, true>), heads, wg, 0, st, a);
    else if (a.dtype == DT_F16) hipLaunchKernelGGL((coded_join_kernel<DT_F16, true>), heads, wg, 0, st, a);
    else hipLaunchKernelGGL((coded_join_kernel<DT_BF16, true>), heads, wg, 0, st, a);
    return hipGetLastError();
}

}  // namespace tka
