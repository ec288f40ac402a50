// The cache held in 8 bits: layout of its blocks, and the launchers over it (coded_store.hip, coded_decode.hip), called by api_coded.hip.
#pragma once
#include "device_utils.h"
#include "internal.h"
#include "ops.h"

namespace tka {

enum { CODED_INT8 = 0, CODED_E4M3 = 1 };

// A block of 64 tokens of a KV head is held whole or not at all, so its bytes lie as the matrix instructions of the decode take them: every load of
// a wave is 1024 neighbouring bytes, and no byte changes its lane.  A lane of mfma 16x16x32 is (j, n) = (lane / 16, lane % 16); its eight bytes of
// a contraction of 32 are a unit, two units of a lane are one 16-byte load.
//   keys    unit (t, c): key 16 t + n, channels 32 c + 8 j .. + 7;  units t D / 32 + c
//   values  unit (t, x): channel 16 t + n, keys 32 x + 4 j .. + 3 and 32 x + 16 + 4 j .. + 3 (the order in which the scores of the first product
//           lie in the lanes);  units 2 t + x
// int8 codes are stored plus 128.
constexpr int kCodedBlock = 64;
__host__ __device__ constexpr int coded_block_bytes(int D) { return kCodedBlock * D; }
__host__ __device__ constexpr int coded_unit_at(int unit, int lane) { return (unit >> 1) * 1024 + lane * 16 + (unit & 1) * 8; }
// channels c .. c + 3 or + 7 of a key (c a multiple of 4)
__host__ __device__ constexpr int coded_key_at(int D, int key, int c) {
    return coded_unit_at((key >> 4) * (D / 32) + (c >> 5), ((c >> 3) & 3) * 16 + (key & 15)) + (c & 7);
}
// keys k .. k + 3 of a channel (k a multiple of 4)
__host__ __device__ constexpr int coded_value_at(int k, int c) {
    return coded_unit_at(2 * (c >> 4) + (k >> 5), ((k >> 2) & 3) * 16 + (c & 15)) + ((k >> 4) & 1) * 4;
}

// Where the arrays of a layer's key streams lie (of the call's first sequence).
struct CodedArrays {
    char* codes[2];             // keys, values: [streams][blocks][64 D] bytes
    float* scales;              // [streams][blocks][2]
    char* open;                 // [streams][2][64][D] rows behind the last full block, as they came
    int32_t* len;               // [B]
    int64_t blocks;             // a stream has room for: max_tokens / 64
};

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Eight codes as fp16, times 2^-9 where they are int8: a byte in front of zeros is the fp16 number 2^-24 byte, and one fused step makes it
// (byte - 128) 2^-9, exactly.
template <int FMT> struct CodeUnit { static constexpr float value = FMT == CODED_INT8 ? 512.f : 1.f; };
template <int FMT>
__device__ __forceinline__ f16x8 code_values(uint32_t w0, uint32_t w1) {
    f16x2 v[4];
    if (FMT == CODED_INT8) {
        const f16x2 unit = {(_Float16)32768.f, (_Float16)32768.f}, zero = {(_Float16)-0.25f, (_Float16)-0.25f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = i < 2 ? w0 : w1;
            const uint32_t pair = __builtin_amdgcn_perm(w, w, i % 2 ? 0x0C030C02u : 0x0C010C00u);
            v[i] = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, pair), unit, zero);
        }
    } else {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.0f, false);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.0f, true);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.0f, false);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.0f, true);
    }
    return f16x8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}

constexpr float kShift = 13.f;          // weights are held times 2^13: fp16 has no numbers below 2^-24

// Queries as fp16, times a power of two that brings a head's largest number to [2^13, 2^14): one part of 16-bit queries is all of them (what lies below 2^-38
// of the largest is not), two of fp32 leave 2^-23 of a number, the half step of 32 bits.
template <int DT> struct QueryParts { static constexpr int value = DT == DT_F32 ? 2 : 1; };

constexpr int kCodedSeqs = 64;  // sequences of a launch of the append
struct CodedAppendCall {
    CodedArrays a;
    const char* src[2];         // element (s, t, h, c) at s * seq + t * token + h * head (bytes) + c
    int64_t seq, token, head;
    int64_t n;                  // rows of every sequence, >= 1
    int64_t wgs;                // workgroups of a key stream and kind: blocks that become full, at least 1
    int B, Hkv, D, dtype, format;
    int32_t base[kCodedSeqs];   // their lengths before the call
};
hipError_t launch_coded_append(const CodedAppendCall& a, hipStream_t st);

struct CodedReadCall {
    CodedArrays a;
    char* dst[2];
    int64_t seq, token, head;   // strides in bytes
    int64_t first, n;           // rows [first, first + n) of every sequence
    int B, Hkv, D, dtype, format;
};
hipError_t launch_coded_read(const CodedReadCall& a, hipStream_t st);

// Attention of one query per sequence and head over the first `sinks` and the newest `window` tokens, or of the last M tokens' (few of them), each over
// what it sees: then a row is a query and a head of the group, m G + g, as in prompt.h.
struct CodedDecodeCall : SplitParts {
    CodedArrays a;
    const void* q;              // [B][Hq][D], or [B][M][Hq][D]
    void* out_rows;             // [B][M][Hq][D] in the type of q (lse [B][M][Hq])
    uint32_t* arrive;           // [B][Hkv][row_blocks] splits that are done; zero between calls
    int64_t sinks, window;
    int64_t reach;              // tokens some query's window has: window + M - 1
    int M;                      // 0: one query per sequence
    int rows;                   // of a key stream: G, or M G
    int B, Hq, Hkv, G, dtype, format;
    int chunk;                  // blocks per split (n_split: of blocks, and one of open rows)
    int join_later;
    int row_blocks;             // blocks of 16 rows
};
// Rows of a key stream (kFewRows at most) up to which a prompt's tokens go through the kernel of single tokens, which takes the codes from memory to the products in
// registers, 16 rows at a time; the prompt kernel widens them into LDS once for 128 rows.  The two, in us, of 16 / 32 / 48 / 64 / 96 / 128 rows (8 KV heads, groups of 4):
//   d = 256, fp16, 4 sequences of 8000                41.1 / 49.5 / 64.4 / 72.8 / 88.0 / 112  and 59.8 / 60.6 / 63.2 / 64.0 / 66.5 / 69.3
//   d = 256, fp16, 16 sequences of 8000               113 / 124 / 165 / 187 / 260 / 325       and 192 / 193 / 199 / 200 / 205 / 215
//   d = 256, fp16, 4 sequences of up to 32000         82.2 / 97.6 / 135 / 141 / 182 / 217     and 188 / 190 / 195 / 196 / 201 / 206
//   d = 256, bf16, e4m3, 24000 tokens                 32.0 / 36.3 / 45.4 / 50.5 / 68.4 / 82.9 and 44.7 / 45.5 / 46.8 / 48.0 / 50.6 / 53.3
//   d = 256, fp32, 4 sequences of 8000                42.8 / 54.5 / 92.8 / 80.5 / 133 / 126   and 118 / 119 / 127 / 128 / 136 / 143
//   d = 128, bf16, 24000 tokens                       21.4 / 24.8 / 32.3 / 37.7 / 50.1 / 59.0 and 29.8 / 30.3 / 31.3 / 31.9 / 33.6 / 34.8
//   d = 128, fp32, 30000                              24.6 / 30.2 / 39.2 / 44.4 / 63.1 / 76.4 and 45.4 / 46.1 / 47.8 / 48.4 / 50.3 / 52.7
//   d = 64, fp32, 4 sequences of 16000                23.7 / 35.0 / 38.8 / 57.5 / 64.4 / 97.8 and 38.2 / 38.8 / 60.4 / 60.9 / 61.6 / 62.6
//   d = 64, fp16, 8 sequences of 16000                37.6 / 59.2 / 64.8 / 101 / 110 / 131    and 47.2 / 47.5 / 76.5 / 76.7 / 78.3 / 77.3
//   d = 32, bf16, 4 sequences of 16000                20.6 / 29.7 / 48.0 / 48.2 / 79.6 / 79.3 and 24.7 / 24.8 / 38.2 / 38.5 / 38.4 / 39.2
inline int few_rows(int dtype, int D) { return D == 256 ? (dtype == DT_F32 ? kFewRows : 64) : dtype == DT_F32 ? 64 : D == 128 ? 32 : 16; }
inline int64_t coded_decode_wgs(const CodedDecodeCall& a) {
    const int64_t units = (int64_t)a.B * a.Hkv * a.n_split;
    return a.row_blocks > 1 ? (units + 7) / 8 * 8 * a.row_blocks : units;
}
hipError_t launch_coded_decode(const CodedDecodeCall& a, hipStream_t st);

// Blocks of a sequence that a new token's query sees a token of: those of the sinks, then those of the window.
struct CodedWalk {
    int64_t N, first, sinks, full, sink_blocks, first_block;
    __host__ __device__ CodedWalk(int64_t n, int64_t sinks_, int64_t window) : N(n) {
        first = window < n ? n - window : 0;
        sinks = sinks_;
        if (sinks >= first) { first = 0; sinks = 0; }
        full = n / kCodedBlock;
        first_block = first / kCodedBlock < full ? first / kCodedBlock : full;
        sink_blocks = (sinks + kCodedBlock - 1) / kCodedBlock;
        if (sink_blocks > first_block) sink_blocks = first_block;      // (of a block that both see a part of: the window's)
    }
    __host__ __device__ int64_t blocks() const { return sink_blocks + full - first_block; }
    __host__ __device__ int64_t block(int64_t i) const { return i < sink_blocks ? i : first_block + (i - sink_blocks); }
    __host__ __device__ bool whole(int64_t block) const { return block * kCodedBlock >= first || (block + 1) * kCodedBlock <= sinks; }
    __host__ __device__ bool sees(int64_t t) const { return t >= first || t < sinks; }
    // whether an open row is seen (some row always is: the newest token's, unless it closed its block)
    __host__ __device__ bool open() const { return N > full * kCodedBlock; }
};

}  // namespace tka
