// Host side of the operators over a cache: the device a call runs on, and how the keys of a decode are split.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

namespace tka {

// A handle's device, current while the call enqueues.
class DeviceOf {
  public:
    explicit DeviceOf(int device) {
        ok_ = hipGetDevice(&before_) == hipSuccess && (before_ == device || hipSetDevice(device) == hipSuccess);
        changed_ = ok_ && before_ != device;
    }
    ~DeviceOf() { if (changed_) (void)hipSetDevice(before_); }
    bool ok() const { return ok_; }
  private:
    int before_ = 0;
    bool ok_ = false, changed_ = false;
};

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
inline int64_t pages_per_split(const int64_t* pages, int n, double weight, int64_t longest, int64_t max_splits, int n_cu, double row_bytes) {
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

}  // namespace tka
