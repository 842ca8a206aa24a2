// Attention over packed sequences: arguments of the launchers, and what every kernel does with them: the rows that a
// row sees (its sequence, found in the starts) and the bucket of a relative position.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

namespace bp {

int cu_count();          // compute units of the device

constexpr int kMaxBuckets = 128;
constexpr int kPackedMaxHeadDim = 512;
constexpr int kPackedTile = 64;             // rows that share one partial of the bias table's gradient
constexpr int kShort = 256;                 // keys up to which delta of a bf16 row is not taken from its rounded ctx

// Buckets of a relative position: `first` of the offsets in front of the query (0), behind it (n; bidirectional only),
// plus the number of starts at or below the distance, minus one.
struct RelPos {
    int buckets = 0;                        // all of them; 0: no bias
    int n = 0;                              // of a direction
    int exact = 0;                          // buckets of one distance each
    int far = 0;                            // start[n - 1]: the last bucket has everything from there on
    float log2_exact = 0.f, per_octave = 0.f;      // bucket ~ exact + (log2(distance) - log2_exact) * per_octave, off by less than one
    const float* table = nullptr;           // [buckets, heads]
    int start[kMaxBuckets] = {};
};

struct PackedArgs {
    int T, n_seq, heads, kv_heads, d, causal;
    const int32_t* starts;
    float scale;
    int ld_q, ld_k, ld_v, ld_o;
    const void* q; const void* k; const void* v;
    void* ctx;
    float* lse;                             // [heads, T]
    // backward
    const void* dctx;
    void* dq; void* dk; void* dv;
    float* delta;                           // [heads, T]
    float* table_part;                      // [tiles of kPackedTile rows][heads][buckets], or null: no gradient of the table
    float* dtable;                          // [buckets, heads]: (+)= the sums of the partials
    int overwrite;
    int splits;                             // parts of the heads of a key / value head whose dK, dV are summed apart
    float* dkv_part;                        // splits > 1: [splits][T][kv_heads][dK, dV][d]
    RelPos rel;
};

// Parts into which the heads that share a key / value head are divided for dK and dV: as many as make `blocks` blocks of 64
// keys for a CU.  Few blocks, each with the work of a group of heads, leave most of the chip idle; the parts' sums go through
// memory, which long sequences pay and short ones do not.  Whole backward with 1 / 2 / 4 blocks a CU, us, from 256 of one
// part on: one sequence of 8192, 8 heads of 128 on 2 905 / 624 / 508; 2048 tokens, 32 on 8 252 / 187 / 168; 4 sequences
// of 512 92.7 / 89.3 / 96.8; from 512, 16 of 256 tokens 100 / 99 / 125; 200 of 1 to 40, 32 of 96 on 4 73 / 81 / 92.
// The host does not know the lengths, so the rule goes by their mean, empty sequences and rows of none included.  Where they
// differ: 3000, 517, 1777, 90 and 408 tokens, 8 heads of 128 on 2 215 / 161 / 162, 16 on 4 376 / 273 / 266; 2000, 30, 500,
// 10, 1, 700, 32 of 128 on 8 274 / 211 / 228: the second of each, as it should be.  One long sequence among many short or
// empty ones is taken for short: 4000 and 200 of 20, 32 of 96 on 4 716 / 501 / 446; 4096 and 60 empty, 8 of 128 on 2
// 257 / 185 / 186; 1500 and 20 of 20, 32 of 64 on 4 80 / 71 / 71: the first of each, up to 1.6 times the best.
inline int split_heads(const PackedArgs& a, int cus) {
    const int G = a.heads / a.kv_heads, mean = a.T / a.n_seq, blocks = mean >= 1024 ? 4 : mean >= 128 ? 2 : 1;
    const long one = (long)((a.T + kPackedTile - 1) / kPackedTile) * a.kv_heads;
    int s = 1;
    while (s < G && (G % s || one * s < (long)blocks * cus)) ++s;
    return s;
}

inline int packed_tiles(int T) { return (T + kPackedTile - 1) / kPackedTile; }

// one row per block, any head width, strides and alignment
hipError_t launch_packed_fwd_rows(int dtype, const PackedArgs& a, hipStream_t s);
hipError_t launch_packed_bwd_rows(int dtype, const PackedArgs& a, hipStream_t s);
// on the matrix cores: head widths that are multiples of 8 up to 128, 16-byte rows
hipError_t launch_packed_bf16(const PackedArgs& a, bool back, hipStream_t s);
hipError_t launch_packed_f32(const PackedArgs& a, bool back, hipStream_t s);

#ifdef __HIPCC__
// Rows lo .. hi - 1 of the sequence that row t lies in; false: in none.  Whatever the starts hold, the rows named are
// rows of the tensors.
__device__ __forceinline__ bool packed_row_range(const PackedArgs& a, int t, int& lo, int& hi) {
    int s = 0, e = a.n_seq;                 // starts[s] <= t < starts[e], if they do at the ends
    if (a.starts[0] > t || a.starts[a.n_seq] <= t) return false;
    while (e - s > 1) {
        const int m = (s + e) >> 1;
        if (a.starts[m] <= t) s = m; else e = m;
    }
    lo = max(a.starts[s], 0);
    hi = min(a.starts[e], a.T);
    return lo <= t && t < hi;
}

// A value of the bias table as the kernels take it.  Next to the type's lowest it is -inf: it has no room for the scores, and
// -inf is what leaves a query with nothing else NaN in both directions (p from lse would be 1 for each of its keys).
__device__ __forceinline__ float packed_bias(float value) { return value <= -1e30f ? -INFINITY : value; }

// bucket of an offset (key minus query); with a causal mask only offsets up to 0 occur
__device__ __forceinline__ int packed_bucket(const RelPos& r, const int* start, int causal, int offset) {
    const int dist = offset < 0 ? -offset : offset;
    int s = 0, e = r.n;
    while (e - s > 1) {
        const int m = (s + e) >> 1;
        if (start[m] <= dist) s = m; else e = m;
    }
    return s + (!causal && offset > 0 ? r.n : 0);
}

// dtable of a head (+)= its partials, by 256 threads in a fixed order: each takes every (256 / buckets)-th of a bucket, then
// these are added
__device__ __forceinline__ void sum_table_part(const PackedArgs& a, int head, float* sums) {
    const int buckets = a.rel.buckets, per = 256 / buckets, b = threadIdx.x % buckets, first = threadIdx.x / buckets;
    const int tiles = (a.T + kPackedTile - 1) / kPackedTile;
    float s = 0.f;
    if (first < per) {
#pragma unroll 8
        for (int i = first; i < tiles; i += per) s += a.table_part[((size_t)i * a.heads + head) * buckets + b];
    }
    sums[threadIdx.x] = s;
    __syncthreads();
    if (first) return;
    for (int i = 1; i < per; ++i) s += sums[i * buckets + b];
    float* out = a.dtable + (size_t)b * a.heads + head;
    *out = a.overwrite ? s : *out + s;
}
#endif

}  // namespace bp
