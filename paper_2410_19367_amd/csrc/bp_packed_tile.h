// Attention over packed sequences on the gfx950 matrix cores: forward, dQ, dK / dV, for the element types that supply a
// policy P (bf16, fp32): tiles of 64 rows in LDS and the products on them.
//
// The rows of all sequences are cut into blocks where they lie, wherever the sequences begin: a block may hold the end of
// one sequence, several whole ones and the start of another, so thousands of short sequences cost no more blocks than one
// long one.  What a row sees is a range of rows (its sequence, up to itself under a causal mask), and so is what a key is
// seen by; a block walks the tiles from the first row of its first range to the last of its last, and masks by range only
// the pieces of 32 x 32 that are not inside every row's range.  Ranges come from the starts: one load of 64 of them and a
// scalar walk in every wave, no launch before the kernel and nothing on the host.
//
// Scores stand transposed where that keeps the softmax row of a query in one lane (forward, dQ: lane <-> query, registers
// <-> keys; dK/dV: lane <-> key, registers <-> queries), and leave the accumulators as the B operand of the next product.
//
// Values that are not finite.  A masked pair has p = 0, but zero times NaN is not zero in the second product.  Only NaN
// comes of that, so a block that ends with NaN in a result takes its tiles once more, with the second products done row by
// row on the vector units and the masked pairs left out (every value NaN: forward 9 - 32 times as long, backward 17 - 35).
// A block without NaN pays one look at its results; the second walk is code of its own, without a branch to the matrix
// cores in it, which kept all accumulators twice (registers of the forward at width 64: 112 alone, 118 with this walk, 162
// with the branch).
//
// Key / value heads that several query heads share: blocks of query heads of the same one run on the same XCD (position
// modulo kv_heads first), and a dK/dV block walks its heads one after the other, so shared gradients are sums in
// registers, in a fixed order.
#pragma once
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "bp_device.h"
#include "bp_packed.h"
#include "bp_tile.h"

namespace bp {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// The lane, anew for each walk over the tiles: what one walk makes of it does not wait in registers for the next.
__device__ __forceinline__ int lane_of(unsigned thread) {
    int lane = thread & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

// Kernel arguments are cold at every launch: named at the top they are loaded together, with one wait.
__device__ __forceinline__ void packed_args_now(const PackedArgs& a) {
    asm volatile("" ::"s"(a.T), "s"(a.n_seq), "s"(a.heads), "s"(a.kv_heads), "s"(a.d), "s"(a.causal), "s"(a.starts), "s"(a.scale),
                 "s"(a.ld_q), "s"(a.ld_k), "s"(a.ld_v), "s"(a.ld_o), "s"(a.q), "s"(a.k), "s"(a.v));
}

// ---- what a row sees

// Ranges of the sequences that rows first + lane + 64 r lie in (lo < 0: none), the same rows in every wave of a block.
// Nothing the starts hold leads outside [0, T).
template <int R>
__device__ __forceinline__ void seq_ranges(const int32_t* starts, int n_seq, int T, int first, int lane, int (&lo)[R], int (&hi)[R]) {
    const int last = first + 64 * R - 1;
    int base = 0, count = n_seq + 1;
    while (count > 64) {                    // 64 samples narrow the place of `first` to a 64th
        const int stride = (count + 63) >> 6, i = lane * stride;
        const int v = i < count ? starts[base + i] : 0x7fffffff;
        const int below = max((int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(v <= first)), 1) - 1;
        base += below * stride;
        count = min(stride, count - below * stride);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) { lo[r] = -1; hi[r] = 0x7fffffff; }
    for (int w = base; w <= n_seq; w += 64) {
        const int v = w + lane <= n_seq ? starts[w + lane] : 0x7fffffff;
        const int n = min(64, n_seq + 1 - w);
        int st = 0;
        for (int e = 0; e < n; ++e) {
            st = __builtin_amdgcn_readlane(v, e);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int row = first + lane + 64 * r;
                if (st <= row) { lo[r] = max(st, 0); hi[r] = 0x7fffffff; }
                else hi[r] = min(hi[r], st);
            }
            if (st > last) break;
        }
        if (st > last) break;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = first + lane + 64 * r;
        if (hi[r] == 0x7fffffff || row >= T) lo[r] = -1;
        hi[r] = min(hi[r], T);
    }
}

// The ranges of a lane's row, of the 32 rows of its wave and of all rows of its block.  Ranges of rows that follow one
// another begin and end in that order, so the outermost and innermost ends are those of the first and last row that has one.
// (A wave takes pieces that none of its rows sees like others, masked: left out by a branch, they made the compiler keep
// two sets of accumulators.  dK/dV at width 128 spilled 580 bytes a lane, then 136, in 256 registers.)
struct Ranges {
    int lo, hi;                             // of this lane's row; lo == hi: none
    int inner_lo, inner_hi;                 // what all rows of the wave see; inner_hi 0: it has none
    int blk_lo, blk_hi;                     // outermost ends of the block's; blk_hi 0: none
    int short_lo, short_hi;                 // and of its ranges of up to kShort rows; short_hi 0: none (64 rows only)
    uint64_t alone;                         // a bit for each row of the block: a sequence of one row (64 rows only)
};
// rows: 64 or 128 of a block; mine: this lane's row within it.  by_key: what a key is seen by, else what a query sees
template <int QB>
__device__ __forceinline__ Ranges block_ranges(const PackedArgs& a, int first, int mine, int lane, bool by_key) {
    constexpr int R = QB / 64;
    int lo[R], hi[R];
    seq_ranges<R>(a.starts, a.n_seq, a.T, first, lane, lo, hi);
    Ranges x;
    x.blk_lo = x.blk_hi = x.short_lo = x.short_hi = 0;
    x.alone = R == 1 ? __builtin_amdgcn_ballot_w64(lo[0] >= 0 && hi[0] - lo[0] == 1) : 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = first + lane + 64 * r;
        const bool ok = lo[r] >= 0;
        if (ok && a.causal) { if (by_key) lo[r] = row; else hi[r] = row + 1; }
        if (!ok) lo[r] = hi[r] = 0;
        const uint64_t valid = __builtin_amdgcn_ballot_w64(ok);
        if (valid) {
            if (!x.blk_hi) x.blk_lo = __builtin_amdgcn_readlane(lo[r], __builtin_ctzll(valid));
            x.blk_hi = __builtin_amdgcn_readlane(hi[r], 63 - __builtin_clzll(valid));
        }
        const uint64_t few = R == 1 ? __builtin_amdgcn_ballot_w64(ok && hi[r] - lo[r] <= kShort) : 0;
        if (few) {
            x.short_lo = __builtin_amdgcn_readlane(lo[r], __builtin_ctzll(few));
            x.short_hi = __builtin_amdgcn_readlane(hi[r], 63 - __builtin_clzll(few));
        }
    }
    x.lo = __shfl(lo[0], mine & 63, 64);
    x.hi = __shfl(hi[0], mine & 63, 64);
    if (R == 2 && mine >= 64) {             // (the same answer in every lane of a wave)
        x.lo = __shfl(lo[R - 1], mine & 63, 64);
        x.hi = __shfl(hi[R - 1], mine & 63, 64);
    }
    const uint64_t valid = __builtin_amdgcn_ballot_w64(x.hi > x.lo);
    x.inner_lo = x.inner_hi = 0;
    if (valid) {
        x.inner_lo = __builtin_amdgcn_readlane(x.lo, 63 - __builtin_clzll(valid));
        x.inner_hi = __builtin_amdgcn_readlane(x.hi, __builtin_ctzll(valid));
        // (lanes l and l + 32 hold the same row; the last of the first half is the last row)
    }
    return x;
}

// Block `bid` of a launch: blocks of rows from the last on (under a causal mask a sequence's last rows have most to do), all
// heads of one before the next, heads of the same key / value head a multiple of kv_heads apart.  HP heads share a block.
template <int HP>
__device__ __forceinline__ void packed_coords(const PackedArgs& a, int bid, int nblk, int& blk, int& head, int& kvh) {
    const int per = a.heads / HP, i = bid / per, p = bid - i * per, g = p / a.kv_heads;
    kvh = p - g * a.kv_heads;
    head = kvh * (a.heads / a.kv_heads) + g * HP;
    blk = nblk - 1 - i;
}

// ---- pieces of tiles

// Direct copy of rows [first, end) of a tile of 64 rows into LDS; its other rows, and columns at and beyond the head width,
// become zeros: they lie outside the buffer descriptor's range (up to 2^31 bytes), against which the lane's offset is checked.
template <class P, int NW>
struct TileLoader {
    static constexpr int E = sizeof(typename P::elem), CPR = P::D * E / 16;        // 16-byte chunks per row
    static constexpr int NI = CPR / NW, ROWSTEP = NW * 64 / CPR;        // rows between a lane's consecutive chunks
    static constexpr int NO = ROWSTEP >= 16 ? 1 : 16 / ROWSTEP;         // chunks after which the swizzle repeats
    static constexpr uint32_t kBeyond = 0x80000000u;                    // and so is this plus any row's offset
    uint32_t off[NO];
    __device__ __forceinline__ void init(int wave, int lane, int ld, int d) {
        const int p = wave * 64 + lane;
#pragma unroll
        for (int i = 0; i < NO; ++i) {
            const int row = p / CPR + i * ROWSTEP, c = (p % CPR) ^ P::swizzle(row);
            off[i] = c * (16 / E) < d ? (uint32_t)(row * ld + c * (16 / E)) * E : kBeyond;
        }
    }
    __device__ __forceinline__ void issue(const typename P::elem* base, int ld, int d, int first, int end, char* lds, int wave) const {
        const rsrc_t src = make_rsrc(base, end > 0 ? (uint32_t)((min(end, 64) - 1) * ld + d) * E : 0u);
        const uint32_t step = (uint32_t)(ROWSTEP * NO * ld) * E;
        if (first > 0) {
            const int row = (wave * 64 + (int)__lane_id()) / CPR;
#pragma unroll
            for (int i = 0; i < NI; ++i)
                dma16(src, row + i * ROWSTEP < first ? kBeyond : off[i % NO] + (i / NO) * step, 0, lds + (wave + NW * i) * 1024);
            return;
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) dma16(src, off[i % NO] + (i / NO) * step, 0, lds + (wave + NW * i) * 1024);
    }
};

__device__ __forceinline__ int piece_row(int v, int h) { return 8 * (v >> 2) + 4 * h + (v & 3); }

// out^T += tile[row0 .. row0 + 31]^T x without the pairs outside [lo, hi), the lane's range counted from row0
template <class P>
__device__ __forceinline__ void contract_by_rows(const char* tile, int row0, int lane, int lo, int hi, const f32x16& x,
                                                 f32x16 (&out)[P::DT]) {
#pragma unroll 1
    for (int r = 0; r < 32; ++r) {
        int h = lane >> 5;
        asm volatile("" : "+v"(h));         // nothing that is made of it waits in registers outside the loop
        const int reg = (r & 3) + 4 * (r >> 3);
        float mine = x[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) mine = v == reg ? x[v] : mine;
        const float other = __shfl_xor(mine, 32, 64);
        const float w = ((r >> 2) & 1) == h ? mine : other;
        const bool ok = r >= lo && r < hi;
#pragma unroll
        for (int t = 0; t < P::DT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 e = P::four(tile, row0 + r, 32 * t + 8 * g + 4 * h);
#pragma unroll
                for (int i = 0; i < 4; ++i) out[t][4 * g + i] += ok ? w * e[i] : 0.f;
                __builtin_amdgcn_sched_barrier(0);
            }
    }
}

template <int DT>
__device__ __forceinline__ bool any_nan(const f32x16 (&x)[DT]) {
    bool bad = false;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) bad |= x[t][v] != x[t][v];
    return bad;
}
template <int DT>
__device__ __forceinline__ void clear(f32x16 (&x)[DT]) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) x[t][v] = 0.f;
}

// What a lane has of a piece, in pairs: sums over the pieces of a long row that take these have a sixteenth of the terms, each
// rounded to the size of the sum.  (16 values one after the other, 5091 tokens without a causal mask: gradient of the bias
// table off by 8.6e-7, now 7.7e-7, at the same speed.)
__device__ __forceinline__ float sum_of(const f32x16& x) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (x[4 * i] + x[4 * i + 1]) + (x[4 * i + 2] + x[4 * i + 3]);
    return (y[0] + y[1]) + (y[2] + y[3]);
}

// a wave's own LDS: what its lanes have written is there for all of them
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// Sums of a piece along its offsets: lane o < 63 gets the sum over the rows r of what lane r - o + 31 of a half has for row r.
// Eight rows at a time go to LDS, each moved on by its place, and come back as columns: 16 writes and 32 reads without a
// bank conflict.  (16 ds_add_f32 at the offsets, some 2.5 cycles a lane each: dQ with the table's gradient, 8 sentences, 16
// heads of 64, 130 us, now 68; 6 documents, 32 heads of 128, 1160 us, now 608.)  What the writes leave out is zero throughout.
constexpr int kSkewPitch = 40;              // offsets 0 .. 38 of eight rows, and a column of zeros
__device__ __forceinline__ float sum_by_offset(float* skew, const f32x16& x, int lane) {
    const int h = lane >> 5;
    float* put = skew + 4 * h * (kSkewPitch + 1) + 31 - (lane & 31);
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        wave_sync();
#pragma unroll
        for (int e = 0; e < 4; ++e) put[e * (kSkewPitch + 1)] = x[4 * g + e];
        wave_sync();
        const float* get = skew + ((unsigned)(lane - 8 * g) < 39u ? lane - 8 * g : 39);
#pragma unroll
        for (int r = 0; r < 8; ++r) sum += get[r * kSkewPitch];
    }
    return sum;
}

// step(i, i % 2) for i < n.  TWO: two steps a turn, so that the stage is a constant and its LDS offset part of the
// instructions (2 - 5 % of the time at width 128; where registers are short already, it costs more)
template <bool TWO, class S>
__device__ __forceinline__ void each_step(int n, S step) {
    if constexpr (TWO) {
        for (int i = 0; i < n; i += 2) {
            step(i, 0);
            if (i + 1 < n) step(i + 1, 1);
        }
    } else {
        for (int i = 0; i < n; ++i) step(i, i & 1);
    }
}

// ---- the bias of a piece
//
// A piece of 32 x 32 pairs has 63 offsets.  Far from the diagonal they share a bucket, and the bias is one number that
// joins the softmax's reference point: no work per pair.  Around the diagonal, where buckets are narrow, the values of
// kWindow offsets lie in LDS for the whole launch, and a pair reads the one at a fixed distance from its lane's place.
// A piece outside this window that a border of buckets crosses gets its values by a look-up, a lane for each offset.
constexpr int kWindow = 256;
__device__ __forceinline__ int window_base(int causal) { return causal ? kWindow - 32 : kWindow / 2; }     // place of offset 0
struct RelLds {
    const int* start;       // of the buckets
    const float* tab;       // [buckets] of the head, in the units of P::expo
    const float* win;       // [kWindow] by offset
    float* slice;           // [64] of the wave
};
__device__ __forceinline__ int fast_bucket(const RelPos& r, const int* start, int causal, int offset) {
    const int dist = causal ? max(-offset, 0) : abs(offset);        // (offsets above 0 are masked then)
    const float up = __builtin_amdgcn_logf((float)max(dist, 1)) - r.log2_exact;
    int b = min(max(r.exact + (int)(up * r.per_octave), 0), r.n - 1);
    const int s0 = start[b], s1 = start[min(b + 1, r.n - 1)];       // the estimate is off by less than one
    if (s0 > dist) --b;
    else if (b + 1 < r.n && s1 <= dist) ++b;
    if (dist < r.exact) b = dist;
    return b + (!causal && offset > 0 ? r.n : 0);
}
enum { ONE_BUCKET, IN_WINDOW, LOOKED_UP };
// The piece whose offsets are offset0 .. offset0 + 62: ONE_BUCKET: `value` is its bias and `bucket` the bucket; else `by`
// points at offset0's value, and after LOOKED_UP `bucket` is that of the lane's offset (the last one again in lane 63).
__device__ __forceinline__ int bias_of_piece(const RelPos& r, const RelLds& x, int causal, int offset0, int lane, float& value,
                                             int& bucket, const float*& by) {
    const int place = offset0 + window_base(causal);
    if ((unsigned)place <= (unsigned)(kWindow - 63)) {
        by = x.win + place;
        return IN_WINDOW;
    }
    by = x.slice;
    if (offset0 + 62 <= -r.far || (!causal && offset0 >= r.far)) {
        bucket = offset0 < 0 ? r.n - 1 : 2 * r.n - 1;
        value = x.tab[bucket];
        return ONE_BUCKET;
    }
    bucket = fast_bucket(r, x.start, causal, offset0 + min(lane, 62));
    value = x.tab[bucket];
    const int b0 = __builtin_amdgcn_readlane(bucket, 0), b1 = __builtin_amdgcn_readlane(bucket, 62);
    if (b0 == b1) {
        value = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(value), 0));
        bucket = b0;
        return ONE_BUCKET;
    }
    x.slice[lane] = value;
    wave_sync();
    return LOOKED_UP;
}

// LDS behind the stages: starts of the buckets, values by bucket and by offset of the block's HP heads, a slice per wave
constexpr int kRelHead = kMaxBuckets + kWindow;
template <int NW, int HP> constexpr size_t rel_lds() { return (kMaxBuckets + HP * kRelHead + NW * 64) * sizeof(float); }

// hw: which of the block's heads is the wave's
template <class P, int NW, int HP>
__device__ __forceinline__ RelLds rel_init(const PackedArgs& a, char* lds, int head, int hw, int wave) {
    int* start = (int*)lds;
    float* tab = (float*)lds + kMaxBuckets;
    for (int i = threadIdx.x; i < a.rel.n; i += NW * 64) start[i] = a.rel.start[i];
#pragma unroll
    for (int u = 0; u < HP; ++u) {
        for (int i = threadIdx.x; i < a.rel.buckets; i += NW * 64)
            tab[u * kRelHead + i] = packed_bias(a.rel.table[(size_t)i * a.heads + head + u]) * P::kUnit;
        for (int i = threadIdx.x; i < kWindow; i += NW * 64)
            tab[u * kRelHead + kMaxBuckets + i] =
                packed_bias(a.rel.table[(size_t)fast_bucket(a.rel, a.rel.start, a.causal, i - window_base(a.causal)) * a.heads + head + u]) * P::kUnit;
    }
    tab += hw * kRelHead;
    return {start, tab, tab + kMaxBuckets, (float*)lds + kMaxBuckets + HP * kRelHead + wave * 64};
}

// Adds what the lanes have for offsets offset0 + lane (buckets `bucket`) to the wave's sums by bucket.  Offsets of one bucket
// are neighbours: the first lane of them ends up with their sum.
__device__ __forceinline__ void add_by_bucket(float* sums, int bucket, float sum, int lane) {
    const int before = __shfl_up(bucket, 1, 64);
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const float next = __shfl_down(sum, k, 64);
        const int other = __shfl_down(bucket, k, 64);
        if (lane + k < 64 && other == bucket) sum += next;
    }
    if (lane == 0 || before != bucket) sums[bucket] += sum;
}

// =====================================================================================
// Forward.  A block of 64 queries: 2 groups of 32 x 2 halves of every tile of 64 keys; every wave keeps its own online
// softmax, and the halves are merged through LDS at the end.  WIDE: a wave takes 32 queries and whole tiles, half the loads
// and barriers per product and nothing to merge: 1: 128 queries of a head, 2: 64 queries of two heads that share keys.
// =====================================================================================
template <class P, int WIDE, bool BIAS>
__global__ __launch_bounds__(256, P::D * sizeof(typename P::elem) <= 256 ? 2 : 1) void packed_fwd_kernel(PackedArgs a) {
    typedef typename P::elem elem;
    constexpr int HP = WIDE ? WIDE : 1, QB = WIDE ? 128 / HP : 64, NH = WIDE ? 2 : 1;
    constexpr int NW = 4, DT = P::DT, TILE = P::TILE, STAGE = 2 * TILE;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    packed_args_now(a);

    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hw = HP == 2 ? wave >> 1 : 0, qg = HP == 2 ? wave & 1 : WIDE ? wave : wave >> 1, kh = WIDE ? 0 : wave & 1;
    int blk, head, kvh;
    packed_coords<HP>(a, blockIdx.x, (a.T + QB - 1) / QB, blk, head, kvh);
    const int head0 = head;
    head += hw;
    const int q_wave = blk * QB + qg * 32, q_lane = q_wave + (lane & 31);
    const elem* kbase = (const elem*)a.k + kvh * a.d;
    const elem* vbase = (const elem*)a.v + kvh * a.d;
    typename P::Rows qf;
    P::load(qf, (const elem*)a.q + (size_t)min(q_lane, a.T - 1) * a.ld_q + head * a.d, h, a.d);
    const Ranges x = block_ranges<QB>(a, blk * QB, qg * 32 + (lane & 31), lane, false);
    if (!x.blk_hi) return;
    const int t0 = x.blk_lo >> 6, nt = ((x.blk_hi + 63) >> 6) - t0;
    const float c = a.scale * P::kUnit;
    RelLds rel{};
    if constexpr (BIAS) rel = rel_init<P, NW, HP>(a, smem + 2 * STAGE, head0, hw, wave);

    TileLoader<P, NW> lk, lv;
    lk.init(wave, lane, a.ld_k, a.d);
    lv.init(wave, lane, a.ld_v, a.d);
    auto request = [&](int t) {
        char* st = smem + (t & 1) * STAGE;
        const int r0 = (t0 + t) * 64;
        lk.issue(kbase + (size_t)r0 * a.ld_k, a.ld_k, a.d, x.blk_lo - r0, x.blk_hi - r0, st, wave);
        lv.issue(vbase + (size_t)r0 * a.ld_v, a.ld_v, a.d, x.blk_lo - r0, x.blk_hi - r0, st + TILE, wave);
    };

    f32x16 ot[DT];
    float m, lsum;
    auto walk = [&](auto by_rows) __attribute__((always_inline)) {
        const int lane = lane_of(threadIdx.x), h = lane >> 5;
        clear<DT>(ot);
        m = -INFINITY;
        lsum = 0.f;
        request(0);
        auto step = [&](int t, int slot) __attribute__((always_inline)) {
            BP_WAIT_VMCNT(0);
            __syncthreads();
            if (t + 1 < nt) request(t + 1);
            const int kw = (t0 + t) * 64 + 32 * kh;
            const char* sk = smem + slot * STAGE;
            const char* sv = sk + TILE;
            f32x16 s[NH];
            clear<NH>(s);
            P::template scores<NH>(sk, 32 * kh, lane, qf, s);
            float f[NH], o[NH];             // score in the units of expo: f s + o
#pragma unroll
            for (int u = 0; u < NH; ++u) {
                f[u] = c;
                o[u] = 0.f;
                if constexpr (BIAS) {
                    float value;
                    int bucket;
                    const float* b;
                    if (bias_of_piece(a.rel, rel, a.causal, kw + 32 * u - q_wave - 31, lane, value, bucket, b) != ONE_BUCKET) {
                        b += 31 + 4 * h - (lane & 31);
#pragma unroll
                        for (int v = 0; v < 16; ++v) s[u][v] = __builtin_fmaf(s[u][v], c, b[8 * (v >> 2) + (v & 3)]);
                        f[u] = 1.f;
                    } else {
                        o[u] = value;
                    }
                }
            }
            const bool masked = kw < x.inner_lo || kw + 32 * NH > x.inner_hi;
            if (masked) {
                asm volatile("");           // keeps the condition a branch, not a select per pair of every tile
#pragma unroll
                for (int u = 0; u < NH; ++u) {
                    // (a row that sees nothing of the piece: its bucket's bias may be NaN or infinite)
                    if (BIAS && (kw + 32 * u >= x.hi || kw + 32 * u + 32 <= x.lo)) o[u] = 0.f;
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if ((unsigned)(kw + 32 * u + piece_row(v, h) - x.lo) >= (unsigned)(x.hi - x.lo)) s[u][v] = -INFINITY;
                }
            }
            float mx = -INFINITY, w[NH];
#pragma unroll
            for (int u = 0; u < NH; ++u) {
                w[u] = s[u][0];
#pragma unroll
                for (int v = 1; v < 16; ++v) w[u] = fmaxf(w[u], s[u][v]);
                mx = fmaxf(mx, BIAS ? __builtin_fmaf(w[u], f[u], o[u]) : w[u]);
            }
            mx = halves_max(mx);
            if (!BIAS) mx *= c;
            // the reference point moves only when a score is more than 8 binary orders above it
            if (__builtin_amdgcn_ballot_w64(mx > m + 8.f * P::kBit) != 0) {
                const float m_new = fmaxf(m, mx);
                const float alpha = m == -INFINITY ? 0.f : P::expo(m - m_new);
                m = m_new;
                lsum *= alpha;
#pragma unroll
                for (int t2 = 0; t2 < DT; ++t2)
#pragma unroll
                    for (int v = 0; v < 16; ++v) ot[t2][v] *= alpha;
            }
            const float m_use = m == -INFINITY ? 0.f : m;       // nothing but -inf so far: no inf - inf
#pragma unroll
            for (int u = 0; u < NH; ++u) {
                float off = -m_use;
                if constexpr (BIAS) {
                    off = o[u] - m_use;
                    // A value beyond some 2^27 rounds the scores away in m, not in s: they join it here, one by one, or the
                    // exponential of a large score, with nothing subtracted, would be infinite.
                    if (__builtin_amdgcn_ballot_w64(__builtin_fmaf(w[u], f[u], off) > 16.f * P::kBit) != 0) {
                        asm volatile("");
#pragma unroll
                        for (int v = 0; v < 16; ++v) s[u][v] = __builtin_fmaf(s[u][v], f[u], o[u]);
                        f[u] = 1.f;
                        off = -m_use;
                    }
                }
                float ps = 0.f;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float p = P::expo(__builtin_fmaf(s[u][v], f[u], off));
                    s[u][v] = p;
                    ps += p;
                }
                lsum += ps;
            }
#pragma unroll
            for (int u = 0; u < NH; ++u) {
                if constexpr (decltype(by_rows)::value)
                    contract_by_rows<P>(sv, 32 * (kh + u), lane, x.lo - kw - 32 * u, x.hi - kw - 32 * u, s[u], ot);
                else
                    P::contract(sv, 32 * (kh + u), lane, s[u], ot);
            }
        };
        each_step<true>(nt, step);
    };
    walk(std::false_type{});
    if (__syncthreads_or(x.hi > x.lo && any_nan<DT>(ot))) walk(std::true_type{});

    float l = halves_sum(lsum), mm = m;
    if constexpr (!WIDE) {                  // the waves of the second halves hand (m, l, O^T) over; a half may have seen nothing
        __syncthreads();
        float* xo = (float*)smem + qg * (DT * 16 * 64 + 128);
        if (kh) {
#pragma unroll
            for (int t2 = 0; t2 < DT; ++t2)
#pragma unroll
                for (int v = 0; v < 16; ++v) xo[(t2 * 16 + v) * 64 + lane] = ot[t2][v];
            xo[DT * 16 * 64 + lane] = m;
            xo[DT * 16 * 64 + 64 + lane] = l;
        }
        __syncthreads();
        if (kh) return;
        const float m1 = xo[DT * 16 * 64 + lane];
        mm = fmaxf(m, m1);
        const float use = mm == -INFINITY ? 0.f : mm, a0 = P::expo(m - use), a1 = P::expo(m1 - use);
        l = l * a0 + xo[DT * 16 * 64 + 64 + lane] * a1;
#pragma unroll
        for (int t2 = 0; t2 < DT; ++t2)
#pragma unroll
            for (int v = 0; v < 16; ++v) ot[t2][v] = ot[t2][v] * a0 + xo[(t2 * 16 + v) * 64 + lane] * a1;
    }
    if (x.hi <= x.lo) return;
    const float inv = 1.f / l;
    elem* out = (elem*)a.ctx + (size_t)q_lane * a.ld_o + head * a.d;
#pragma unroll
    for (int t2 = 0; t2 < DT; ++t2)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = t2 * 32 + 8 * g + 4 * h;
            if (col < a.d) P::store(out + col, f32x4{ot[t2][4 * g] * inv, ot[t2][4 * g + 1] * inv, ot[t2][4 * g + 2] * inv, ot[t2][4 * g + 3] * inv});
        }
    if (h == 0) a.lse[(size_t)head * a.T + q_lane] = mm * P::kToNatural + log2f(l) * 0.6931471805599453f;
}

// =====================================================================================
// dQ, and delta for dK/dV.  Decomposed as the forward (PAIR: 64 queries of two heads that share keys):
//   S^T = K Q^T, P^T = exp(S^T - lse), dP^T = V dO^T, dS^T = P^T (dP^T - delta), dQ^T += K^T dS^T
// delta = dO . ctx, or the sum of P dP over a first walk of the keys where the rounding of ctx to bf16 would be felt:
//   the table's gradient is wanted: the last buckets' sums are small differences of many pairs (half a percent of them came
//     from the rounding at 2048 tokens);
//   a row has few keys, so that delta is not small beside dP: up to kShort; the walk is over the tiles of such rows only
//     (relative error of dQ over sequences of 1 to 40 tokens 2.8e-3 before, now 2.4e-3; 1.7e-3 is the rounding of dQ itself
//     and as much that of dS).
//
// The table's gradient: a piece of one bucket adds dS to a register; others are summed by offset (sum_by_offset).  Sums by
// offset become sums by bucket with a segmented sum over the lanes: of the window once, at the end; of a piece outside at once.
// =====================================================================================
template <int NW> constexpr size_t table_lds() { return (size_t)NW * (8 * kSkewPitch + kMaxBuckets + kWindow) * sizeof(float); }

template <class P, bool PAIR, bool BIAS>
__global__ __launch_bounds__(256, P::D * sizeof(typename P::elem) <= 256 ? 2 : 1) void packed_dq_kernel(PackedArgs a) {
    static_assert(!(PAIR && BIAS), "the table's gradient: one head a block");
    typedef typename P::elem elem;
    constexpr int HP = PAIR ? 2 : 1, QB = 64, NH = PAIR ? 2 : 1;
    constexpr int NW = 4, DT = P::DT, TILE = P::TILE, STAGE = 2 * TILE;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    packed_args_now(a);

    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hw = PAIR ? wave >> 1 : 0, qg = PAIR ? wave & 1 : wave >> 1, kh0 = PAIR ? 0 : wave & 1;
    int blk, head, kvh;
    packed_coords<HP>(a, blockIdx.x, (a.T + QB - 1) / QB, blk, head, kvh);
    head += hw;
    const int q_wave = blk * QB + qg * 32, q_lane = q_wave + (lane & 31), q_src = min(q_lane, a.T - 1);
    const elem* kbase = (const elem*)a.k + kvh * a.d;
    const elem* vbase = (const elem*)a.v + kvh * a.d;
    typename P::Rows qf, dof;
    P::load(qf, (const elem*)a.q + (size_t)q_src * a.ld_q + head * a.d, h, a.d);
    P::load(dof, (const elem*)a.dctx + (size_t)q_src * a.ld_o + head * a.d, h, a.d);
    const size_t li = (size_t)head * a.T + q_src;
    float lse = a.lse[li] * P::kUnit, delta;
    {
        typename P::Rows of;
        P::load(of, (const elem*)a.ctx + (size_t)q_src * a.ld_o + head * a.d, h, a.d);
        delta = halves_sum(P::dot(of, dof));
    }
    const Ranges x = block_ranges<QB>(a, blk * QB, qg * 32 + (lane & 31), lane, false);
    // Of one key alone dS is 0, not what two roundings of dP and delta leave (but NaN where they are not finite).
    const bool one = x.hi - x.lo == 1;
    if (one && kh0 == 0 && h == 0) a.delta[li] = delta;
    if (one && delta - delta == 0.f) {
        P::zero(dof);
        delta = 0.f;
    }
    const bool grad = BIAS && a.table_part;
    auto put_part = [&](float v) { a.table_part[((size_t)blk * a.heads + head) * a.rel.buckets + threadIdx.x] = v; };
    if (!x.blk_hi) {
        if (grad && threadIdx.x < a.rel.buckets) put_part(0.f);
        return;
    }
    const int t0 = x.blk_lo >> 6, nt = ((x.blk_hi + 63) >> 6) - t0;
    const float c = a.scale * P::kUnit;
    RelLds rel{};
    float* skew = nullptr;      // of the wave: for sum_by_offset
    float* near = nullptr;      // sums by offset, in the window
    float* sums = nullptr;      // sums by bucket
    if constexpr (BIAS) {
        if (x.hi <= x.lo) {     // a row of no sequence, whatever it holds, adds nothing to the table's gradient
            P::zero(qf);
            P::zero(dof);
            delta = 0.f;
            lse = INFINITY;
        }
        rel = rel_init<P, NW, 1>(a, smem + 2 * STAGE, head, 0, wave);
        float* tg = (float*)(smem + 2 * STAGE + rel_lds<NW, 1>());
        skew = tg + wave * 8 * kSkewPitch;
        sums = tg + NW * 8 * kSkewPitch + wave * kMaxBuckets;
        near = tg + NW * (8 * kSkewPitch + kMaxBuckets) + wave * kWindow;
    }
    TileLoader<P, NW> lk, lv;
    lk.init(wave, lane, a.ld_k, a.d);
    lv.init(wave, lane, a.ld_v, a.d);
    auto request = [&](int tile, int slot) {
        char* st = smem + slot * STAGE;
        const int r0 = tile * 64;
        lk.issue(kbase + (size_t)r0 * a.ld_k, a.ld_k, a.d, x.blk_lo - r0, x.blk_hi - r0, st, wave);
        lv.issue(vbase + (size_t)r0 * a.ld_v, a.ld_v, a.d, x.blk_lo - r0, x.blk_hi - r0, st + TILE, wave);
    };

    f32x16 dq[DT];
    // what a walk over the keys is for: delta; dQ; dQ once more for values that are not finite
    enum { DELTA, GRAD, BY_ROWS };
    auto walk_keys = [&](auto what) __attribute__((always_inline)) {
        constexpr int walk = decltype(what)::value;
        const int lane = lane_of(threadIdx.x), h = lane >> 5;
        clear<DT>(dq);
        float far = 0.f, pdp = 0.f;         // sum of dS in pieces of one bucket; of P dP
        int far_bucket = -1;
        auto flush = [&]() {
            if (far_bucket < 0) return;
            const float s = wave_sum(far);
            if (lane == 0) sums[far_bucket] += s;
            far = 0.f;
        };
        if (grad) {
            for (int i = lane; i < a.rel.buckets; i += 64) sums[i] = 0.f;
            for (int i = lane; i < kWindow; i += 64) near[i] = 0.f;
            for (int i = lane; i < 8 * kSkewPitch; i += 64) skew[i] = 0.f;
        }
        const bool all = walk != DELTA || grad;
        const int first = all ? t0 : x.short_lo >> 6, n = all ? nt : ((x.short_hi + 63) >> 6) - first;
        request(first, 0);
        auto step = [&](int t, int slot) __attribute__((always_inline)) {
            BP_WAIT_VMCNT(0);
            __syncthreads();
            if (t + 1 < n) request(first + t + 1, 1 - slot);
            const char* sk = smem + slot * STAGE;
            const char* sv = sk + TILE;
#pragma unroll
            for (int kh = kh0; kh < kh0 + NH; ++kh) {
                const int kw = (first + t) * 64 + 32 * kh;
                f32x16 s, dp;
                // (-delta as the start of dP's sums saves a subtraction.  With a bias the sums are the first walk's, bit for bit:
                // the matrix cores' sums are not rounded evenly, and what they are off by from another start has the same sign
                // in every row.  Gradient of the last bucket at 4096 tokens: off by 3.1e-6 of the table's, now 0.7e-6.)
                const float d0 = BIAS || walk == DELTA ? 0.f : -delta;
#pragma unroll
                for (int v = 0; v < 16; ++v) { s[v] = 0.f; dp[v] = d0; }
                P::scores2(sk, sv, 32 * kh, lane, qf, dof, s, dp);
                float f = c, o = -lse;
                int kind = ONE_BUCKET, bucket = 0;
                if constexpr (BIAS) {
                    float value;
                    const float* b;
                    kind = bias_of_piece(a.rel, rel, a.causal, kw - q_wave - 31, lane, value, bucket, b);
                    if (kind != ONE_BUCKET) {
                        b += 31 + 4 * h - (lane & 31);
#pragma unroll
                        for (int v = 0; v < 16; ++v) s[v] = __builtin_fmaf(s[v], c, b[8 * (v >> 2) + (v & 3)]);
                        f = 1.f;
                    } else {
                        o = value - lse;
                    }
                }
                const bool masked = kw < x.inner_lo || kw + 32 > x.inner_hi;
                if (masked) {
                    asm volatile("");
                    if (BIAS && walk == DELTA && (kw >= x.hi || kw + 32 <= x.lo)) o = -lse;     // (as in the forward)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if ((unsigned)(kw + piece_row(v, h) - x.lo) >= (unsigned)(x.hi - x.lo)) {
                            s[v] = -INFINITY;
                            if (walk == DELTA) dp[v] = 0.f;     // (NaN otherwise, which brings about the last walk)
                        }
                }
#pragma unroll
                for (int v = 0; v < 16; ++v)                // dS^T, or P dP
                    dp[v] = (BIAS && walk != DELTA ? dp[v] - delta : dp[v]) * P::expo(__builtin_fmaf(s[v], f, o));
                // delta or lse of a row may be NaN: pairs that the row does not see are left out of the sums below by its
                // own range, also in pieces that other rows see whole, for a row of no sequence
                if constexpr (BIAS && walk == BY_ROWS)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if ((unsigned)(kw + piece_row(v, h) - x.lo) >= (unsigned)(x.hi - x.lo)) dp[v] = 0.f;
                if constexpr (walk == DELTA) {
                    pdp += sum_of(dp);
                    continue;
                }
                if constexpr (BIAS) {
                    if (grad && kind == ONE_BUCKET) {
                        bucket = __builtin_amdgcn_readfirstlane(bucket);
                        if (bucket != far_bucket) flush();
                        far_bucket = bucket;
                        far += sum_of(dp);
                    } else if (grad) {
                        const float sum = sum_by_offset(skew, dp, lane);
                        if (kind == LOOKED_UP) add_by_bucket(sums, bucket, sum, lane);
                        else if (lane < 63) near[kw - q_wave - 31 + window_base(a.causal) + lane] += sum;
                    }
                }
                if constexpr (walk == BY_ROWS) contract_by_rows<P>(sk, 32 * kh, lane, x.lo - kw, x.hi - kw, dp, dq);
                else P::contract(sk, 32 * kh, lane, dp, dq);
            }
        };
        each_step<!BIAS || DT == 4>(n, step);
        if constexpr (walk == DELTA) {
            float sum = halves_sum(pdp);
            if constexpr (!PAIR) {          // two waves have half the keys of a row each
                float* ex = (float*)(smem + 2 * STAGE + (BIAS ? rel_lds<NW, 1>() : 0));      // the place of `skew`
                ex[wave * 64 + lane] = sum;
                __syncthreads();
                sum = ex[(wave & 2) * 64 + lane] + ex[(wave | 1) * 64 + lane];
            }
            if (all || x.hi - x.lo <= kShort) delta = sum;          // (a rule on the row alone, whatever else was walked)
            __syncthreads();                // (and the stages are free for the next walk)
        } else if (grad) {
            flush();
            wave_sync();
            for (int i = lane; i < kWindow; i += 64)
                add_by_bucket(sums, fast_bucket(a.rel, rel.start, a.causal, i - window_base(a.causal)), near[i], lane);
        }
    };
    if constexpr (P::kRounds)
        if (grad || x.short_hi) walk_keys(std::integral_constant<int, DELTA>{});
    walk_keys(std::integral_constant<int, GRAD>{});
    if (__syncthreads_or(x.hi > x.lo && any_nan<DT>(dq))) walk_keys(std::integral_constant<int, BY_ROWS>{});
    if (kh0 == 0 && h == 0 && x.hi > x.lo + 1) a.delta[li] = delta;

    __syncthreads();
    if (grad && threadIdx.x < a.rel.buckets) {
        const float* tg = (const float*)(smem + 2 * STAGE + rel_lds<NW, 1>()) + NW * 8 * kSkewPitch + threadIdx.x;
        put_part(tg[0] + tg[kMaxBuckets] + (tg[2 * kMaxBuckets] + tg[3 * kMaxBuckets]));
    }
    float* xo = (float*)smem + (PAIR ? 0 : qg * (DT * 16 * 64));
    if constexpr (!PAIR) {
        if (kh0 == 1) {
#pragma unroll
            for (int t2 = 0; t2 < DT; ++t2)
#pragma unroll
                for (int v = 0; v < 16; ++v) xo[(t2 * 16 + v) * 64 + lane] = dq[t2][v];
        }
        __syncthreads();
        if (kh0 == 1) return;
    }
    if (x.hi <= x.lo) return;
    elem* out = (elem*)a.dq + (size_t)q_lane * a.ld_q + head * a.d;
#pragma unroll
    for (int t2 = 0; t2 < DT; ++t2)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = (PAIR ? dq[t2][4 * g + e] : dq[t2][4 * g + e] + xo[(t2 * 16 + 4 * g + e) * 64 + lane]) * a.scale;
            const int col = t2 * 32 + 8 * g + 4 * h;
            if (col < a.d) P::store(out + col, w);
        }
}

// =====================================================================================
// dK and dV of 64 keys of a key / value head: 2 groups of 32 keys x 2 halves of every tile of 64 queries, the tiles of the
// heads that share them one after the other: all of them, or with a.splits > 1 an equal part, whose fp32 sums
// go to the workspace and are joined in a fixed order by packed_join_kernel (split_heads).
//   S = Q K^T, P = exp(S - lse[q]), dP = dO V^T, dS = P (dP - delta[q]), dV^T += dO^T P, dK^T += Q^T dS
// =====================================================================================
template <class P, bool BIAS>
__global__ __launch_bounds__(256, P::kDkvBlocks) void packed_dkv_kernel(PackedArgs a) {
    typedef typename P::elem elem;
    constexpr int NW = 4, DT = P::DT, KB = 64, TILE = P::TILE;
    constexpr int STAGE = 2 * TILE + 512;               // Q, dO, -lse[64], -delta[64]
    constexpr int KL = P::kKeysInLds ? P::kKeysInLds - BIAS : 0;        // (two blocks of a CU share 160 KB)
    extern __shared__ __attribute__((aligned(16))) char smem[];
    packed_args_now(a);

    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kg = wave >> 1, qh = wave & 1;
    const int G = a.heads / a.kv_heads / a.splits;                      // heads of this block
    const int blk = blockIdx.x / (a.kv_heads * a.splits);               // the first rows have most to do
    const int part = (blockIdx.x - blk * a.kv_heads * a.splits) / a.kv_heads, kvh = blockIdx.x % a.kv_heads;
    const int head0 = kvh * (a.heads / a.kv_heads) + part * G;
    const int k_wave = blk * KB + kg * 32, k_lane = k_wave + (lane & 31), k_src = min(k_lane, a.T - 1);
    typename P::Rows kf, vf;
    P::load(kf, (const elem*)a.k + (size_t)k_src * a.ld_k + kvh * a.d, h, a.d);
    P::load(vf, (const elem*)a.v + (size_t)k_src * a.ld_v + kvh * a.d, h, a.d);
    const Ranges x = block_ranges<KB>(a, blk * KB, kg * 32 + (lane & 31), lane, true);
    if (!x.blk_hi) return;
    const int t0 = x.blk_lo >> 6, nt = ((x.blk_hi + 63) >> 6) - t0;
    const float c = a.scale * P::kUnit;
    RelLds rel{};
    float* values = nullptr;                // by bucket and by offset, of the heads of even and of odd number
    if constexpr (BIAS) {
        int* start = (int*)(smem + 2 * STAGE);
        for (int i = threadIdx.x; i < a.rel.n; i += 256) start[i] = a.rel.start[i];
        values = (float*)(start + kMaxBuckets);
        rel = {start, nullptr, nullptr, values + 2 * kRelHead + wave * 64};
    }
    int my_bucket = 0;                      // of this thread's place in the window
    if constexpr (BIAS) my_bucket = fast_bucket(a.rel, a.rel.start, a.causal, (int)threadIdx.x - window_base(a.causal));
    static_assert(kWindow == 256, "a place for every thread");
    TileLoader<P, NW> lq, lo;
    lq.init(wave, lane, a.ld_q, a.d);
    lo.init(wave, lane, a.ld_o, a.d);
    char* keys = smem + 2 * STAGE + (BIAS ? rel_lds<4, 2>() : 0) + kg * KL * 1024;
    if constexpr (KL > 0)
        if (qh == 0) P::template put_rows<KL>(kf, keys, lane);
    // Step i takes tile t0 + i % nt of head head0 + i / nt.  Statistics (waves 0 and 1) and a head's values go through
    // registers, where they get the sign and the base that the exponential and the accumulators want; they are fetched two
    // steps ahead, so that nothing waits for them but the wait at the top of a step.
    const int steps = nt * G;
    const float* stat = wave == 0 ? a.lse : a.delta;
    const float stat_factor = wave == 0 ? -P::kUnit : -1.f;
    auto fetch_stat = [&](int g, int t) {
        // (rows of the tile that the block's keys are not seen by have those of one that does: what others hold may be NaN)
        const int row = min(max((t0 + t) * 64 + lane, x.blk_lo), x.blk_hi - 1);
        return wave < 2 && g < G ? stat[(size_t)(head0 + g) * a.T + row] : 0.f;
    };
    auto put_stat = [&](float v, char* stage) {
        if (wave < 2) ((float*)(stage + 2 * TILE))[wave * 64 + lane] = v * stat_factor;
    };
    auto fetch_tab = [&](int g) {
        return BIAS && g < G && threadIdx.x < a.rel.buckets ? a.rel.table[(size_t)threadIdx.x * a.heads + head0 + g] : 0.f;
    };
    auto fetch_win = [&](int g) { return BIAS && g < G ? a.rel.table[(size_t)my_bucket * a.heads + head0 + g] : 0.f; };
    auto put_values = [&](float tab, float win, int g) {
        float* to = values + (g & 1) * kRelHead;
        if (threadIdx.x < a.rel.buckets) to[threadIdx.x] = packed_bias(tab) * P::kUnit;
        to[kMaxBuckets + threadIdx.x] = packed_bias(win) * P::kUnit;
    };
    auto request = [&](int g, int t, char* stage) {
        const int r0 = (t0 + t) * 64, col = (head0 + g) * a.d;
        lq.issue((const elem*)a.q + (size_t)r0 * a.ld_q + col, a.ld_q, a.d, x.blk_lo - r0, x.blk_hi - r0, stage, wave);
        lo.issue((const elem*)a.dctx + (size_t)r0 * a.ld_o + col, a.ld_o, a.d, x.blk_lo - r0, x.blk_hi - r0, stage + TILE, wave);
    };
    auto advance = [&](int& g, int& t) { if (++t == nt) { t = 0; ++g; } };

    f32x16 dk[DT], dv[DT];
    auto walk = [&](auto by_rows) __attribute__((always_inline)) {
        const int lane = lane_of(threadIdx.x), h = lane >> 5;
        clear<DT>(dk);
        clear<DT>(dv);
        int g = 0, t = 0, g1 = 0, t1 = 0, g2 = 0, t2 = 0;       // this step's head and tile; the next step's; those after it
        advance(g1, t1);
        const float st0 = fetch_stat(0, 0);
        float st1 = fetch_stat(g1, t1), tab1 = 0.f, win1 = 0.f;
        if constexpr (BIAS) {
            put_values(fetch_tab(0), fetch_win(0), 0);
            if (t1 == 0) { tab1 = fetch_tab(g1); win1 = fetch_win(g1); }
        }
        request(0, 0, smem);
        put_stat(st0, smem);
        auto step = [&](int i, int slot) __attribute__((always_inline)) {
            BP_WAIT_VMCNT(0);
            __syncthreads();
            if (i + 1 < steps) {
                put_stat(st1, smem + (1 - slot) * STAGE);
                // (the values that a head's first step replaces are those of the last but one)
                if (BIAS && t1 == 0) put_values(tab1, win1, g1);
                request(g1, t1, smem + (1 - slot) * STAGE);
                g2 = g1; t2 = t1;
                advance(g2, t2);
                st1 = fetch_stat(g2, t2);
                if (BIAS && t2 == 0) { tab1 = fetch_tab(g2); win1 = fetch_win(g2); }
            }
            const char* sq = smem + slot * STAGE;
            const char* sdo = sq + TILE;
            const int q0 = (t0 + t) * 64;
            if constexpr (BIAS) {
                rel.tab = values + (g & 1) * kRelHead;
                rel.win = rel.tab + kMaxBuckets;
            }
            g = g1; t = t1; g1 = g2; t1 = t2;
            const int qw = q0 + 32 * qh;
            const float* nlse = (const float*)(sq + 2 * TILE) + 32 * qh;
            const float* ndlt = nlse + 64;
            f32x16 s, dp;
#pragma unroll
            for (int v = 0; v < 16; ++v) { s[v] = 0.f; dp[v] = ndlt[piece_row(v, h)]; }
            if constexpr (KL > 0) P::template scores2<KL>(sq, sdo, 32 * qh, lane, keys, kf, vf, s, dp);
            else P::scores2(sq, sdo, 32 * qh, lane, kf, vf, s, dp);
            float f = c, o = 0.f;
            if constexpr (BIAS) {
                int bucket;
                float value;
                const float* b;
                if (bias_of_piece(a.rel, rel, a.causal, k_wave - qw - 31, lane, value, bucket, b) != ONE_BUCKET) {
                    b += 31 + (lane & 31) - 4 * h - 27;         // offsets fall with the register's row, 0 .. 27 here
#pragma unroll
                    for (int v = 0; v < 16; ++v) s[v] = __builtin_fmaf(s[v], c, b[27 - 8 * (v >> 2) - (v & 3)]);
                    f = 1.f;
                } else {
                    o = value;
                }
            }
            const bool masked = qw < x.inner_lo || qw + 32 > x.inner_hi;
            if (masked) {
                asm volatile("");
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if ((unsigned)(qw + piece_row(v, h) - x.lo) >= (unsigned)(x.hi - x.lo)) {
                        s[v] = -INFINITY;
                        if (decltype(by_rows)::value) dp[v] = 0.f;
                    }
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                s[v] = P::expo(__builtin_fmaf(s[v], f, BIAS ? nlse[piece_row(v, h)] + o : nlse[piece_row(v, h)]));     // P
                dp[v] *= s[v];                                                                                        // dS
            }
            if constexpr (decltype(by_rows)::value) {
                contract_by_rows<P>(sdo, 32 * qh, lane, x.lo - qw, x.hi - qw, s, dv);
                contract_by_rows<P>(sq, 32 * qh, lane, x.lo - qw, x.hi - qw, dp, dk);
            } else {
                P::contract2(sdo, sq, 32 * qh, lane, s, dp, dv, dk);
            }
        };
        each_step<!BIAS>(steps, step);
    };
    walk(std::false_type{});
    if (__syncthreads_or(x.hi > x.lo && (any_nan<DT>(dk) || any_nan<DT>(dv)))) walk(std::true_type{});
    float* xo = (float*)smem + kg * (2 * DT * 16 * 64);
    __syncthreads();
    if (qh == 1) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                xo[(t * 16 + v) * 64 + lane] = dk[t][v];
                xo[((DT + t) * 16 + v) * 64 + lane] = dv[t][v];
            }
    }
    __syncthreads();
    if (qh == 1) return;
    if (x.hi <= x.lo) return;
    const float scale = (x.alone >> (kg * 32 + (lane & 31))) & 1 ? 0.f : a.scale;       // (dS is 0 there, as in dQ)
    elem* dk_out = (elem*)a.dk + (size_t)k_lane * a.ld_k + kvh * a.d;
    elem* dv_out = (elem*)a.dv + (size_t)k_lane * a.ld_v + kvh * a.d;
    float* sums = a.splits > 1 ? a.dkv_part + (((size_t)part * a.T + k_lane) * a.kv_heads + kvh) * 2 * a.d : nullptr;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int col = t * 32 + 8 * g + 4 * h;
            f32x4 k4, v4;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                k4[e] = (dk[t][4 * g + e] + xo[(t * 16 + 4 * g + e) * 64 + lane]) * scale;
                v4[e] = dv[t][4 * g + e] + xo[((DT + t) * 16 + 4 * g + e) * 64 + lane];
            }
            if (col >= a.d) continue;
            if (sums) {
                *reinterpret_cast<f32x4*>(sums + col) = k4;
                *reinterpret_cast<f32x4*>(sums + a.d + col) = v4;
            } else {
                P::store(dk_out + col, k4);
                P::store(dv_out + col, v4);
            }
        }
}

// What is left to sum after dK/dV, in one launch: blocks below a.heads the partials of the table's gradient, if it is wanted,
// the others dK and dV from the parts' sums, four columns of a row to a thread.
template <class P>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedArgs a) {
    __shared__ float sums[256];
    int block = blockIdx.x;
    if (a.table_part) {
        if (block < a.heads) {
            sum_table_part(a, block, sums);
            return;
        }
        block -= a.heads;
    }
    const int per = a.kv_heads * 2 * a.d / 4;           // threads a row
    const size_t i = (size_t)block * 256 + threadIdx.x;
    const int row = (int)(i / per), c = (int)(i - (size_t)row * per) * 4, kvh = c / (2 * a.d), col = c - kvh * 2 * a.d;
    if (row >= min(a.starts[a.n_seq], a.T) || row < a.starts[0]) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < a.splits; ++p) s += *reinterpret_cast<const f32x4*>(a.dkv_part + ((size_t)p * a.T + row) * a.kv_heads * 2 * a.d + c);
    if (col < a.d) P::store((typename P::elem*)a.dk + (size_t)row * a.ld_k + kvh * a.d + col, s);
    else P::store((typename P::elem*)a.dv + (size_t)row * a.ld_v + kvh * a.d + col - a.d, s);
}

// ---- host side

// set: a bit for each device that knows
template <typename K>
static hipError_t allow_lds(K kern, size_t bytes, std::atomic<uint64_t>& set) {
    if (bytes <= 64 * 1024) return hipSuccess;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess || (set.load(std::memory_order_acquire) >> (dev & 63) & 1)) return e;
    e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess) set.fetch_or(1ull << (dev & 63), std::memory_order_release);
    return e;
}

template <class P, int WIDE, bool BIAS>
static hipError_t launch_fwd(const PackedArgs& a, hipStream_t s) {
    constexpr int HP = WIDE ? WIDE : 1, QB = WIDE ? 128 / HP : 64;
    constexpr size_t stages = (size_t)2 * 2 * P::TILE + (BIAS ? rel_lds<4, HP>() : 0);
    constexpr size_t merge = WIDE ? 0 : (size_t)2 * (P::DT * 16 * 64 + 128) * sizeof(float);
    constexpr size_t smem = std::max(stages, merge);
    static std::atomic<uint64_t> set{0};
    const hipError_t e = allow_lds(packed_fwd_kernel<P, WIDE, BIAS>, smem, set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((packed_fwd_kernel<P, WIDE, BIAS>), dim3((a.T + QB - 1) / QB * (a.heads / HP)), dim3(256), smem, s, a);
    return hipGetLastError();
}
template <class P, bool PAIR, bool BIAS>
static hipError_t launch_dq(const PackedArgs& a, hipStream_t s) {
    constexpr size_t stages = (size_t)2 * 2 * P::TILE + (BIAS ? rel_lds<4, 1>() + table_lds<4>() : 4 * 64 * sizeof(float));
    constexpr size_t smem = std::max(stages, PAIR ? (size_t)0 : (size_t)2 * P::DT * 16 * 64 * sizeof(float));
    static std::atomic<uint64_t> set{0};
    const hipError_t e = allow_lds(packed_dq_kernel<P, PAIR, BIAS>, smem, set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((packed_dq_kernel<P, PAIR, BIAS>), dim3(packed_tiles(a.T) * (a.heads / (PAIR ? 2 : 1))), dim3(256), smem, s, a);
    return hipGetLastError();
}
template <class P, bool BIAS>
static hipError_t launch_dkv(const PackedArgs& a, hipStream_t s) {
    constexpr size_t stages = (size_t)2 * (2 * P::TILE + 512) + (BIAS ? rel_lds<4, 2>() : 0) +
                              (P::kKeysInLds ? (P::kKeysInLds - BIAS) * 2 * 1024 : 0);
    constexpr size_t smem = std::max(stages, (size_t)2 * 2 * P::DT * 16 * 64 * sizeof(float));
    static std::atomic<uint64_t> set{0};
    const hipError_t e = allow_lds(packed_dkv_kernel<P, BIAS>, smem, set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((packed_dkv_kernel<P, BIAS>), dim3(packed_tiles(a.T) * a.kv_heads * a.splits), dim3(256), smem, s, a);
    // (parts are for launches of fewer than 4 blocks a CU, so rows * kv_heads stays below 65536 on 256 CUs, threads below 2^23)
    const size_t threads = a.splits > 1 ? (size_t)a.T * (a.kv_heads * 2 * a.d / 4) : 0;
    const unsigned blocks = (unsigned)((threads + 255) / 256) + (a.table_part ? a.heads : 0);
    if (blocks) hipLaunchKernelGGL((packed_join_kernel<P>), dim3(blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace bp
