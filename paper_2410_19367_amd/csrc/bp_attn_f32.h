// Pieces of the fp32 attention kernels on the matrix cores: the layout of a tile of 64 rows in LDS, the copy that fills it,
// its rows and columns as MFMA operands, and the products.
#pragma once
#include "bp_device.h"
#include "bp_tile.h"

namespace bp {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// tile [64][D] floats: 16-byte chunk c of row r sits at c ^ (r & 15)
template <int D> __device__ __forceinline__ int f32_tile_off(int row, int chunk) {
    return row * (D * 4) + ((chunk ^ (row & 15)) << 4);
}

// Direct global->LDS copy of the first `rows` rows of a [64][D] tile by four waves (keys: up to the valid
// length, since what padding holds must not reach the products: zero times NaN); the other rows and
// the columns at and beyond the head width dr lie outside the buffer descriptor's range: zeros.
template <int D>
struct F32Tile {
    static constexpr int CPR = D / 4, NI = 64 * CPR / 64 / 4;
    uint32_t off[NI];
    __device__ __forceinline__ void init(int wave, int lane, int ld, int dr) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int P = (wave + 4 * i) * 64 + lane, row = P / CPR, c = (P % CPR) ^ (row & 15);
            off[i] = c * 4 < dr ? 4u * (uint32_t)(row * ld + c * 4) : kOutside;
        }
    }
    __device__ __forceinline__ void issue(const float* base, int ld, int dr, int rows, char* lds, int wave) const {
        const rsrc_t src = make_rsrc(base, 4u * (uint32_t)((min(rows, 64) - 1) * ld + dr));
#pragma unroll
        for (int i = 0; i < NI; ++i) dma16(src, off[i], 0, lds + (wave + 4 * i) * 1024);
    }
};

// chunk pair j (columns 8j .. 8j+7, this lane's half of them) of row row0 + lane % 32
template <int D>
__device__ __forceinline__ f32x4 rows4(const char* lds, int row0, int j, int lane) {
    return *reinterpret_cast<const f32x4*>(lds + f32_tile_off<D>(row0 + (lane & 31), 2 * j + (lane >> 5)));
}
// element (row, col0 + lane % 32)
template <int D>
__device__ __forceinline__ float col1(const char* lds, int row, int col0, int lane) {
    const int col = col0 + (lane & 31);
    return *reinterpret_cast<const float*>(lds + f32_tile_off<D>(row, col >> 2) + (col & 3) * 4);
}
// load(i + 1) is issued before use(i), and nothing moves across the end of a step: one step's LDS reads are
// in flight while the previous one's MFMAs run, and the compiler does not pull all the reads of a tile
// to its front (which spilled registers in the backward kernels)
template <int N, typename L, typename U>
__device__ __forceinline__ void pipelined(L load, U use) {
    load(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i + 1 < N) load(i + 1);
        use(i);
        __builtin_amdgcn_sched_barrier(0);
    }
}
__device__ __forceinline__ f32x4 row_piece(const float* row, int col, int dr) {
    return col < dr ? *reinterpret_cast<const f32x4*>(row + col) : f32x4{0.f, 0.f, 0.f, 0.f};
}
__device__ __forceinline__ int f32_acc_row(int v, int h) { return 8 * (v >> 2) + 4 * h + (v & 3); }
// out^T (D x 32) += tile[row0 .. row0 + 31][.]^T x, x as a score accumulator holds it
template <int D, int DC>
__device__ __forceinline__ void contract(const char* tile, int row0, int lane, const f32x16& x, f32x16 (&out)[DC / 32]) {
    constexpr int DT = DC / 32;
    float av[2][4][DT];
    pipelined<4>([&](int g) {
#pragma unroll
                     for (int e = 0; e < 4; ++e)
#pragma unroll
                         for (int t = 0; t < DT; ++t)
                             av[g & 1][e][t] = col1<D>(tile, row0 + f32_acc_row(4 * g + e, lane >> 5), 32 * t, lane);
                 },
                 [&](int g) {
#pragma unroll
                     for (int e = 0; e < 4; ++e)
#pragma unroll
                         for (int t = 0; t < DT; ++t)
                             out[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(av[g & 1][e][t], x[4 * g + e], out[t], 0, 0, 0);
                 });
}
// s += A b^T and p += C d^T over the head width: 32 rows of the tiles A and C, b and d in registers
template <int D, int DC>
__device__ __forceinline__ void scores(const char* tile_a, const char* tile_c, int row0, int lane,
                                       const f32x4 (&b)[DC / 8], const f32x4 (&d)[DC / 8], f32x16& s, f32x16& p) {
    f32x4 fa[2], fc[2];
    pipelined<DC / 8>([&](int j) {
                         fa[j & 1] = rows4<D>(tile_a, row0, j, lane);
                         fc[j & 1] = rows4<D>(tile_c, row0, j, lane);
                     },
                     [&](int j) {
#pragma unroll
                         for (int e = 0; e < 4; ++e) {
                             s = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[j & 1][e], b[j][e], s, 0, 0, 0);
                             p = __builtin_amdgcn_mfma_f32_32x32x2f32(fc[j & 1][e], d[j][e], p, 0, 0, 0);
                         }
                     });
}
// exp(s scale - m).  The difference is taken before the change of base: scores are then rounded relative to what is left
// of them and not to themselves (with log2 e folded into the scale, a score of 200 that is its row's only one
// had the probability 1 +- 1e-5).
__device__ __forceinline__ float exp_diff(float s, float scale, float m) {
    return __builtin_amdgcn_exp2f(__builtin_fmaf(s, scale, -m) * kLog2e);
}
__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int v = 0; v < 16; ++v) z[v] = 0.f;
    return z;
}

}  // namespace bp
