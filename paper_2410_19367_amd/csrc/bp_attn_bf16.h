// Pieces of the bf16 attention kernels on the matrix cores: the layout of a tile of 64 rows in LDS, its fragments as MFMA
// operands, and an accumulator as the operand of the next product.
#pragma once
#include "bp_device.h"
#include "bp_tile.h"

namespace bp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// bare v_exp_f32: arguments here are <= 8 and anything below -126 may flush to zero
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// An empty asm that keeps a wave-uniform condition a branch: left alone the compiler turns masking loops into one
// branch per element (forward, dQ) or into a compare and a select per element of every tile (dK/dV).  With the
// statistics of a dK/dV tile scaled once per row: forward, S 6144, 16 heads of 64, causal 122 -> 110 us, backward
// 345 -> 312 us; S 2048, 16 heads of 128 36 -> 34, 118 -> 109 us.
__device__ __forceinline__ void stay_a_branch() { asm volatile(""); }

// 8 consecutive elements of a row starting at column `col`, zeros at and beyond column dr
__device__ __forceinline__ bf16x8 load_frag(const bf16_t* row, int col, int dr) {
    bf16x8 z;
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = (bf16_t)0.f;
    return col < dr ? *reinterpret_cast<const bf16x8*>(row + col) : z;
}

// ---- tile layout: [rows][D] bf16, 16-byte chunks XOR-swizzled by row
template <int D> __device__ __forceinline__ int swz(int row) {
    return D == 128 ? (((row & 3) << 2) | ((row >> 2) & 3))
                    : ((((row >> 1) & 1) << 2) | ((row >> 2) & 3));
}
template <int D> __device__ __forceinline__ int tile_off(int row, int chunk) {
    return row * (D * 2) + ((chunk ^ swz<D>(row)) << 4);
}

// plain fragment: 8 consecutive columns (k16 step s, half h) of row (row0 + lane%32)
template <int D>
__device__ __forceinline__ bf16x8 frag_rows(const char* lds, int row0, int s, int lane) {
    return *reinterpret_cast<const bf16x8*>(lds + tile_off<D>(row0 + (lane & 31), 2 * s + (lane >> 5)));
}
// transposed fragment for a product whose contraction runs over the tile's rows: lane gets, for
// column (col0 + lane%32), the rows {r0 + 4h .. +3} and {r0 + 8 + 4h .. +3} (h = lane/32): the
// row order in which a 32x32 accumulator hands its 16 rows to the next MFMA.
template <int D>
__device__ __forceinline__ bf16x8 frag_cols(const char* lds, int r0, int col0, int lane) {
    const int i = lane & 15, g2 = (lane >> 4) & 1, h = lane >> 5;
    const int col = col0 + 16 * g2 + 4 * (i & 3);
    const int chunk = col >> 3, byte = (col & 7) * 2;
    const int ra = r0 + 4 * h + (i >> 2);
    s16x4 lo = lds_read_tr((const lds_s16x4*)(lds + tile_off<D>(ra, chunk) + byte));
    s16x4 hi = lds_read_tr((const lds_s16x4*)(lds + tile_off<D>(ra + 8, chunk) + byte));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// accumulator registers 8*half .. 8*half+7 of a 32x32 tile as a bf16 B operand
__device__ __forceinline__ bf16x8 acc_to_b(const f32x16& a, int half) {
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (bf16_t)a[8 * half + e];
    return r;
}

// row index inside a 32-row accumulator tile held in register v by a lane of half h
__device__ __forceinline__ int acc_row(int v, int h) { return 8 * (v >> 2) + 4 * h + (v & 3); }

}  // namespace bp
