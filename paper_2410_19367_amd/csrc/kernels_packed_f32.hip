// Attention over packed sequences, fp32: the kernels of bp_packed_tile.h on v_mfma_f32_32x32x2_f32.  Bound by the fp32
// matrix rate (an eighth of the bf16 one): blocks of 64 rows only.
#include "bp_attn_f32.h"
#include "bp_packed_tile.h"

namespace bp {

// DC: computed head width, 32 .. 128; narrower heads are padded with zeros
template <int DC>
struct PackedF32 {
    typedef float elem;
    static constexpr int D = DC <= 64 ? 64 : 128, KS = DC / 8, DT = DC / 32, TILE = 64 * D * 4;
    static constexpr int kDkvBlocks = D == 64 ? 2 : 1, kKeysInLds = 0;
    static constexpr bool kRounds = false;
    // natural units: the difference to the reference point is taken before the change of base, so that large scores are
    // rounded relative to what is left of them
    static constexpr float kUnit = 1.f, kBit = kLn2, kToNatural = 1.f;
    static __device__ __forceinline__ float expo(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
    static __device__ __forceinline__ int swizzle(int row) { return row & 15; }

    struct Rows { f32x4 f[KS]; };
    static __device__ __forceinline__ void load(Rows& r, const elem* row, int h, int d) {
#pragma unroll
        for (int j = 0; j < KS; ++j) r.f[j] = row_piece(row, 8 * j + 4 * h, d);
    }
    static __device__ __forceinline__ void zero(Rows& r) {
#pragma unroll
        for (int j = 0; j < KS; ++j) r.f[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    static __device__ __forceinline__ float dot(const Rows& a, const Rows& b) {
        float x = 0.f;
#pragma unroll
        for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) x += a.f[j][e] * b.f[j][e];
        return x;
    }
    template <int NH>
    static __device__ __forceinline__ void scores(const char* tile, int row0, int lane, const Rows& b, f32x16 (&s)[NH]) {
        static_assert(NH == 1, "blocks of 64 rows");
        f32x4 f[2];
        pipelined<KS>([&](int j) { f[j & 1] = rows4<D>(tile, row0, j, lane); },
                      [&](int j) {
#pragma unroll
                          for (int e = 0; e < 4; ++e) s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(f[j & 1][e], b.f[j][e], s[0], 0, 0, 0);
                      });
    }
    static __device__ __forceinline__ void scores2(const char* ta, const char* tb, int row0, int lane, const Rows& a, const Rows& b,
                                                   f32x16& s, f32x16& p) {
        bp::scores<D, DC>(ta, tb, row0, lane, a.f, b.f, s, p);
    }
    static __device__ __forceinline__ void contract(const char* tile, int row0, int lane, const f32x16& x, f32x16 (&out)[DT]) {
        bp::contract<D, DC>(tile, row0, lane, x, out);
    }
    static __device__ __forceinline__ void contract2(const char* ta, const char* tb, int row0, int lane, const f32x16& x,
                                                     const f32x16& y, f32x16 (&a)[DT], f32x16 (&b)[DT]) {
        bp::contract<D, DC>(ta, row0, lane, x, a);
        bp::contract<D, DC>(tb, row0, lane, y, b);
    }
    static __device__ __forceinline__ f32x4 four(const char* tile, int row, int col) {
        return *reinterpret_cast<const f32x4*>(tile + f32_tile_off<D>(row, col >> 2));
    }
    static __device__ __forceinline__ void store(elem* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
};

template <class P, bool BIAS>
static hipError_t both(const PackedArgs& a, bool back, hipStream_t s) {
    if (!back) return launch_fwd<P, 0, BIAS>(a, s);
    const hipError_t e = launch_dq<P, false, BIAS>(a, s);
    return e != hipSuccess ? e : launch_dkv<P, BIAS>(a, s);
}
template <int DC>
static hipError_t width(const PackedArgs& a, bool back, hipStream_t s) {
    return a.rel.buckets ? both<PackedF32<DC>, true>(a, back, s) : both<PackedF32<DC>, false>(a, back, s);
}
hipError_t launch_packed_f32(const PackedArgs& a, bool back, hipStream_t s) {
    return a.d <= 32 ? width<32>(a, back, s) : a.d <= 64 ? width<64>(a, back, s) :
           a.d <= 96 ? width<96>(a, back, s) : width<128>(a, back, s);
}

}  // namespace bp
