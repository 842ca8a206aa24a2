// Attention over packed sequences, bf16: the kernels of bp_packed_tile.h on v_mfma_f32_32x32x16_bf16.  P and dS are rounded
// to bf16 for the second products, 2^-8 of each term at most; what that leaves in a result is about as large as the rounding
// of the result itself (forward and backward off by 2.4e-3 of the exact results, these rounded by 1.7e-3).  Scores, softmax,
// sums and the table's gradient are fp32.
#include "bp_attn_bf16.h"
#include "bp_packed_tile.h"

namespace bp {

// DC: computed head width, 32 .. 128; narrower heads are padded with zeros
template <int DC>
struct PackedBf16 {
    typedef bf16_t elem;
    static constexpr int D = DC <= 64 ? 64 : 128, KS = DC / 16, DT = DC / 32, TILE = 64 * D * 2;
    static constexpr int kDkvBlocks = 2;
    // dK/dV: steps of the scores' contraction whose half of the keys stays in LDS, 2 KB each, where registers are short
    static constexpr int kKeysInLds = DC == 128 ? 6 : 0;
    static constexpr bool kRounds = true;               // ctx is rounded
    static constexpr float kUnit = kLog2e, kBit = 1.f, kToNatural = kLn2;      // scores in units of a binary order
    static __device__ __forceinline__ float expo(float x) { return fast_exp2(x); }
    static __device__ __forceinline__ int swizzle(int row) { return swz<D>(row); }

    struct Rows { bf16x8 f[KS]; };
    static __device__ __forceinline__ void load(Rows& r, const elem* row, int h, int d) {
#pragma unroll
        for (int s = 0; s < KS; ++s) r.f[s] = load_frag(row, 16 * s + 8 * h, d);
    }
    static __device__ __forceinline__ void zero(Rows& r) {
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) r.f[s][e] = (bf16_t)0.f;
    }
    static __device__ __forceinline__ float dot(const Rows& a, const Rows& b) {
        float x = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) x += (float)a.f[s][e] * (float)b.f[s][e];
        return x;
    }
    // s[u] += rows row0 + 32 u .. of the tile times b
    template <int NH>
    static __device__ __forceinline__ void scores(const char* tile, int row0, int lane, const Rows& b, f32x16 (&s)[NH]) {
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int u = 0; u < NH; ++u)
                s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<D>(tile, row0 + 32 * u, k, lane), b.f[k], s[u], 0, 0, 0);
    }
    static __device__ __forceinline__ void scores2(const char* ta, const char* tb, int row0, int lane, const Rows& a, const Rows& b,
                                                   f32x16& s, f32x16& p) {
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<D>(ta, row0, k, lane), a.f[k], s, 0, 0, 0);
            p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<D>(tb, row0, k, lane), b.f[k], p, 0, 0, 0);
        }
    }
    // the same with the first KL steps of a in LDS, as put_rows left them
    template <int KL>
    static __device__ __forceinline__ void put_rows(const Rows& a, char* lds, int lane) {
#pragma unroll
        for (int k = 0; k < KL; ++k) *reinterpret_cast<bf16x8*>(lds + k * 1024 + lane * 16) = a.f[k];
    }
    template <int KL>
    static __device__ __forceinline__ void scores2(const char* ta, const char* tb, int row0, int lane, const char* lds, const Rows& a,
                                                   const Rows& b, f32x16& s, f32x16& p) {
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const bf16x8 ak = k < KL ? *reinterpret_cast<const bf16x8*>(lds + k * 1024 + lane * 16) : a.f[k];
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<D>(ta, row0, k, lane), ak, s, 0, 0, 0);
            p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<D>(tb, row0, k, lane), b.f[k], p, 0, 0, 0);
        }
    }
    static __device__ __forceinline__ void contract(const char* tile, int row0, int lane, const f32x16& x, f32x16 (&out)[DT]) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const bf16x8 xb = acc_to_b(x, s);
#pragma unroll
            for (int t = 0; t < DT; ++t)
                out[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<D>(tile, row0 + 16 * s, t * 32, lane), xb, out[t], 0, 0, 0);
        }
    }
    static __device__ __forceinline__ void contract2(const char* ta, const char* tb, int row0, int lane, const f32x16& x,
                                                     const f32x16& y, f32x16 (&a)[DT], f32x16 (&b)[DT]) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const bf16x8 xb = acc_to_b(x, s), yb = acc_to_b(y, s);
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                a[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<D>(ta, row0 + 16 * s, t * 32, lane), xb, a[t], 0, 0, 0);
                b[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<D>(tb, row0 + 16 * s, t * 32, lane), yb, b[t], 0, 0, 0);
            }
        }
    }
    // four columns of a row
    static __device__ __forceinline__ f32x4 four(const char* tile, int row, int col) {
        const uint2 r = *reinterpret_cast<const uint2*>(tile + tile_off<D>(row, col >> 3) + (col & 7) * 2);
        return {__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u)};
    }
    static __device__ __forceinline__ void store(elem* p, f32x4 v) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
};

// Which form of a kernel a launch takes.  n: blocks of 64 rows of all heads.  What the sequences are is
// not known here, so the rules are by what holds whatever they are; measured on 256 CUs, narrow / wide, with sequences of
// 256, 512, 1000 to 4168, 2048 and 8192 tokens:
//   forward, d 128 (and 96): n 8192 1.20 - 1.32, 4096 1.2, 2048 1.04 - 1.3 (four long ones without a mask 0.91), 1024 with 16
//     heads or more 1.01 - 1.35, with 8 heads 0.75 - 0.94 and 1.22, 512 0.8 - 1.05, fewer 0.73 - 0.84;
//     d 64 and less: n 4096 1.0 - 1.09, 2048 0.87 - 1.13 (32 heads 1.05 - 1.28), 1024 0.8 - 1.13, fewer 0.7 - 1.0;
//     two heads to a block against 128 rows, where both can be: 1.00 - 1.12;
//   dQ (of the whole backward), two heads to a block: 32 heads or more, n from 2048 on 0.99 - 1.18, else 0.8 - 1.09; with the
//     table's gradient 0.92 - 1.01.
static bool wide_fwd(const PackedArgs& a) {
    const long cu = cu_count(), n = (long)packed_tiles(a.T) * a.heads;
    if (a.d > 64) return n >= (a.heads >= 16 ? 4 : 8) * cu;
    return n >= (a.heads >= 32 ? 8 : 16) * cu;
}
static bool pair_dq(const PackedArgs& a) {
    return a.heads / a.kv_heads % 2 == 0 && a.heads >= 32 && (long)packed_tiles(a.T) * a.heads >= 8L * cu_count();
}
template <class P, bool BIAS>
static hipError_t fwd(const PackedArgs& a, hipStream_t s) {
    if (!wide_fwd(a)) return launch_fwd<P, 0, BIAS>(a, s);
    return a.heads / a.kv_heads % 2 ? launch_fwd<P, 1, BIAS>(a, s) : launch_fwd<P, 2, BIAS>(a, s);
}
template <class P, bool BIAS>
static hipError_t bwd(const PackedArgs& a, hipStream_t s) {
    hipError_t e;
    if constexpr (BIAS) e = launch_dq<P, false, BIAS>(a, s);
    else e = pair_dq(a) ? launch_dq<P, true, BIAS>(a, s) : launch_dq<P, false, BIAS>(a, s);
    if (e != hipSuccess) return e;
    return launch_dkv<P, BIAS>(a, s);
}
template <int DC>
static hipError_t width(const PackedArgs& a, bool back, hipStream_t s) {
    typedef PackedBf16<DC> P;
    if (back) return a.rel.buckets ? bwd<P, true>(a, s) : bwd<P, false>(a, s);
    return a.rel.buckets ? fwd<P, true>(a, s) : fwd<P, false>(a, s);
}
hipError_t launch_packed_bf16(const PackedArgs& a, bool back, hipStream_t s) {
    return a.d <= 32 ? width<32>(a, back, s) : a.d <= 64 ? width<64>(a, back, s) :
           a.d <= 96 ? width<96>(a, back, s) : width<128>(a, back, s);
}

}  // namespace bp
