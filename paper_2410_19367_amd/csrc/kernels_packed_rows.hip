// Attention over packed sequences, one row per block, in fp32: forward and dQ of one query, dK and dV of one key of a
// group of heads.  Any head width, stride and alignment; nothing but the rows that the row's own sequence lets it see
// is read.  Keys (queries) come in chunks of 256, one to a thread: its scores need the whole of one row, so reads are
// as wide as an element and the time goes by their latency.  For the calls that the matrix-core kernels do not take (forward
// and backward of 11 sequences of 5 to 512 tokens, 12 heads, bf16: width 36 here 1.95 ms, width 40 there 43 us; with a bias of
// 32 buckets and its gradient, 4 key / value heads, 18.4 ms and 66 us).
// A chunk is summed by itself before it joins the sum of all, which would round each of its terms to its own size.
#include "bp_packed.h"
#include "bp_device.h"

namespace bp {

constexpr float kLn2 = 0.6931471805599453f;
constexpr int CHUNK = 256, COLS = kPackedMaxHeadDim / CHUNK;

__device__ __forceinline__ float block_sum(float v, float* red) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}
__device__ __forceinline__ float block_max(float v, float* red) {
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}
template <typename T> __device__ __forceinline__ float dot(const float* x, const T* y, int d) {
    float s = 0.f;
    for (int c = 0; c < d; ++c) s += x[c] * to_float<T>(y[c]);
    return s;
}
__device__ __forceinline__ void load_starts(const RelPos& r, int* start) {
    for (int i = threadIdx.x; i < r.n; i += CHUNK) start[i] = r.start[i];
}
__device__ __forceinline__ float bias_of(const PackedArgs& a, const int* start, int head, int offset) {
    return a.rel.buckets ? packed_bias(a.rel.table[(size_t)packed_bucket(a.rel, start, a.causal, offset) * a.heads + head]) : 0.f;
}

template <typename T>
__global__ __launch_bounds__(CHUNK) void packed_fwd_rows_kernel(PackedArgs a) {
    __shared__ float qs[kPackedMaxHeadDim], p[CHUNK], red[4];
    __shared__ int start[kMaxBuckets];
    const int t = blockIdx.x, head = blockIdx.y, kvh = head / (a.heads / a.kv_heads), tid = threadIdx.x;
    int lo, hi;
    if (!packed_row_range(a, t, lo, hi)) return;
    if (a.causal) hi = t + 1;
    load_starts(a.rel, start);
    const T* q = (const T*)a.q + (size_t)t * a.ld_q + head * a.d;
    for (int c = tid; c < a.d; c += CHUNK) qs[c] = to_float<T>(q[c]);
    __syncthreads();
    const T* kb = (const T*)a.k + kvh * a.d;
    const T* vb = (const T*)a.v + kvh * a.d;
    float m = -INFINITY, l = 0.f, acc[COLS] = {};
    for (int j0 = lo; j0 < hi; j0 += CHUNK) {
        const int n = min(CHUNK, hi - j0), j = j0 + tid;
        float z = -INFINITY;
        if (tid < n) z = dot<T>(qs, kb + (size_t)j * a.ld_k, a.d) * a.scale + bias_of(a, start, head, j - t);
        const float mn = fmaxf(m, block_max(z, red));
        // a chunk of nothing but -inf: no inf - inf
        const float use = mn == -INFINITY ? 0.f : mn, alpha = m == -INFINITY ? 0.f : __expf(m - use);
        const float e = tid < n ? __expf(z - use) : 0.f;
        p[tid] = e;
        l = l * alpha + block_sum(e, red);
        m = mn;
#pragma unroll
        for (int i = 0; i < COLS; ++i) {
            const int c = tid + i * CHUNK;
            if (c >= a.d) break;
            float s = 0.f;
            for (int x = 0; x < n; ++x) s += p[x] * to_float<T>(vb[(size_t)(j0 + x) * a.ld_v + c]);
            acc[i] = acc[i] * alpha + s;
        }
        __syncthreads();
    }
    T* out = (T*)a.ctx + (size_t)t * a.ld_o + head * a.d;
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < COLS; ++i)
        if (tid + i * CHUNK < a.d) out[tid + i * CHUNK] = from_float<T>(acc[i] * inv);
    if (tid == 0) a.lse[(size_t)head * a.T + t] = m + log2f(l) * kLn2;
}

// Each block takes `rows` queries one after the other; with a table gradient these are the rows of one partial.
template <typename T>
__global__ __launch_bounds__(CHUNK) void packed_dq_rows_kernel(PackedArgs a, int rows) {
    __shared__ float qs[kPackedMaxHeadDim], dos[kPackedMaxHeadDim], ds[CHUNK], red[4];
    __shared__ int start[kMaxBuckets];
    const int head = blockIdx.y, kvh = head / (a.heads / a.kv_heads), tid = threadIdx.x;
    const T* kb = (const T*)a.k + kvh * a.d;
    const T* vb = (const T*)a.v + kvh * a.d;
    load_starts(a.rel, start);
    float table = 0.f;                  // gradient of bucket `tid`
    for (int t = blockIdx.x * rows; t < min((int)(blockIdx.x + 1) * rows, a.T); ++t) {
        int lo, hi;
        if (!packed_row_range(a, t, lo, hi)) continue;
        if (a.causal) hi = t + 1;
        const T* q = (const T*)a.q + (size_t)t * a.ld_q + head * a.d;
        const T* o = (const T*)a.ctx + (size_t)t * a.ld_o + head * a.d;
        const T* g = (const T*)a.dctx + (size_t)t * a.ld_o + head * a.d;
        __syncthreads();                // the row before is done with the LDS
        float part = 0.f;
        for (int c = tid; c < a.d; c += CHUNK) {
            qs[c] = to_float<T>(q[c]);
            dos[c] = to_float<T>(g[c]);
            part += dos[c] * to_float<T>(o[c]);
        }
        __syncthreads();
        const float lse = a.lse[(size_t)head * a.T + t];
        auto scores = [&](int j, float& p, float& dp) {
            p = __expf(dot<T>(qs, kb + (size_t)j * a.ld_k, a.d) * a.scale + bias_of(a, start, head, j - t) - lse);
            dp = dot<T>(dos, vb + (size_t)j * a.ld_v, a.d);
        };
        const bool once = hi - lo <= CHUNK;     // a key to a thread: what it has of its pair serves delta and dQ
        float p = 0.f, dp = 0.f;
        if (once && tid < hi - lo) scores(lo + tid, p, dp);
        // delta from the probabilities where the rounding of ctx would be felt: the table's gradient, rows of few keys
        if (a.table_part || (sizeof(T) == 2 && hi - lo <= kShort)) {
            part = once ? p * dp : 0.f;
            for (int j = lo + tid; !once && j < hi; j += CHUNK) {
                scores(j, p, dp);
                part += p * dp;
            }
        }
        const float delta = block_sum(part, red);
        if (tid == 0) a.delta[(size_t)head * a.T + t] = delta;
        float acc[COLS] = {};
        for (int j0 = lo; j0 < hi; j0 += CHUNK) {
            const int n = min(CHUNK, hi - j0);
            if (!once && tid < n) scores(j0 + tid, p, dp);
            ds[tid] = tid < n ? p * (dp - delta) * (hi - lo == 1 ? 0.f : 1.f) : 0.f;    // 0 of one key alone, NaN if it is
            __syncthreads();
#pragma unroll
            for (int i = 0; i < COLS; ++i) {
                const int c = tid + i * CHUNK;
                if (c >= a.d) break;
                float s = 0.f;
                for (int x = 0; x < n; ++x) s += ds[x] * to_float<T>(kb[(size_t)(j0 + x) * a.ld_k + c]);
                acc[i] += s;
            }
            if (a.table_part && tid < a.rel.buckets) {
                float s = 0.f;
                for (int x = 0; x < n; ++x)
                    if (packed_bucket(a.rel, start, a.causal, j0 + x - t) == tid) s += ds[x];
                table += s;
            }
            __syncthreads();
        }
        T* out = (T*)a.dq + (size_t)t * a.ld_q + head * a.d;
#pragma unroll
        for (int i = 0; i < COLS; ++i)
            if (tid + i * CHUNK < a.d) out[tid + i * CHUNK] = from_float<T>(acc[i] * a.scale);
    }
    if (a.table_part && tid < a.rel.buckets) a.table_part[((size_t)blockIdx.x * a.heads + head) * a.rel.buckets + tid] = table;
}

template <typename T>
__global__ __launch_bounds__(CHUNK) void packed_dkv_rows_kernel(PackedArgs a) {
    __shared__ float ks[kPackedMaxHeadDim], vs[kPackedMaxHeadDim], ps[CHUNK], ds[CHUNK];
    __shared__ int start[kMaxBuckets];
    const int t = blockIdx.x, kvh = blockIdx.y, G = a.heads / a.kv_heads, tid = threadIdx.x;
    int lo, hi;
    if (!packed_row_range(a, t, lo, hi)) return;
    const float scale = hi - lo == 1 ? 0.f : a.scale;       // dS of one key alone is 0
    if (a.causal) lo = t;
    load_starts(a.rel, start);
    for (int c = tid; c < a.d; c += CHUNK) {
        ks[c] = to_float<T>(((const T*)a.k)[(size_t)t * a.ld_k + kvh * a.d + c]);
        vs[c] = to_float<T>(((const T*)a.v)[(size_t)t * a.ld_v + kvh * a.d + c]);
    }
    __syncthreads();
    float dk[COLS] = {}, dv[COLS] = {};
    for (int head = kvh * G; head < kvh * G + G; ++head) {
        const T* qb = (const T*)a.q + head * a.d;
        const T* gb = (const T*)a.dctx + head * a.d;
        const size_t stat = (size_t)head * a.T;
        for (int i0 = lo; i0 < hi; i0 += CHUNK) {
            const int n = min(CHUNK, hi - i0), i = i0 + tid;
            if (tid < n) {
                const float z = dot<T>(ks, qb + (size_t)i * a.ld_q, a.d) * a.scale + bias_of(a, start, head, t - i);
                const float p = __expf(z - a.lse[stat + i]);
                ps[tid] = p;
                ds[tid] = p * (dot<T>(vs, gb + (size_t)i * a.ld_o, a.d) - a.delta[stat + i]);
            }
            __syncthreads();
#pragma unroll
            for (int x = 0; x < COLS; ++x) {
                const int c = tid + x * CHUNK;
                if (c >= a.d) break;
                float sv = 0.f, sk = 0.f;
                for (int y = 0; y < n; ++y) {
                    sv += ps[y] * to_float<T>(gb[(size_t)(i0 + y) * a.ld_o + c]);
                    sk += ds[y] * to_float<T>(qb[(size_t)(i0 + y) * a.ld_q + c]);
                }
                dv[x] += sv;
                dk[x] += sk;
            }
            __syncthreads();
        }
    }
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
        const int c = tid + x * CHUNK;
        if (c >= a.d) break;
        ((T*)a.dk)[(size_t)t * a.ld_k + kvh * a.d + c] = from_float<T>(dk[x] * scale);
        ((T*)a.dv)[(size_t)t * a.ld_v + kvh * a.d + c] = from_float<T>(dv[x]);
    }
}

__global__ __launch_bounds__(256) void packed_table_grad_kernel(PackedArgs a) {
    __shared__ float sums[256];
    sum_table_part(a, blockIdx.x, sums);
}

template <typename T>
static hipError_t bwd_rows(const PackedArgs& a, hipStream_t s) {
    const int rows = a.table_part ? kPackedTile : 1;
    hipLaunchKernelGGL((packed_dq_rows_kernel<T>), dim3((a.T + rows - 1) / rows, a.heads), dim3(CHUNK), 0, s, a, rows);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((packed_dkv_rows_kernel<T>), dim3(a.T, a.kv_heads), dim3(CHUNK), 0, s, a);
    if (a.table_part) hipLaunchKernelGGL(packed_table_grad_kernel, dim3(a.heads), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_packed_fwd_rows(int dtype, const PackedArgs& a, hipStream_t s) {
    if (dtype) hipLaunchKernelGGL((packed_fwd_rows_kernel<bf16_t>), dim3(a.T, a.heads), dim3(CHUNK), 0, s, a);
    else hipLaunchKernelGGL((packed_fwd_rows_kernel<float>), dim3(a.T, a.heads), dim3(CHUNK), 0, s, a);
    return hipGetLastError();
}
hipError_t launch_packed_bwd_rows(int dtype, const PackedArgs& a, hipStream_t s) {
    return dtype ? bwd_rows<bf16_t>(a, s) : bwd_rows<float>(a, s);
}

}  // namespace bp
