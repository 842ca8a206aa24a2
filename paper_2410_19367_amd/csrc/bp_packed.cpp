// C ABI of the attention over packed sequences: argument checks, the borders of the position buckets, and which
// kernels take a call.
#include <math.h>

#include "bp_host.h"
#include "bp_packed.h"

using bp::fail;

namespace bp {
namespace {

// Whole numbers of up to 256 * 32 bits: x^m e^k with factors below 2^24 and m + k below 256 has fewer.
struct Wide {
    uint32_t w[256] = {1};
    int n = 1;
    void times(uint32_t f, int count) {
        for (; count > 0; --count) {
            uint64_t carry = 0;
            for (int i = 0; i < n; ++i) {
                carry += (uint64_t)w[i] * f;
                w[i] = (uint32_t)carry;
                carry >>= 32;
            }
            if (carry) w[n++] = (uint32_t)carry;
        }
    }
    bool at_least(const Wide& o) const {
        if (n != o.n) return n > o.n;
        for (int i = n - 1; i >= 0; --i)
            if (w[i] != o.w[i]) return w[i] > o.w[i];
        return true;
    }
};

// Smallest whole x with x >= e (far / e)^(k / m).  Where the value in 64 bits is next to a whole number the powers decide,
// so that a distance on a border belongs to the bucket that begins there.
int border(int e, int far, int k, int m) {
    const double y = e * exp(log((double)far / e) * k / m), r = nearbyint(y);
    if (fabs(y - r) > 1e-11 * y) return (int)ceil(y);
    Wide a, b;
    a.times((uint32_t)r, m); a.times((uint32_t)e, k);
    b.times((uint32_t)far, k); b.times((uint32_t)e, m);
    return a.at_least(b) ? (int)r : (int)r + 1;
}

int make_relpos(int causal, int buckets, int max_distance, RelPos& r) {
    const int n = causal ? buckets : buckets / 2, e = n / 2;
    if (buckets > kMaxBuckets || n < 2 || (!causal && buckets % 2))
        return fail(BP_EINVAL, "buckets = %d: with a causal mask 2 .. %d, else even and 4 .. %d", buckets, kMaxBuckets, kMaxBuckets);
    if (max_distance <= e || max_distance >= 1 << 24)
        return fail(BP_EINVAL, "max_distance = %d must be above %d (buckets of one distance) and below 2^24", max_distance, e);
    r.buckets = buckets; r.n = n; r.exact = e;
    for (int i = 0; i < e; ++i) r.start[i] = i;
    for (int i = e; i < n; ++i) r.start[i] = border(e, max_distance, i - e, n - e);
    r.far = r.start[n - 1];
    r.log2_exact = (float)log2((double)e);
    r.per_octave = (float)((n - e) / log2((double)max_distance / e));
    return BP_OK;
}

int dense(int ld, int heads, int d) { return ld ? ld : heads * d; }

// everything about the layout and the bias; pointers of the tensors are the callers' business
int make_args(int dtype, const bp_packed* p, const bp_relpos* bias, PackedArgs& a) {
    if (dtype != BP_F32 && dtype != BP_BF16) return fail(BP_EINVAL, "unknown dtype %d", dtype);
    if (!p) return fail(BP_EINVAL, "null layout");
    if (!p->starts) return fail(BP_EINVAL, "null starts");
    if (p->tokens <= 0 || p->sequences <= 0 || p->heads <= 0 || p->kv_heads <= 0 || p->head_dim <= 0)
        return fail(BP_EINVAL, "tokens, sequences, heads, kv_heads, head_dim must be positive");
    if (p->heads % p->kv_heads) return fail(BP_EINVAL, "%d heads cannot share %d key/value heads evenly", p->heads, p->kv_heads);
    if (!(p->scale >= 0.f) || isinf(p->scale)) return fail(BP_EINVAL, "scale must be positive and finite, or 0");
    // (the kernels count starts in 32 bits, and one wave may have to look at all that share a row)
    if (p->sequences >= 1 << 24) return fail(BP_ESHAPE, "sequences = %d must be below 2^24", p->sequences);
    if (p->tokens >= 1 << 24) return fail(BP_ESHAPE, "tokens = %d must be below 2^24", p->tokens);
    if (p->head_dim > kPackedMaxHeadDim) return fail(BP_ESHAPE, "head_dim = %d must be at most %d", p->head_dim, kPackedMaxHeadDim);
    if (p->heads > 65535 / 8) return fail(BP_ESHAPE, "heads = %d must be at most %d", p->heads, 65535 / 8);
    a.T = p->tokens; a.n_seq = p->sequences; a.heads = p->heads; a.kv_heads = p->kv_heads; a.d = p->head_dim;
    a.causal = p->causal != 0;
    a.starts = p->starts;
    a.scale = p->scale > 0.f ? p->scale : 1.f / sqrtf((float)p->head_dim);
    a.ld_q = dense(p->ld_q, a.heads, a.d);
    a.ld_k = dense(p->ld_k, a.kv_heads, a.d);
    a.ld_v = dense(p->ld_v, a.kv_heads, a.d);
    a.ld_o = dense(p->ld_ctx, a.heads, a.d);
    if (a.ld_q < a.heads * a.d || a.ld_o < a.heads * a.d || a.ld_k < a.kv_heads * a.d || a.ld_v < a.kv_heads * a.d)
        return fail(BP_EINVAL, "leading dimension smaller than the row length");
    if (a.ld_q >= 1 << 24 || a.ld_k >= 1 << 24 || a.ld_v >= 1 << 24 || a.ld_o >= 1 << 24)
        return fail(BP_ESHAPE, "leading dimensions must be below 2^24");
    // A launch of the kernels of 64 rows has up to this many blocks of 256 threads, and fewer than 2^32 threads: forward and dQ
    // a block for each tile and head, dK/dV for each tile and part of the heads.  (One row a block: tokens below 2^24 keep the
    // grid's first dimension there, heads are its second; the joined sums' launch: see launch_dkv.)
    if ((int64_t)packed_tiles(a.T) * a.heads >= 1 << 24)
        return fail(BP_ESHAPE, "%d tokens of %d heads: (tokens + 63) / 64 * heads must be below 2^24", a.T, a.heads);
    if (bias) {
        if (!bias->table) return fail(BP_EINVAL, "null bias table");
        const int rc = make_relpos(a.causal, bias->buckets, bias->max_distance, a.rel);
        if (rc) return rc;
        a.rel.table = bias->table;
    }
    return BP_OK;
}

// What the kernels on the matrix cores take: heads whose rows are whole 16-byte pieces and fit a tile, and tiles of 64 rows
// within the 2 GiB that an offset into them may have.
bool on_matrix_cores(int dtype, const PackedArgs& a) {
    const int e = dtype == BP_BF16 ? 2 : 4;
    if (a.d % 8 || a.d > 128) return false;
    for (int ld : {a.ld_q, a.ld_k, a.ld_v, a.ld_o})
        if (ld * e % 16 || (int64_t)ld * e * 64 > (int64_t)1 << 31) return false;
    for (const void* p : {a.q, a.k, a.v, (const void*)a.ctx, a.dctx, (const void*)a.dq, (const void*)a.dk, (const void*)a.dv})
        if ((uintptr_t)p & 15) return false;
    return true;
}
hipError_t launch(int dtype, const PackedArgs& a, bool back, hipStream_t s) {
    if (on_matrix_cores(dtype, a)) return dtype == BP_BF16 ? launch_packed_bf16(a, back, s) : launch_packed_f32(a, back, s);
    return back ? launch_packed_bwd_rows(dtype, a, s) : launch_packed_fwd_rows(dtype, a, s);
}

// floats of the backward's workspace: delta, the partials of the table's gradient, and sums of dK and dV, which a call can
// do without
size_t delta_floats(const PackedArgs& a) { return ((size_t)a.heads * a.T + 3) & ~(size_t)3; }
size_t needed_floats(const PackedArgs& a) {
    return delta_floats(a) + (((size_t)packed_tiles(a.T) * a.heads * a.rel.buckets + 3) & ~(size_t)3);
}
size_t part_floats(const PackedArgs& a, int splits) {
    return splits > 1 ? (size_t)splits * a.T * a.kv_heads * 2 * a.d : 0;
}

}  // namespace
}  // namespace bp

extern "C" {

int bp_relpos_bucket(int causal, int buckets, int max_distance, int offset) {
    bp::RelPos r;
    const int rc = bp::make_relpos(causal, buckets, max_distance, r);
    if (rc) return rc;
    if (causal && offset > 0) return fail(BP_EINVAL, "offset %d: a causal query sees no later key", offset);
    const int64_t dist = offset < 0 ? -(int64_t)offset : offset;
    int b = r.n - 1;
    while (r.start[b] > dist) --b;
    return b + (offset > 0 ? r.n : 0);
}

int bp_op_attention_packed_fwd(int dtype, const bp_packed* layout, const bp_relpos* bias, const void* q, const void* k,
                               const void* v, void* ctx, float* lse, void* stream) {
    bp::PackedArgs a{};
    const int rc = bp::make_args(dtype, layout, bias, a);
    if (rc) return rc;
    if (!q || !k || !v || !ctx || !lse) return fail(BP_EINVAL, "null pointer");
    a.q = q; a.k = k; a.v = v; a.ctx = ctx; a.lse = lse;
    const hipError_t e = bp::launch(dtype, a, false, (hipStream_t)stream);
    if (e != hipSuccess) return fail(BP_EHIP, "packed attention forward: %s", hipGetErrorString(e));
    return BP_OK;
}

size_t bp_op_attention_packed_workspace(int dtype, const bp_packed* layout, const bp_relpos* bias) {
    bp::PackedArgs a{};
    if (bp::make_args(dtype, layout, bias, a)) return 0;
    return bp::needed_floats(a) + bp::part_floats(a, bp::split_heads(a, bp::cu_count()));
}

int bp_op_attention_packed_bwd(int dtype, const bp_packed* layout, const bp_relpos* bias, const void* q, const void* k,
                               const void* v, const void* ctx, const float* lse, const void* dctx, void* dq, void* dk,
                               void* dv, float* dtable, int overwrite, float* workspace, size_t workspace_elems,
                               void* stream) {
    bp::PackedArgs a{};
    const int rc = bp::make_args(dtype, layout, bias, a);
    if (rc) return rc;
    if (!q || !k || !v || !ctx || !lse || !dctx || !dq || !dk || !dv || !workspace) return fail(BP_EINVAL, "null pointer");
    if (dtable && !bias) return fail(BP_EINVAL, "the gradient of a bias table without a bias");
    if (workspace_elems < bp::needed_floats(a))
        return fail(BP_EINVAL, "workspace of %zu floats, %zu needed", workspace_elems, bp::needed_floats(a));
    if ((uintptr_t)workspace & 15) return fail(BP_EINVAL, "workspace must be aligned to 16 bytes");
    a.q = q; a.k = k; a.v = v; a.ctx = (void*)ctx; a.lse = (float*)lse;
    a.dctx = dctx; a.dq = dq; a.dk = dk; a.dv = dv;
    a.delta = workspace;
    a.table_part = dtable ? workspace + bp::delta_floats(a) : nullptr;
    a.dtable = dtable;
    a.overwrite = overwrite != 0;
    a.dkv_part = workspace + bp::needed_floats(a);
    a.splits = bp::split_heads(a, bp::cu_count());
    if (workspace_elems < bp::needed_floats(a) + bp::part_floats(a, a.splits)) a.splits = 1;
    const hipError_t e = bp::launch(dtype, a, true, (hipStream_t)stream);
    if (e != hipSuccess) return fail(BP_EHIP, "packed attention backward: %s", hipGetErrorString(e));
    return BP_OK;
}

}  // extern "C"
