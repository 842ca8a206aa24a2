"""GPU: attention over packed sequences where a row holds what is not finite or sees nothing, where a bucket of the bias is far
from every score, against a 64-bit form that takes visible pairs only; the precision of the kernels of one row a block; and sequences of thousands of tokens."""
import numpy as np
import pytest

import synth_inputs as si
from oracle import packed_oracle as po
from tests.test_gpu_packed import UNIT, Call

pytestmark = pytest.mark.gpu


def by_rows(c):
    """The definition row by row in fp64, in the layout of po.attention: nothing is made of a pair that is not visible, so
    what is not finite in the result depends on what is not finite in the inputs.  abs_*: sums of absolute terms."""
    G = c.H // c.Hk
    shapes = dict(ctx=c.q.shape, lse=(c.H, c.T), dq=c.q.shape, dk=c.k.shape, dv=c.v.shape)
    r = {p + n: np.zeros(s) for n, s in shapes.items() for p in ("", "abs_")}
    if c.table is not None:
        r |= {"dtable": np.zeros(c.table.shape), "abs_dtable": np.zeros(c.table.shape)}
    bucket = {}
    z_most = 0.0
    with np.errstate(all="ignore"):
        for s0, s1 in zip(c.starts[:-1], c.starts[1:]):
            for i in range(s0, s1):
                js = np.arange(s0, i + 1 if c.causal else s1)
                if c.table is not None:
                    of = js - i
                    for o in of:
                        if o not in bucket:
                            bucket[o] = po.bucket(c.causal, len(c.table), c.far, int(o))
                    b = np.array([bucket[o] for o in of])
                for h in range(c.H):
                    K, V, g = c.k[js, h // G], c.v[js, h // G], c.g[i, h]
                    z, zabs = c.scale * (K @ c.q[i, h]), c.scale * (np.abs(K) @ np.abs(c.q[i, h]))
                    if np.isfinite(zabs).all():
                        z_most = max(z_most, float(zabs.max()))
                    if c.table is not None:
                        z = z + np.where(c.table[b, h] <= -1e30, -np.inf, c.table[b, h])
                    top = z.max()
                    e = np.exp(z - top)
                    p = e / e.sum()
                    dp, dpa = V @ g, np.abs(V) @ np.abs(g)
                    ds = p * (dp - (p * dp).sum())
                    dsa = p * (dpa + (p * dpa).sum())
                    r["lse"][h, i] = top + np.log(e.sum())
                    r["ctx"][i, h], r["abs_ctx"][i, h] = p @ V, p @ np.abs(V)
                    r["dq"][i, h], r["abs_dq"][i, h] = c.scale * (ds @ K), c.scale * (dsa @ np.abs(K))
                    r["dk"][js, h // G] += c.scale * ds[:, None] * c.q[i, h]
                    r["abs_dk"][js, h // G] += c.scale * dsa[:, None] * np.abs(c.q[i, h])
                    r["dv"][js, h // G] += p[:, None] * g
                    r["abs_dv"][js, h // G] += p[:, None] * np.abs(g)
                    if c.table is not None:
                        np.add.at(r["dtable"][:, h], b, ds)
                        np.add.at(r["abs_dtable"][:, h], b, dsa)
    r["abs_lse"] = np.abs(r["lse"])
    r["z"] = z_most
    return r


def check(c, got, r):
    """Finite where the definition is, within the bounds, and not where it is not (lse of a row that sees nothing is -inf)."""
    with np.errstate(all="ignore"):
        tol = po.bounds(r, c.longest, c.d, c.H // c.Hk, UNIT[c.dtype])
    for name, a in got.items():
        ref, t = r[name], tol[name] * np.ones_like(r[name])
        if name != "dtable":
            rows = slice(c.starts[0], c.starts[-1])
            a, ref, t = (x[:, rows] if name == "lse" else x[rows] for x in (a, ref, t))
        if name in ("dq", "dk") and c.dtype == "bf16":
            t = 2.0 * t                         # ctx's rounding in delta, as in Call.check
        fine = np.isfinite(ref)
        assert not np.isfinite(a[~fine]).any(), (name, "finite where the definition is not")
        assert np.isfinite(a[fine]).all(), (name, np.argwhere(fine & ~np.isfinite(a))[:8].tolist())
        if fine.any():
            off = np.abs(a[fine] - ref[fine]) / (t[fine] + 1e-30)
            assert off.max() <= 1.0, (name, float(off.max()))


# head width and shift of the pointers: the matrix-core kernels and the row kernels
KERNELS = [(64, 0), (128, 0), (64, 1)]


@pytest.mark.parametrize("d,shift", KERNELS)
@pytest.mark.parametrize("lens,causal,at", [([40, 24], True, 50), ([24, 40], True, 20), ([300, 3], True, 301), ([2, 300, 60], True, 30),
                                            ([40, 24], False, 50), ([300, 3], False, 301)])
@pytest.mark.parametrize("where", ["q", "g", "k", "v"])
@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_table_gradient_takes_nothing_from_pairs_that_are_not_visible(dtype, value, where, lens, causal, at, d, shift):
    """NaN or infinity in a row inside a sequence reaches the buckets of the distances that its queries see, in its heads, and no others."""
    c = Call(lens, 4, 2, d, causal, dtype, front=3, back=5, buckets=16, far=40, shift=shift)
    getattr(c, where)[c.starts[0] + at, 1, 3] = value
    for x in (c.q, c.k, c.v, c.g):
        x[:3] = np.nan
        x[c.starts[-1]:] = np.nan
    r = by_rows(c)
    assert np.isnan(r["dtable"]).any() and np.isfinite(r["dtable"]).any()
    check(c, c.run(), r)


@pytest.mark.parametrize("d,shift", KERNELS)
@pytest.mark.parametrize("low", [-np.inf, -3.0e38, -1.0e31])
@pytest.mark.parametrize("buckets,causal", [([0], True), ([0, 1, 2], True), ([0, 1, 9], False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_query_that_sees_nothing_is_nan_and_reaches_its_own_keys_only(dtype, buckets, causal, low, d, shift):
    """Buckets taken out of one head leave the first rows of its sequences (without a mask: sequences of one and two rows)
    nothing to look at."""
    c = Call([70, 1, 2, 150, 30], 4, 2, d, causal, dtype, front=2, back=3, buckets=16, far=40, shift=shift)
    c.table[buckets, 1] = low
    r = by_rows(c)
    assert np.isnan(r["ctx"][:, 1]).any() and np.isfinite(r["ctx"][:, [0, 2, 3]]).all()
    check(c, c.run(), r)


@pytest.mark.parametrize("d,shift", KERNELS)
@pytest.mark.parametrize("value", [-1e9, -1e12, -1e20, -3.0e38, 1e12])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bucket_far_from_all_scores(dtype, causal, value, d, shift):
    """Scores of hundreds, and a bucket whose bias is far below (or above) them: it takes no probability (or all of it, spread
    evenly where the bias rounds the scores away).  Far pieces, which a row meets first, lie in this bucket."""
    c = Call([400, 90], 2, 1, d, causal, dtype, back=2, buckets=16, far=40, std=8.0, shift=shift)
    c.table[[7, 15] if not causal else [15]] = value
    if value > 0:                               # only that the result is finite and an average of what the bucket holds
        got = c.run(backward=False)
        assert np.isfinite(got["ctx"][:c.starts[-1]]).all()
        assert np.abs(got["ctx"][:c.starts[-1]]).max() <= np.abs(c.v).max() * (1 + 2 ** -7)
        return
    r = by_rows(c)
    assert r["z"] > 300
    check(c, c.run(), r)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,shift", [(64, 1), (40, 1), (7, 0), (136, 0)])
def test_row_kernels_short_sequences(causal, d, shift):
    """delta of rows with few keys does not come from the rounded ctx in the kernels of one row a block either.  These keep
    probabilities and score gradients in fp32, so the rounding of dQ and dK itself is all, and a tenth for all else."""
    c = Call([20, 30, 9, 25, 14, 200], 8, 2, d, causal, "bf16", shift=shift)
    got, r = c.run(), c.reference()
    for name in ("dq", "dk"):
        one = np.linalg.norm(si.round_bf16(r[name]) - r[name])
        assert np.linalg.norm(got[name] - r[name]) <= 1.1 * one, (name, np.linalg.norm(got[name] - r[name]) / one)


def test_row_kernels_long_sums():
    """Equal terms by the ten thousand: the sums of a chunk of 256 are joined, not every term added to the whole, whose
    rounding would have the same sign each time.  A term goes through at most 256 additions of its chunk, those of the chunks
    of its row (of its 64 rows for the table's gradient) and of its heads, and of the tiles: terms * 2^-24 of the sum of
    absolute terms bounds their roundings, `share` is what the probabilities are off by (oracle/packed_oracle.py)."""
    n, H, Hk, d, far = 4000, 4, 1, 7, 40
    c = Call([n], H, Hk, d, False, "f32", buckets=8, far=far)
    c.q[:], c.k[:], c.g[:], c.table[:] = 0.05, 0.01, 0.3, 0.0
    c.v[:] = 0.7 * (1 + (np.arange(n) % 2 == 0)[:, None, None] * 0.01)
    c.v[::100] = 5.0
    got, r = c.run(), c.reference()
    f = 2.0 ** -24
    chunks = -(-n // 256)
    share = 2.0 * (d + 16) * f * (1.0 + r["z"])
    terms = {"ctx": 256 + chunks, "dq": 256 + chunks, "dk": 256 + chunks * H, "dv": 256 + chunks * H,
             "dtable": 256 + 64 * chunks + 64}
    for name, t in terms.items():
        bound = r["abs_" + name] * (share + (t + 2 * d + 64) * f)
        off = np.max(np.abs(got[name] - r[name]) / (bound + 1e-30))
        assert off <= 1.0, (name, float(off))


def in_64_bits(c):
    """po.attention's dict from whole matrices in fp64 on the GPU, a head at a time (finite inputs).  A value of the table beyond
    1e6 takes no part in "z": pairs that have it have no probability."""
    import torch
    dev = dict(dtype=torch.float64, device="cuda")
    q, k, v, g = (torch.tensor(x, **dev) for x in (c.q, c.k, c.v, c.g))
    G = c.H // c.Hk
    r = {n: torch.zeros(s, **dev) for n, s in (("ctx", c.q.shape), ("lse", (c.H, c.T)), ("dq", c.q.shape), ("dk", c.k.shape), ("dv", c.v.shape))}
    r |= {"abs_" + n: torch.zeros_like(t) for n, t in r.items()}
    if c.table is not None:
        table = torch.tensor(c.table, **dev)
        size = torch.where(table.abs() < 1e6, table.abs(), 0.0)
        r |= {"dtable": torch.zeros_like(table), "abs_dtable": torch.zeros_like(table)}
    z_most = 0.0
    for s0, s1 in zip(c.starts[:-1], c.starts[1:]):
        n, R = s1 - s0, slice(s0, s1)
        if not n:
            continue
        at = torch.arange(n, device="cuda")
        offset = at[None] - at[:, None]
        later = offset > 0
        if c.table is not None:
            by_offset = torch.tensor([po.bucket(c.causal, len(c.table), c.far, o) if not (c.causal and o > 0) else 0
                                      for o in range(1 - n, n)], device="cuda")
            of = by_offset[offset + n - 1]
        for h in range(c.H):
            Q, K, V, D = q[R, h], k[R, h // G], v[R, h // G], g[R, h]
            z, zabs = c.scale * (Q @ K.t()), c.scale * (Q.abs() @ K.abs().t())
            if c.table is not None:
                z, zabs = z + table[:, h][of], zabs + size[:, h][of]
            if c.causal:
                z, zabs = z.masked_fill(later, -float("inf")), zabs.masked_fill(later, 0.0)
            z_most = max(z_most, float(zabs.max()))
            r["lse"][h, R] = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            dp, dpa = D @ V.t(), D.abs() @ V.abs().t()
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            dsa = p * (dpa + (p * dpa).sum(1, keepdim=True))
            r["ctx"][R, h], r["abs_ctx"][R, h] = p @ V, p @ V.abs()
            r["dq"][R, h], r["abs_dq"][R, h] = c.scale * (ds @ K), c.scale * (dsa @ K.abs())
            r["dk"][R, h // G] += c.scale * (ds.t() @ Q)
            r["abs_dk"][R, h // G] += c.scale * (dsa.t() @ Q.abs())
            r["dv"][R, h // G] += p.t() @ D
            r["abs_dv"][R, h // G] += p.t() @ D.abs()
            if c.table is not None:
                for name, x in (("dtable", ds), ("abs_dtable", dsa)):       # along the diagonals first: each row moved on by one
                    x = torch.nn.functional.pad(x.flip(0), (0, n)).flatten()[:-n].view(n, 2 * n - 1).sum(0)
                    r[name][:, h].index_add_(0, by_offset, x)
    r["abs_lse"] = r["lse"].abs()
    return {n: t.cpu().numpy() for n, t in r.items()} | {"z": z_most}


# Sequences of thousands of tokens: far pieces of one bucket, borders of buckets far from the diagonal, hundreds of steps;
# few blocks, blocks of two heads, of 128 rows
@pytest.mark.parametrize("lens,H,Hk,d,causal", [([2900, 37, 1200], 4, 2, 128, True), ([5091], 2, 1, 64, False), ([17, 4100], 32, 8, 64, True),
                                                ([2500, 2500], 16, 16, 128, True)])
@pytest.mark.parametrize("buckets,far", [(0, 0), (32, 128), (64, 3000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_long_sequences(dtype, buckets, far, lens, H, Hk, d, causal):
    if dtype == "f32":
        H, Hk = H // Hk, 1
    c = Call(lens, H, Hk, d, causal, dtype, front=1, back=6, buckets=buckets, far=far, fused=True)
    c.check(c.run(), in_64_bits(c))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_row_kernels_long_sequences(dtype):
    c = Call([1700, 33], 2, 1, 20, True, dtype, front=1, back=2, buckets=32, far=500, shift=1)
    c.check(c.run(), in_64_bits(c))


@pytest.mark.parametrize("H,Hk,d", [(32, 8, 64), (33, 11, 64), (16, 8, 128)])
def test_bucket_far_from_all_scores_in_wide_blocks(H, Hk, d):
    """The same in launches of blocks of two heads and of 128 rows."""
    c = Call([2100, 70, 2000], H, Hk, d, True, "bf16", back=2, buckets=16, far=40, std=8.0)
    c.table[15] = -1e12
    c.check(c.run(), in_64_bits(c))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_gradient_of_a_row_does_not_depend_on_what_lies_behind_it(d, causal):
    """How delta of a bf16 row is found depends on its own number of keys: with the forward's results given, dQ of a sequence
    has the same bits with and without a short sequence behind it in its last block, which holds rows of 217 to 270 keys."""
    import torch
    import paper_2410_19367_amd as bp
    H, Hk, front, n, more = 4, 2, 40, 270, 10
    c = Call([n, more], H, Hk, d, causal, "bf16", front=front)
    end = front + n
    q, k, v, g = (torch.tensor(x.reshape(end + more, -1), dtype=torch.bfloat16, device="cuda") for x in (c.q, c.k, c.v, c.g))
    ctx, lse, seen = torch.zeros_like(q), torch.zeros((H, end + more), device="cuda"), []
    bp.bp_op_attention_packed_fwd(c.dt, bp.bp_packed(end + more, 2, c.starts_dev, H, Hk, d, causal), q, k, v, ctx, lse)
    for sequences, T in ((2, end + more), (1, end + more), (1, end)):       # the short sequence, rows of none, nothing
        layout = bp.bp_packed(T, sequences, c.starts_dev, H, Hk, d, causal)
        a = [t[:T] for t in (q, k, v, ctx)]
        dq, dk, dv = (torch.zeros_like(t) for t in a[:3])
        ws = torch.zeros(bp.bp_op_attention_packed_workspace(c.dt, layout), device="cuda")
        bp.bp_op_attention_packed_bwd(c.dt, layout, *a, lse[:, :T].contiguous(), g[:T], dq, dk, dv, ws)
        seen.append(dq[front:end])
    torch.cuda.synchronize()
    assert torch.equal(seen[0], seen[1]) and torch.equal(seen[0], seen[2])


@pytest.mark.parametrize("d,shift", KERNELS)
@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("lens,causal", [([100, 30], True), ([20, 100, 17], False), ([300, 20, 60], True), ([20, 300], False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bucket_that_is_not_finite_reaches_queries_that_see_it(dtype, lens, causal, value, d, shift):
    """Sequences too short for the far bucket keep their results, also where they share a block with one that has it."""
    c = Call(lens, 4, 2, d, causal, dtype, front=3, back=5, buckets=16, far=40, shift=shift)
    c.table[[15] if causal else [7, 15], 1] = value
    r = by_rows(c)
    assert np.isnan(r["ctx"][:, 1]).any() and np.isfinite(r["ctx"][:, [0, 2, 3]]).all()
    assert any(np.isfinite(r["dq"][s0:s1]).all() for s0, s1 in zip(c.starts[:-1], c.starts[1:]))
    check(c, c.run(), r)
