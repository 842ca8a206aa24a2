"""Attention over packed sequences with grouped heads and a relative position bias by buckets, from the definition in
fp64 numpy, one sequence and one head at a time; and how far a result may be off when products take rounded factors.
Test infrastructure: nothing here is shared with the HIP path."""
from __future__ import annotations

import math

import numpy as np


def bucket(causal, buckets, max_distance, offset):
    """Bucket of key position minus query position, in whole numbers: bucket e + m of a direction begins at the smallest
    distance x with (x / e)^(n - e) >= (max_distance / e)^m."""
    n = buckets if causal else buckets // 2
    e, dist, first = n // 2, abs(offset), n if offset > 0 else 0
    if dist < e:
        return first + dist
    b = e
    while b + 1 < n:
        m = b + 1 - e
        if dist ** (n - e) * e ** m < max_distance ** m * e ** (n - e):
            break
        b += 1
    return first + b


def bucket_matrix(n, causal, buckets, max_distance):
    """[n, n] buckets of (query, key); where a causal query does not look, bucket 0."""
    row = {o: bucket(causal, buckets, max_distance, o) for o in range(-n + 1, 1 if causal else n)}
    return np.array([[row.get(j - i, 0) for j in range(n)] for i in range(n)], dtype=np.int64).reshape(n, n)


def attention(starts, q, k, v, causal, scale, table=None, max_distance=0, dctx=None, ctx_given=None):
    """q [T, heads, d], k and v [T, kv_heads, d], table [buckets, heads].  Returns a dict: ctx, lse [heads, T] and with
    dctx the gradients dq, dk, dv, dtable; and under the same names with "abs_" the sums of the absolute values of what
    each element is a sum of, for bounds.  ctx_given: delta from this ctx (as a caller hands it to a backward pass) in
    place of the exact one.  Rows of no sequence stay NaN."""
    T, H, d = q.shape
    G = H // k.shape[1]
    names = [("ctx", q.shape), ("lse", (H, T))]
    if dctx is not None:
        names += [("dq", q.shape), ("dk", k.shape), ("dv", v.shape)]
    r = {n: np.full(s, np.nan) for n, s in names}
    r |= {"abs_" + n: np.full(s, np.nan) for n, s in names}
    r["z"] = 0.0                                    # largest sum of absolute terms of a score
    if table is not None:
        r["dtable"], r["abs_dtable"] = np.zeros(table.shape), np.zeros(table.shape)
    for s0, s1 in zip(starts[:-1], starts[1:]):
        n = s1 - s0
        if n <= 0:
            continue
        R = slice(s0, s1)
        if dctx is not None:
            for name in ("dk", "dv"):
                r[name][R] = 0.0
                r["abs_" + name][R] = 0.0
        ok = np.tril(np.ones((n, n), bool)) if causal else np.ones((n, n), bool)
        if table is not None:
            bk = bucket_matrix(n, causal, table.shape[0], max_distance)
        for h in range(H):
            Q, K, V = q[R, h], k[R, h // G], v[R, h // G]
            z = scale * (Q @ K.T)
            zabs = scale * (np.abs(Q) @ np.abs(K).T)
            if table is not None:
                z = z + table[bk, h]
                zabs = zabs + np.abs(table[bk, h])
            r["z"] = max(r["z"], float(np.max(zabs[ok])))
            z = np.where(ok, z, -np.inf)
            top = z.max(1, keepdims=True)
            e = np.exp(z - top)
            p = e / e.sum(1, keepdims=True)
            r["lse"][h, R] = (top + np.log(e.sum(1, keepdims=True)))[:, 0]
            r["abs_lse"][h, R] = np.abs(r["lse"][h, R])
            r["ctx"][R, h], r["abs_ctx"][R, h] = p @ V, p @ np.abs(V)
            if dctx is None:
                continue
            D = dctx[R, h]
            dp, dpa = D @ V.T, np.abs(D) @ np.abs(V).T
            delta = (p * dp).sum(1, keepdims=True)
            if ctx_given is not None:
                delta = (D * ctx_given[R, h]).sum(1, keepdims=True)
            ds = p * (dp - delta)
            dsa = p * (dpa + (p * dpa).sum(1, keepdims=True))
            r["dq"][R, h], r["abs_dq"][R, h] = scale * (ds @ K), scale * (dsa @ np.abs(K))
            r["dk"][R, h // G] += scale * (ds.T @ Q)
            r["abs_dk"][R, h // G] += scale * (dsa.T @ np.abs(Q))
            r["dv"][R, h // G] += p.T @ D
            r["abs_dv"][R, h // G] += p.T @ np.abs(D)
            if table is not None:
                np.add.at(r["dtable"][:, h], bk[ok], ds[ok])
                np.add.at(r["abs_dtable"][:, h], bk[ok], dsa[ok])
    return r


def bounds(r, longest, d, heads_per_kv, u):
    """Elementwise bounds on |result - exact| for inputs that are exact in a type of unit roundoff u (2^-8 bf16, 2^-24 fp32):
      products of sums    the factor that is an intermediate (p, ds) is rounded once: u times the sum of absolute terms;
      results             rounded once: u times the value (ctx, dq, dk, dv);
      fp32 arithmetic     sums of `terms` values: at most terms * 2^-24 of the sum of absolute terms;
      probabilities       a score and its log-sum-exp are each off by up to (d + 8) * 2^-24 of the largest sum of absolute
                          terms of a score, and four roundings of numbers of that size go into the change of base: p is off
                          by that share, twice (score, normaliser), and so is everything made of it.
    With u = 2^-24 the first two vanish in the third."""
    f = 2.0 ** -24
    share = 2.0 * (d + 16) * f * (1.0 + r["z"])
    out = {}
    for name in ("ctx", "dq", "dk", "dv"):
        if name not in r:
            continue
        terms = longest * (heads_per_kv if name in ("dk", "dv") else 1) + 2 * d + 64
        out[name] = r["abs_" + name] * (u + share + terms * f) + np.abs(r[name]) * u
    out["lse"] = share / 2 + (longest + 8) * f + r["abs_lse"] * 4 * f
    if "dtable" in r:
        # a rounding stays inside the kernel's fp32: sums over keys, then over rows of a tile, then over tiles
        out["dtable"] = r["abs_dtable"] * (share + (2 * longest + 2 * d + 512) * f)
    return out
