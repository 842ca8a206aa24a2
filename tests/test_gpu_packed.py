"""GPU parity of attention over packed sequences and of its relative position bias against the fp64 oracle, element by
element within bounds that follow from the roundings (oracle/packed_oracle.py), through the C ABI."""
import numpy as np
import pytest

import synth_inputs as si
from oracle import packed_oracle as po
from tests import harness as hz

pytestmark = pytest.mark.gpu

UNIT = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _randn(role, shape, std, dtype):
    return si.round_to(si.normal(si.stream_key(0, role, *shape), shape, std), dtype).astype(np.float64)


class Call:
    """Inputs and device buffers of one packed batch.  `front` / `back`: rows of no sequence in front and behind; `gap`:
    elements between the rows of a tensor beyond the dense ones; `shift`: elements by which every pointer is off 16 bytes."""

    def __init__(self, lens, H, Hk, d, causal, dtype, front=0, back=0, buckets=0, far=0, scale=0.0, fused=False, gap=0, shift=0,
                 std=1.0, table_std=1.0):
        import torch
        import paper_2410_19367_amd as bp
        self.bp, self.torch, self.dtype, self.d, self.H, self.Hk = bp, torch, dtype, d, H, Hk
        self.dt = bp.BP_BF16 if dtype == "bf16" else bp.BP_F32
        self.starts = [front + int(x) for x in np.cumsum([0] + list(lens))]
        self.T = T = self.starts[-1] + back
        self.causal, self.far, self.scale = causal, far, scale or d ** -0.5
        self.longest = max(max(lens), 1)
        self.q, self.k, self.v = (_randn(n, (T, h, d), std, dtype) for n, h in (("pq", H), ("pk", Hk), ("pv", Hk)))
        self.g = _randn("pg", (T, H, d), 1.0, dtype)
        self.table = _randn("pt", (buckets, H), table_std, "f32") if buckets else None
        self.fused, self.gap, self.shift = fused, gap, shift
        self.starts_dev = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        self.scale_arg = scale

    def put(self, arr):
        """[T, heads, d] on the device as rows of their own pitch, everything around them NaN."""
        T, h, d = arr.shape
        ld = h * d + self.gap
        t = self.torch.full((T * ld + self.shift + 8,), float("nan"), device="cuda",
                            dtype=self.torch.bfloat16 if self.dtype == "bf16" else self.torch.float32)
        v = t[self.shift:self.shift + T * ld].view(T, ld)[:, :h * d]
        v.copy_(hz.to_dev(arr.reshape(T, h * d), self.dtype))
        return v

    def tensors(self, *arrs):
        if not self.fused:
            return [self.put(a) for a in arrs]
        whole = self.put(np.concatenate(arrs, 1))
        out, c = [], 0
        for a in arrs:
            out.append(whole[:, c:c + a.shape[1] * self.d])
            c += a.shape[1] * self.d
        return out

    def layout(self, q, k, v, o):
        lds = [t.stride(0) if t.shape[0] > 1 else 0 for t in (q, k, v, o)]
        return self.bp.bp_packed(self.T, len(self.starts) - 1, self.starts_dev, self.H, self.Hk, self.d, self.causal, self.scale_arg, *lds)

    def reference(self, ctx_given=None, want=True):
        return po.attention(self.starts, self.q, self.k, self.v, self.causal, self.scale, self.table, self.far,
                            dctx=self.g if want else None, ctx_given=ctx_given)

    def run(self, *args, **kw):
        out = self.start(*args, **kw)
        self.torch.cuda.synchronize()
        return self.finish(out)

    def finish(self, out):
        host = {n: hz.to_host(t) for n, t in out.items()}
        return {n: a if n in ("lse", "dtable") else a.reshape(self.T, -1, self.d) for n, a in host.items()}

    def start(self, stream=None, backward=True, want_table=True, dtable0=None):
        bp, torch = self.bp, self.torch
        q, k, v = self.tensors(self.q, self.k, self.v)
        mark = 7.0                                       # what rows of no sequence hold afterwards
        ctx = self.put(np.full_like(self.q, mark))
        lse = torch.full((self.H, self.T), mark, device="cuda")
        lay = self.layout(q, k, v, ctx)
        bias = table = None
        if self.table is not None:
            table = torch.tensor(self.table, dtype=torch.float32, device="cuda")
            bias = bp.bp_relpos(self.table.shape[0], self.far, table)
        bp.bp_op_attention_packed_fwd(self.dt, lay, q, k, v, ctx, lse, bias=bias, stream=stream)
        out = {"ctx": ctx, "lse": lse}
        if backward:
            g = self.put(self.g)
            dq, dk, dv = self.tensors(*(np.full_like(a, mark) for a in (self.q, self.k, self.v)))
            ws = torch.full((bp.bp_op_attention_packed_workspace(self.dt, lay, bias),), float("nan"), device="cuda")
            dtable = None
            if bias is not None and want_table:
                dtable = torch.full_like(table, float("nan")) if dtable0 is None else torch.tensor(dtable0, dtype=torch.float32, device="cuda")
            bp.bp_op_attention_packed_bwd(self.dt, lay, q, k, v, ctx, lse, g, dq, dk, dv, ws, bias=bias, dtable=dtable,
                                          overwrite=int(dtable0 is None), stream=stream)
            out |= {"dq": dq, "dk": dk, "dv": dv}
            if dtable is not None:
                out["dtable"] = dtable
        return out

    def check(self, got, r=None, mark=7.0):
        if r is None:
            r = self.reference(want="dq" in got)
        tol = po.bounds(r, self.longest, self.d, self.H // self.Hk, UNIT[self.dtype])
        inside = np.zeros(self.T, bool)
        inside[self.starts[0]:self.starts[-1]] = True
        for name, a in got.items():
            ref, t = r[name], tol[name] * np.ones_like(r[name])
            if name == "lse":
                a, ref, t = a.T, ref.T, t.T
            if name != "dtable":
                assert (a[~inside] == mark).all(), f"{name}: rows of no sequence were written"
                a, ref, t = a[inside], ref[inside], t[inside]
            if not a.size:
                continue
            # what ctx's own rounding does to delta: it is one more rounded factor in ds (a share of abs_ctx . |dctx|,
            # which the sums of absolute terms hold already)
            if name in ("dq", "dk") and self.dtype == "bf16":
                t = 2.0 * t
            off = np.abs(a - ref) / (t + 1e-30)
            worst = np.unravel_index(np.nanargmax(np.where(np.isnan(off), np.inf, off)), off.shape)
            assert off[worst] <= 1.0, (name, worst, float(a[worst]), float(ref[worst]), float(t[worst]))


# lengths, heads, kv heads, d, causal
SHAPES = [
    ([1], 1, 1, 64, True), ([2, 1, 0, 3], 2, 1, 64, True), ([0, 0, 5, 0], 2, 2, 64, False),
    ([31, 33, 1, 64], 4, 2, 64, True), ([63, 65, 127], 2, 2, 128, True), ([64, 128, 32], 4, 1, 64, False),
    ([100, 7, 250, 3], 6, 2, 40, True), ([130, 61], 3, 3, 96, False), ([200], 2, 1, 112, True),
    ([257, 300], 4, 4, 64, False), ([513], 2, 1, 128, True), ([700, 90], 2, 2, 64, True),
    ([3] * 90, 2, 1, 64, True), ([1] * 130, 2, 2, 32, False), ([5, 17] * 70, 4, 2, 128, True),
    ([40, 90, 11], 2, 1, 8, True), ([77, 20], 3, 1, 24, False), ([33, 150], 2, 1, 80, True),
]


@pytest.mark.parametrize("lens,H,Hk,d,causal", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_fwd_bwd(lens, H, Hk, d, causal, dtype):
    c = Call(lens, H, Hk, d, causal, dtype, front=len(lens) % 3, back=5 * (d % 3), fused=d % 16 == 0)
    c.check(c.run())


# head widths, strides and pointers that only the row kernels take
@pytest.mark.parametrize("d,gap,shift", [(1, 0, 0), (7, 3, 1), (33, 0, 0), (64, 1, 0), (64, 0, 1), (100, 4, 0), (136, 0, 0), (300, 5, 0), (512, 0, 0)])
@pytest.mark.parametrize("causal,buckets", [(True, 0), (False, 8)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_any_width_and_alignment(d, gap, shift, causal, buckets, dtype):
    c = Call([30, 1, 80, 0, 300], 4, 2, d, causal, dtype, front=2, back=3, buckets=buckets, far=40, gap=gap, shift=shift)
    c.check(c.run())


# lengths, heads, kv heads, d, causal, buckets, max_distance: all distances in one look-up, borders inside tiles, far tiles
# of one bucket, every tile within exact buckets, two buckets
BIASES = [
    ([1, 2, 0, 3], 2, 1, 64, True, 4, 3), ([200, 64, 31], 4, 2, 64, True, 32, 128), ([200, 64, 31], 4, 2, 64, False, 32, 128),
    ([600], 2, 1, 128, True, 32, 100), ([600], 2, 2, 64, False, 16, 40), ([400, 90], 2, 2, 128, False, 128, 2000),
    ([300, 5, 150], 3, 1, 96, True, 128, 65), ([300], 8, 1, 40, True, 2, 7), ([330, 100], 4, 4, 64, True, 64, 5000),
    ([4] * 70, 2, 1, 64, False, 8, 9), ([900, 60], 1, 1, 32, False, 4, 3),
]


@pytest.mark.parametrize("lens,H,Hk,d,causal,buckets,far", BIASES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bias_fwd_bwd(lens, H, Hk, d, causal, buckets, far, dtype):
    c = Call(lens, H, Hk, d, causal, dtype, front=1, back=2, buckets=buckets, far=far)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("buckets", [0, 32])
def test_packed_every_block_shape(dtype, buckets):
    """Launches from a few blocks to many: the variants for few, some and many blocks."""
    for lens, H, Hk, d, causal in (([300, 900], 16, 4, 64, True), ([1000, 200, 700], 48, 16, 64, True),
                                   ([640] * 4, 24, 24, 64, False), ([512, 1024], 32, 8, 128, True)):
        if dtype == "f32" and sum(lens) * H > 40000:
            continue
        c = Call(lens, H, Hk, d, causal, dtype, back=3, buckets=buckets, far=128)
        c.check(c.run())


# Launches with enough blocks for those of two heads and of 128 rows (on 256 CUs), of sequences that begin anywhere in them
WIDE = [([60] * 140 + [5], 32, 8, 64, True), ([61] * 140, 32, 32, 64, False), ([60] * 140, 16, 16, 128, True),
        ([1, 200, 61, 0, 77] * 25, 16, 8, 96, False), ([130] * 16, 32, 1, 128, True), ([3, 60, 100] * 50, 33, 11, 40, True)]


@pytest.mark.parametrize("lens,H,Hk,d,causal", WIDE)
@pytest.mark.parametrize("buckets", [0, 32])
def test_packed_wide_blocks(lens, H, Hk, d, causal, buckets):
    c = Call(lens, H, Hk, d, causal, "bf16", front=3, back=7, buckets=buckets, far=48, fused=True)
    c.check(c.run())


@pytest.mark.parametrize("lens,H,Hk,d,causal", WIDE[:4])
def test_packed_wide_blocks_what_is_not_finite(lens, H, Hk, d, causal):
    clean = Call(lens, H, Hk, d, causal, "bf16", front=3, back=7)
    r = clean.reference()
    c = Call(lens, H, Hk, d, causal, "bf16", front=3, back=7)
    G, bad = H // Hk, [i for i, n in enumerate(lens) if n > 50][-2]
    at = c.starts[bad] + 40
    c.v[at, Hk - 1, 1] = np.nan
    for x in (c.q, c.k, c.v, c.g):
        x[:3] = np.nan
        x[c.starts[-1]:] = np.nan
    got = c.run()
    tol = po.bounds(r, c.longest, d, G, UNIT["bf16"])
    S = slice(c.starts[bad], c.starts[bad + 1])
    for name in ("ctx", "dq", "dk", "dv"):
        reach = np.zeros(got[name].shape[:2], bool)
        if name in ("ctx", "dq"):
            reach[slice(at, S.stop) if causal else S, H - G:] = True
        else:
            reach[S, Hk - 1] = True
        fine = ~reach
        fine[:3] = fine[c.starts[-1]:] = False
        assert (np.abs(got[name][fine] - r[name][fine]) <= 2 * tol[name][fine] + 1e-30).all(), name
        assert (got[name][:3] == 7.0).all() and (got[name][c.starts[-1]:] == 7.0).all()
    assert np.isnan(got["ctx"][at, H - G:, 1]).all()


@pytest.mark.parametrize("causal", [True, False])
def test_packed_short_sequences_behind_long_ones(causal):
    """delta of rows with few keys does not come from the rounded ctx, also where their block holds the end of a long
    sequence: what is left in dQ of these rows are two roundings of equal size, of dS and of dQ itself (their norms add up to
    sqrt(2) times one), and a tenth for all else."""
    c = Call([700, 20, 30, 600, 9, 25, 300, 14], 8, 2, 64, causal, "bf16")
    got, r = c.run(), c.reference()
    rows = np.concatenate([np.arange(s, e) for s, e in zip(c.starts[:-1], c.starts[1:]) if e - s <= 30])
    one = np.linalg.norm(si.round_bf16(r["dq"][rows]) - r["dq"][rows])
    assert np.linalg.norm(got["dq"][rows] - r["dq"][rows]) <= 1.55 * one


# More starts than a wave loads at once, two and three levels of them; hundreds of empty sequences inside one block of rows
@pytest.mark.parametrize("lens", [[0] * 3000 + [1, 2, 0, 0, 0] * 700 + [0] * 900, [3] + [0] * 500 + [70, 0, 1] + [0] * 130 + [90] + [0] * 64,
                                  [0] * 63 + [100], [0] * 64 + [100], [1] * 63 + [40], [5] * 64 + [0] * 4100 + [61]])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_many_sequences(lens, causal):
    c = Call(lens, 2, 1, 64, causal, "bf16", front=2, back=1, buckets=8, far=30)
    c.check(c.run())


# Rows farther apart than their heads, one key / value head for all, blocks of both kinds
@pytest.mark.parametrize("lens,H,Hk,d,gap", [([200, 31, 90], 64, 1, 64, 8), ([200, 31, 90], 24, 1, 128, 16), ([70, 300], 6, 6, 40, 24),
                                             ([150] * 20, 32, 2, 96, 8)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_row_pitch_and_one_kv_head(lens, H, Hk, d, gap, dtype):
    if dtype == "f32":
        lens = lens[:3]
    c = Call(lens, H, Hk, d, True, dtype, back=4, gap=gap, buckets=16, far=50)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_table_gradient_next_to_what_is_not_finite(dtype):
    """The table's gradient takes nothing from masked pairs or from rows of no sequence: a NaN behind the last token that
    has a gradient, and NaN in every padding row."""
    c = Call([50, 90, 40], 2, 1, 64, True, dtype, front=9, back=30, buckets=16, far=40)
    r = c.reference()
    for x in (c.q, c.k, c.v, c.g):
        x[:9] = np.nan
        x[c.starts[-1]:] = np.nan
    c.check(c.run(), r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_least_workspace(dtype):
    """Without room for the sums of parts, shared heads are summed in one block."""
    import torch
    import paper_2410_19367_amd as bp
    c = Call([100, 70], 8, 1, 64, True, dtype, buckets=16, far=40)
    need = ((8 * c.T + 3) & ~3) + ((c.T + 63) // 64 * 8 * 16 + 3 & ~3)
    full = bp.bp_op_attention_packed_workspace
    try:
        bp.bp_op_attention_packed_workspace = lambda *a: need
        c.check(c.run())
    finally:
        bp.bp_op_attention_packed_workspace = full
    assert full(c.dt, bp.bp_packed(c.T, 2, c.starts_dev, 8, 1, 64, True), None) > 8 * c.T
    torch.cuda.synchronize()


def test_packed_two_calls_at_once():
    """Two streams, a workspace each."""
    import torch
    a, b = Call([400, 90], 8, 2, 64, True, "bf16", buckets=32, far=64), Call([300, 33, 150], 4, 4, 128, False, "bf16")
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(streams[0]):
            x = a.start(streams[0].cuda_stream)
        with torch.cuda.stream(streams[1]):
            y = b.start(streams[1].cuda_stream)
        torch.cuda.synchronize()
        a.check(a.finish(x))
        b.check(b.finish(y))


def test_packed_table_gradient_adds_and_is_optional():
    c = Call([90, 200], 4, 2, 64, True, "bf16", buckets=32, far=64)
    first = c.run()
    base = _randn("pt0", (32, 4), 10.0, "f32")
    added = c.run(dtable0=base)
    assert np.max(np.abs(added["dtable"] - np.float32(base + first["dtable"]))) <= 2.0 ** -20 * (np.max(np.abs(base)) + np.max(np.abs(first["dtable"])))
    without = c.run(want_table=False)
    assert "dtable" not in without
    r = c.reference()
    for name in ("dq", "dk", "dv"):
        assert hz.rel_err(without[name], r[name]) < 2e-2


def test_packed_scale():
    for scale in (1.0, 0.02, 1e-6):
        c = Call([70, 130], 2, 1, 64, True, "f32", buckets=16, far=50, scale=scale, std=0.3)
        c.check(c.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_same_bits_every_time(dtype):
    c = Call([300, 77, 500, 20], 8, 2, 64, True, dtype, buckets=32, far=128)
    a, b = c.run(), c.run()
    for n in a:
        assert np.array_equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal,bias", [(True, 0), (False, 0), (True, 16)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_packed_what_is_not_finite_stays_in_its_sequence(dtype, d, causal, bias, value):
    """A value that is not finite reaches neither other sequences nor, under a causal mask, earlier tokens; padding rows
    may hold anything."""
    lens, bad = [40, 50, 100, 70], 2                    # neighbours share tiles of 64 rows with the bad sequence
    clean = Call(lens, 4, 2, d, causal, dtype, front=3, back=9, buckets=bias, far=30)
    ref = clean.run()
    for where in ("k", "v", "q", "g"):
        c = Call(lens, 4, 2, d, causal, dtype, front=3, back=9, buckets=bias, far=30)
        at = c.starts[bad] + 60
        getattr(c, where)[at, 0, 3] = value
        for x in (c.q, c.k, c.v, c.g):
            x[:3] = np.nan
            x[c.starts[-1]:] = np.nan
        got = c.run(want_table=False)
        r = clean.reference()
        tol = po.bounds(r, c.longest, d, 2, UNIT[dtype])
        G = 2
        heads = {"q": [0], "g": [0]}.get(where, [0, 1])         # heads that read the bad element
        for name in ("ctx", "dq", "dk", "dv"):
            touched = np.zeros(got[name].shape[:2], bool)
            S = slice(c.starts[bad], c.starts[bad + 1])
            for h in heads:
                if name in ("ctx", "dq"):                       # query rows that attend the bad row, or are it
                    touched[slice(at, S.stop) if causal and where in "kv" else slice(at, at + 1) if where in "qg" else S, h] = True
                else:                                           # keys of queries with a bad softmax or gradient
                    touched[S, h // G] = True
            inside = np.zeros(c.T, bool)
            inside[c.starts[0]:c.starts[-1]] = True
            a, b = got[name][inside][~touched[inside]], r[name][inside][~touched[inside]]
            t = tol[name][inside][~touched[inside]]
            assert np.isfinite(a).all(), (where, name)
            assert (np.abs(a - b) <= 2 * t + 1e-30).all(), (where, name)
            assert (got[name][~inside] == 7.0).all(), (where, name)
        # and where it does reach, it shows
        if where == "v":
            assert not np.isfinite(got["ctx"][at, 0, 3]) and not np.isfinite(got["ctx"][at, 1, 3])
        if where == "k" and value != value:
            assert np.isnan(got["ctx"][at, 0]).all()
    assert all(np.isfinite(ref[n]).all() for n in ref)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_masks_of_the_lowest_value(dtype):
    """A bucket whose bias is the type's lowest value or -inf takes no probability; the others share it."""
    for low in (-3.0e38, -np.inf):
        c = Call([150, 40], 2, 1, 64, True, dtype, buckets=16, far=40)
        c.table[3:] = low
        got = c.run()
        r = c.reference()
        tol = po.bounds({**r, "z": 30.0}, c.longest, 64, 2, UNIT[dtype])
        for name in ("ctx", "dq", "dk", "dv"):
            assert (np.abs(got[name] - r[name]) <= 2 * tol[name] + 1e-30).all(), (low, name)
        assert (got["dtable"][3:] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_starts_that_are_no_starts(dtype):
    """Starts outside the tensors or out of order name no rows outside them: the call ends, and rows that the starts
    still describe are right."""
    c = Call([60, 70, 50], 2, 1, 64, True, dtype)
    T = c.T
    for bad in ([0, 60, 130, T + 1000], [-50, 60, 130, T], [0, 130, 60, T], [T, T, T, T], [T + 5, 0, 3, -7], [0, 0, 0, 0]):
        c.starts_dev = c.torch.tensor(bad, dtype=c.torch.int32, device="cuda")
        got = c.run()
        if bad == [0, 60, 130, T + 1000]:
            c.check(got)
        if bad in ([T, T, T, T], [0, 0, 0, 0]):
            assert all((a == 7.0).all() for a in got.values())


def test_packed_other_stream_and_graph():
    """On a stream of the caller's, and captured: replays with new inputs give what eager calls give."""
    import torch
    import paper_2410_19367_amd as bp
    c = Call([200, 30, 90], 4, 2, 64, True, "bf16", buckets=32, far=64)
    eager = c.run()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = c.run(stream=s.cuda_stream)
    for n in eager:
        assert np.array_equal(eager[n], other[n]), n
    q, k, v = (c.put(a) for a in (c.q, c.k, c.v))
    g, ctx, lse = c.put(c.g), c.put(c.q), torch.zeros((4, c.T), device="cuda")
    dq, dk, dv = (torch.zeros_like(t) for t in (q, k, v))
    table = torch.tensor(c.table, dtype=torch.float32, device="cuda")
    dtable = torch.zeros_like(table)
    lay, bias = c.layout(q, k, v, ctx), bp.bp_relpos(32, 64, table)
    ws = torch.zeros(bp.bp_op_attention_packed_workspace(c.dt, lay, bias), device="cuda")

    def step(stream):
        bp.bp_op_attention_packed_fwd(c.dt, lay, q, k, v, ctx, lse, bias=bias, stream=stream)
        bp.bp_op_attention_packed_bwd(c.dt, lay, q, k, v, ctx, lse, g, dq, dk, dv, ws, bias=bias, dtable=dtable, overwrite=1, stream=stream)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream().cuda_stream)
    for i in range(4):
        for t in (q, k, v, g):
            t.copy_(torch.roll(t, 1, 0))
        for t in (dq, dk, dv, dtable, ctx):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        seen = [t.clone() for t in (ctx, lse, dq, dk, dv, dtable)]
        step(None)
        torch.cuda.synchronize()
        for x, y in zip(seen, (ctx, lse, dq, dk, dv, dtable)):
            assert torch.equal(x, y), i


def test_packed_offsets_beyond_32_bits():
    """Rows so far apart that elements lie beyond 2^32 bytes and 2^31 elements: the last rows are right."""
    import torch
    import paper_2410_19367_amd as bp
    T, ld, d, n = 200, (1 << 24) - 8, 64, 120           # 200 rows of 2^24: 3.3e9 elements
    q = torch.zeros(T * ld, dtype=torch.bfloat16, device="cuda").view(T, ld)
    small = torch.from_numpy(_randn("far", (T, 3 * d), 1.0, "bf16").astype(np.float32)).cuda().to(torch.bfloat16)
    q[:, :3 * d] = small
    out = torch.zeros_like(q)
    starts = torch.tensor([0, T - n, T], dtype=torch.int32, device="cuda")
    args = dict(tokens=T, sequences=2, starts=starts, heads=1, kv_heads=1, head_dim=d, causal=True)
    far, near = bp.bp_packed(**args, ld_q=ld, ld_k=ld, ld_v=ld, ld_ctx=ld), bp.bp_packed(**args, ld_q=3 * d, ld_k=3 * d, ld_v=3 * d, ld_ctx=d)
    ctx, ctx2 = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda"), out[:, 3 * d:4 * d]
    lse, lse2 = torch.zeros((1, T), device="cuda"), torch.zeros((1, T), device="cuda")
    s = [small[:, i * d:(i + 1) * d] for i in range(3)]
    f = [q[:, i * d:(i + 1) * d] for i in range(3)]
    bp.bp_op_attention_packed_fwd(bp.BP_BF16, near, *s, ctx, lse)
    bp.bp_op_attention_packed_fwd(bp.BP_BF16, far, *f, ctx2, lse2)
    g2, g = q[:, :d], small[:, :d].contiguous()
    ws = torch.zeros(bp.bp_op_attention_packed_workspace(bp.BP_BF16, far), device="cuda")
    small_out = torch.zeros((T, 3 * d), dtype=torch.bfloat16, device="cuda")
    bp.bp_op_attention_packed_bwd(bp.BP_BF16, near, *s, ctx, lse, g, *(small_out[:, i * d:(i + 1) * d] for i in range(3)), ws)
    bp.bp_op_attention_packed_bwd(bp.BP_BF16, far, *f, ctx2, lse2, g2, *(out[:, i * d:(i + 1) * d] for i in range(3)), ws)
    torch.cuda.synchronize()
    assert torch.equal(ctx, ctx2) and torch.equal(lse, lse2)
    assert torch.equal(small_out, out[:, :3 * d])


def test_packed_block_of_a_layer():
    """The calls as a layer makes them: one projection to q, k and v, attention with its bias, the output projection, and
    all of it backwards into the projection's weight gradient."""
    import torch
    import paper_2410_19367_amd as bp
    lens, H, Hk, d, hid = [90, 33, 128], 4, 2, 64, 256
    T, N = sum(lens), (H + 2 * Hk) * d
    c = Call(lens, H, Hk, d, True, "f32", buckets=16, far=60)
    x, w, wo, gy = (_randn(n, s, std, "f32") for n, s, std in (("bx", (T, hid), 1.0), ("bw", (hid, N), 0.06),
                                                              ("bo", (H * d, hid), 0.06), ("bg", (T, hid), 1.0)))
    dev = {n: hz.to_dev(a, "f32") for n, a in (("x", x), ("w", w), ("wo", wo), ("gy", gy))}
    new = lambda *s: torch.zeros(s, device="cuda")          # noqa: E731
    qkv, ctx, y, lse = new(T, N), new(T, H * d), new(T, hid), new(H, T)
    cut = lambda t: (t[:, :H * d], t[:, H * d:(H + Hk) * d], t[:, (H + Hk) * d:])           # noqa: E731
    lay = bp.bp_packed(T, 3, c.starts_dev, H, Hk, d, True, 0.0, N, N, N)
    table = torch.tensor(c.table, dtype=torch.float32, device="cuda")
    bias, dtable, dqkv, dctx, dw = bp.bp_relpos(16, 60, table), new(16, H), new(T, N), new(T, H * d), new(hid, N)
    ws = new(bp.bp_op_attention_packed_workspace(bp.BP_F32, lay, bias))
    F = bp.BP_F32
    bp.bp_op_gemm(F, 0, 0, T, N, hid, dev["x"], hid, dev["w"], N, qkv, N)
    bp.bp_op_attention_packed_fwd(F, lay, *cut(qkv), ctx, lse, bias=bias)
    bp.bp_op_gemm(F, 0, 0, T, hid, H * d, ctx, H * d, dev["wo"], hid, y, hid)
    bp.bp_op_gemm(F, 0, 1, T, H * d, hid, dev["gy"], hid, dev["wo"], hid, dctx, H * d)
    bp.bp_op_attention_packed_bwd(F, lay, *cut(qkv), ctx, lse, dctx, *cut(dqkv), ws, bias=bias, dtable=dtable)
    bp.bp_op_wgrad_group(F, hid, N, T, [dev["x"]], [dqkv], dw, overwrite=1)
    torch.cuda.synchronize()
    r_qkv = x @ w
    q, k, v = (a.reshape(T, -1, d) for a in cut(r_qkv))
    r = po.attention(c.starts, q, k, v, True, d ** -0.5, c.table, 60, dctx=(gy @ wo.T).reshape(T, H, d))
    assert hz.rel_err(hz.to_host(y), r["ctx"].reshape(T, -1) @ wo) < 1e-5
    r_dqkv = np.concatenate([r[n].reshape(T, -1) for n in ("dq", "dk", "dv")], 1)
    assert hz.rel_err(hz.to_host(dw), x.T @ r_dqkv) < 2e-5
    assert hz.rel_err(hz.to_host(dtable), r["dtable"]) < 2e-5


@pytest.mark.parametrize("d,shift", [(64, 0), (128, 0), (40, 1)])
@pytest.mark.parametrize("causal,buckets", [(True, 0), (False, 0), (True, 16), (False, 16)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_packed_one_key_alone_has_no_gradient_of_its_score(dtype, causal, buckets, d, shift):
    """The one probability is 1 whatever the score is: dq, dk and the table's gradient are 0, not a rounding's remainder."""
    c = Call([1, 0, 1, 1] * 30, 4, 2, d, causal, dtype, front=2, back=3, buckets=buckets, far=32, shift=shift)
    got = c.run()
    for name in ("dq", "dk"):
        assert (got[name][2:-3] == 0).all(), name
    if buckets:
        assert (got["dtable"] == 0).all()
    c.check(got)
