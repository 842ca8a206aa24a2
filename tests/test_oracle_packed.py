"""CPU: pins of the packed-attention oracle, the position buckets of the library against it, and what the library refuses
before anything reaches a GPU."""
import ctypes as C

import numpy as np
import pytest

import paper_2410_19367_amd as bp
from oracle import packed_oracle as po
from oracle import stage_oracle as O


def _inputs(T, H, Hk, d, seed=0):
    g = np.random.default_rng(seed)
    return g.normal(size=(T, H, d)), g.normal(size=(T, Hk, d)), g.normal(size=(T, Hk, d)), g.normal(size=(T, H, d))


@pytest.mark.parametrize("causal", [True, False])
def test_equal_heads_one_length_is_the_stage_oracles_attention(causal):
    B, S, H, d = 3, 7, 2, 8
    q, k, v, g = _inputs(B * S, H, H, d)
    r = po.attention([0, S, 2 * S, 3 * S], q, k, v, causal, d ** -0.5, dctx=g)
    split = lambda t: t.reshape(B, S, H, d).transpose(0, 2, 1, 3)                      # noqa: E731
    merge = lambda t: t.transpose(0, 2, 1, 3).reshape(B * S, H, d)                     # noqa: E731
    ctx, p = O.attention_fwd(split(q), split(k), split(v), causal, None)
    dq, dk, dv = O.attention_bwd(split(g), split(q), split(k), split(v), p)
    for name, ref in (("ctx", ctx), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert np.max(np.abs(r[name] - merge(ref))) < 1e-12, name


@pytest.mark.parametrize("causal", [True, False])
def test_gradients_against_differences(causal):
    starts, H, Hk, d, nb, far = [1, 6, 6, 7, 12], 4, 2, 3, 8, 5
    q, k, v, g = _inputs(13, H, Hk, d)
    table = np.random.default_rng(5).normal(size=(nb, H))
    rows = slice(1, 12)

    def loss(q, k, v, table):
        return float(np.sum(po.attention(starts, q, k, v, causal, 0.7, table, far)["ctx"][rows] * g[rows]))

    r = po.attention(starts, q, k, v, causal, 0.7, table, far, dctx=g)
    h, gen = 1e-5, np.random.default_rng(6)
    for i, name in enumerate(("dq", "dk", "dv", "dtable")):
        args = [q, k, v, table]
        for _ in range(12):
            at = tuple(gen.integers(0, n) for n in args[i].shape)
            if name != "dtable" and not 1 <= at[0] < 12:
                continue
            diff = []
            for sgn in (h, -h):
                x = args[i].copy()
                x[at] += sgn
                diff.append(loss(*args[:i], x, *args[i + 1:]))
            assert abs((diff[0] - diff[1]) / (2 * h) - r[name][at]) < 1e-7, (name, at)


def test_rows_of_no_sequence_and_heads_that_share():
    q, k, v, _ = _inputs(9, 4, 2, 4)
    r = po.attention([2, 5, 5, 8], q, k, v, True, 0.5)
    assert np.isnan(r["ctx"][[0, 1, 8]]).all() and np.isfinite(r["ctx"][2:8]).all()
    assert np.allclose(r["ctx"][2], np.repeat(v[2], 2, axis=0))       # the first token attends itself only
    assert np.allclose(r["ctx"][5], np.repeat(v[5], 2, axis=0))


# one bucket a direction that is logarithmic, powers that fall on borders, borders close together, the widest
BUCKETS = [(1, 2, 5), (1, 32, 128), (0, 32, 128), (1, 32, 1000), (0, 4, 3), (0, 8, 64), (1, 16, 9), (1, 64, 33), (0, 64, 4096),
           (1, 128, 65), (1, 128, 100000), (0, 128, 8192), (1, 7, 81)]


@pytest.mark.parametrize("causal,buckets,far", BUCKETS)
def test_buckets_are_the_oracles(causal, buckets, far):
    offsets = set(range(-300, 1 if causal else 301)) | {-far, -far + 1, -far - 1, -(1 << 30)}
    n = buckets if causal else buckets // 2
    e = n // 2
    for m in range(1, n - e):           # around every border
        x = int(e * (far / e) ** (m / (n - e)))
        offsets |= {-o for o in range(max(0, x - 2), x + 3)}
    if not causal:
        offsets |= {-o for o in offsets} - {1 << 31}
    for o in offsets:
        assert bp.bp_relpos_bucket(causal, buckets, far, o) == po.bucket(causal, buckets, far, o), o


@pytest.mark.parametrize("causal,buckets,far,offset", [(1, 1, 10, 0), (0, 2, 10, 0), (0, 5, 10, 0), (1, 32, 16, 0), (1, 130, 1000, 0),
                                                       (0, 32, 8, 0), (1, 32, 1 << 24, 0), (1, 32, 128, 1), (1, 0, 10, 0), (1, -4, 10, 0)])
def test_buckets_refused(causal, buckets, far, offset):
    with pytest.raises(bp.BitPipeError) as e:
        bp.bp_relpos_bucket(causal, buckets, far, offset)
    assert e.value.code == bp.BP_EINVAL


GOOD = dict(tokens=100, sequences=3, starts=4096, heads=8, kv_heads=2, head_dim=64, causal=True)


def _calls(layout, bias=None, dtype=bp.BP_BF16, missing=None, workspace_elems=1 << 30, dtable=None, workspace_at=4096):
    """Both directions with addresses that nothing may touch before the arguments are refused."""
    a = {n: 4096 for n in ("q", "k", "v", "ctx", "lse", "dctx", "dq", "dk", "dv", "workspace")}
    a["workspace"] = workspace_at
    if missing:
        a[missing] = None
    yield lambda: bp.bp_op_attention_packed_fwd(dtype, layout, a["q"], a["k"], a["v"], a["ctx"], a["lse"], bias=bias)
    yield lambda: bp.bp_op_attention_packed_bwd(dtype, layout, a["q"], a["k"], a["v"], a["ctx"], a["lse"], a["dctx"], a["dq"],
                                                a["dk"], a["dv"], a["workspace"], bias=bias, dtable=dtable,
                                                workspace_elems=workspace_elems)


@pytest.mark.parametrize("change,code", [
    (dict(tokens=0), bp.BP_EINVAL), (dict(sequences=0), bp.BP_EINVAL), (dict(starts=None), bp.BP_EINVAL),
    (dict(heads=0), bp.BP_EINVAL), (dict(kv_heads=0), bp.BP_EINVAL), (dict(kv_heads=3), bp.BP_EINVAL),
    (dict(kv_heads=16), bp.BP_EINVAL), (dict(head_dim=0), bp.BP_EINVAL), (dict(head_dim=513), bp.BP_ESHAPE),
    (dict(tokens=1 << 24), bp.BP_ESHAPE), (dict(heads=16384, kv_heads=2), bp.BP_ESHAPE), (dict(scale=-1.0), bp.BP_EINVAL),
    (dict(tokens=(1 << 24) - 1, heads=128), bp.BP_ESHAPE), (dict(scale=float("nan")), bp.BP_EINVAL), (dict(scale=float("inf")), bp.BP_EINVAL), (dict(ld_q=511), bp.BP_EINVAL),
    (dict(ld_k=127), bp.BP_EINVAL), (dict(ld_v=-8), bp.BP_EINVAL), (dict(ld_ctx=1 << 24), bp.BP_ESHAPE)])
def test_layouts_refused(change, code):
    layout = bp.bp_packed(**{**GOOD, **change})
    for call in _calls(layout):
        with pytest.raises(bp.BitPipeError) as e:
            call()
        assert e.value.code == code and str(e.value)
    assert bp.bp_op_attention_packed_workspace(bp.BP_BF16, layout) == 0


def test_pointers_types_and_workspace_refused():
    layout = bp.bp_packed(**GOOD)
    bias = bp.bp_relpos(32, 128, 4096)
    for call in _calls(layout, dtype=7):
        with pytest.raises(bp.BitPipeError):
            call()
    for missing in ("q", "k", "v", "ctx", "lse"):
        for call in _calls(layout, missing=missing):
            with pytest.raises(bp.BitPipeError) as e:
                call()
            assert e.value.code == bp.BP_EINVAL
    bwd = lambda **kw: list(_calls(layout, **kw))[1]               # noqa: E731
    need = 100 * 8 + 2 * 8 * 32
    assert bp.bp_op_attention_packed_workspace(bp.BP_BF16, layout, bias) >= need
    assert bp.bp_op_attention_packed_workspace(bp.BP_BF16, layout) >= 100 * 8
    for call in [bwd(missing=n) for n in ("dctx", "dq", "dk", "dv", "workspace")] + [
            bwd(bias=bias, workspace_elems=need - 1), bwd(dtable=4096), bwd(workspace_at=4100), *_calls(layout, bp.bp_relpos(32, 128, None)),
            *_calls(layout, bp.bp_relpos(1, 128, 4096)), *_calls(layout, bp.bp_relpos(32, 3, 4096))]:
        with pytest.raises(bp.BitPipeError) as e:
            call()
        assert e.value.code == bp.BP_EINVAL
    assert bp.lib().bp_op_attention_packed_fwd(0, None, None, *[C.c_void_p(4096)] * 5, None) == bp.BP_EINVAL
