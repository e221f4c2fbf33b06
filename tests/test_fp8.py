"""The 8-bit path without a GPU: pins of its oracle (oracle.fp8) and the refusals of
its entry points, which come before any device call (dummy device pointers are
never used)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import fp8 as F
from paper_2606_19667_amd import cw

E, U = cw.CW_EINVAL, cw.CW_EUNSUPPORTED


# ---------------------------------------------------------------- the oracle
def test_decode_is_torchs_e4m3():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    got = F.decode(codes)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])


def test_round_value_is_torchs_conversion_and_nearest():
    rng = np.random.default_rng(1)
    vals = F.decode(np.arange(0x7F, dtype=np.uint8))
    ties = (vals[1:] + vals[:-1]) / 2
    x = np.concatenate([rng.normal(size=4000) * np.exp2(rng.uniform(-12, 8, 4000)), vals, ties, np.nextafter(ties, 1e9),
                        np.nextafter(ties, 0)]).astype(np.float32)
    x = np.concatenate([x, -x])
    x = x[np.abs(x) <= 448]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    got = F.round_value(x)
    assert np.array_equal(got, want.astype(np.float64))
    every = np.concatenate([vals, -vals])
    near = np.abs(every[None, :] - x[:500, None].astype(np.float64)).min(axis=1)
    assert np.allclose(np.abs(got[:500] - x[:500]), near, rtol=0, atol=0)
    assert np.isnan(F.round_value([np.inf, -np.inf, np.nan, 465.0, -1e30])).all()
    assert F.round_value([464.0])[0] == 448.0


def test_scale_for_closed_forms():
    assert F.scale_for(448.0) == 1.0 and F.scale_for(np.nextafter(448.0, 500)) == 2.0
    assert F.scale_for(0.0) == 2.0 ** -100 and F.scale_for(1.75) == 2.0 ** -8 and F.scale_for(1.0) == 2.0 ** -8
    assert F.scale_for(3e38) == 2.0 ** 120 and F.scale_for(0.9) == 2.0 ** -8 and F.scale_for(0.8) == 2.0 ** -9


def test_append_hand_worked():
    """Two rows start a block, a third one raises its scale, a fourth does not."""
    v, s = np.full((2, 1, 4, 2), 7.0), np.full((2, 1), 3.0)
    rows = np.array([[[100.0, 1.0]], [[448.0, 2.0 ** -9]]])
    v, s = F.append(v, s, rows, [[1, 0]], [0, 2], [0], block_size=4)
    assert s.tolist() == [[3.0], [1.0]]                      # block 0 is not touched, block 1 starts anew
    assert v[1, 0].tolist() == [[96.0, 1.0], [448.0, 2.0 ** -9], [7.0, 7.0], [7.0, 7.0]]   # 100 is a tie: even
    v, s = F.append(v, s, np.array([[[1000.0, 0.0]]]), [[1, 0]], [0, 1], [2], block_size=4)
    assert s[1, 0] == 4.0 and v[1, 0, 2].tolist() == [256.0, 0.0]
    assert v[1, 0, 1].tolist() == [112.0, 0.0]               # 2^-11 at scale 4 rounds to nothing
    v2, s2 = F.append(v, s, np.array([[[8.0, 0.0]]]), [[1, 0]], [0, 1], [3], block_size=4)
    assert s2[1, 0] == 4.0 and v2[1, 0, 3].tolist() == [2.0, 0.0] and np.array_equal(v2[1, 0, :3], v[1, 0, :3])
    assert np.isnan(F.append(v, s, np.array([[[np.inf, 1.0]]]), [[0]], [0, 1], [0], block_size=4)[0][0, 0, 0, 0])


def test_linear_and_norm_against_plain_loops():
    rng = np.random.default_rng(2)
    x, w = F.round_value(rng.normal(size=(3, 144)) * 8), F.round_value(rng.normal(size=(160, 144)) * 8)
    xs, ws = rng.uniform(0.1, 2, (3, 2)), rng.uniform(0.1, 2, (2, 2))
    b = rng.normal(size=160)
    y, mag = F.linear(x, xs, w, ws, b)
    for t, n in ((0, 0), (2, 159), (1, 127), (1, 128)):
        terms = [x[t, k] * xs[t, k // 128] * w[n, k] * ws[n // 128, k // 128] for k in range(144)]
        assert math.isclose(y[t, n], math.fsum(terms) + b[n], rel_tol=1e-12)
        assert math.isclose(mag[t, n], math.fsum(map(abs, terms)) + abs(b[n]), rel_tol=1e-12)
    cut, cut2 = F.linear_cut(x, xs, w, ws)
    groups = [max(abs(x[1, k]) for k in range(a, a + 8)) * max(abs(w[130, k]) for k in range(a, a + 8)) *
              xs[1, a // 128] * ws[1, a // 128] for a in range(0, 144, 8)]
    assert math.isclose(cut[1, 130], math.fsum(groups), rel_tol=1e-12)
    assert math.isclose(cut2[1, 130], math.fsum(v * v for v in groups), rel_tol=1e-12)
    h, wt = rng.normal(size=(2, 200)), rng.normal(size=200)
    y, s = F.add_rms_norm(h, None, wt, 1e-3)
    inv = 1 / math.sqrt(math.fsum(v * v for v in h[1]) / 200 + 1e-3)
    assert math.isclose(y[1, 150], h[1, 150] * inv * wt[150], rel_tol=1e-12)
    assert math.isclose(s[1, 1], max(abs(h[1, c] * inv * wt[c]) for c in range(128, 200)) / 448, rel_tol=1e-12)
    assert F.add_rms_norm(np.zeros((1, 16)), None, np.ones(16), 1e-3)[1].tolist() == [[1.0]]


def test_logical_rows_drop_foreign_blocks():
    v, s = np.arange(2 * 1 * 16 * 2, dtype=float).reshape(2, 1, 16, 2), np.array([[2.0], [4.0]])
    out = F.logical_rows(v, s, [1, -1, 0], 35)
    assert out.shape == (35, 1, 2)
    assert np.array_equal(out[:16, 0], v[1, 0] * 4) and not out[16:32].any() and np.array_equal(out[32:, 0], v[0, 0, :3] * 2)


# ---------------------------------------------------------------- refusals
d_ = ctypes.c_void_p(4096)
odd = ctypes.c_void_p(4104)
i32 = lambda *v: np.array(v, np.int32)
p32 = lambda a: a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def _norm(x=d_, xs=64, r=d_, rs=64, w=d_, eps=1e-5, rows=4, hidden=64, ro=d_, o=d_, s=d_):
    return cw.lib().cw_add_rms_norm_fp8(x, xs, r, rs, w, eps, rows, hidden, ro, o, s, None)


@pytest.mark.parametrize("status,change", [
    (E, dict(rows=-1)), (E, dict(x=None)), (E, dict(w=None)), (E, dict(o=None)), (E, dict(s=None)), (E, dict(eps=0.0)),
    (E, dict(eps=float("nan"))), (E, dict(eps=2.0)), (E, dict(xs=56)), (E, dict(xs=68)), (E, dict(rs=56)),
    (E, dict(x=odd)), (E, dict(ro=odd)), (E, dict(o=odd)), (U, dict(hidden=24, xs=64)), (U, dict(hidden=0)),
    (U, dict(hidden=16400, xs=16400, rs=16400)), (U, dict(rows=2 ** 31)), (U, dict(rows=2 ** 22 + 1)),
])
def test_norm_refusals(status, change):
    assert _norm(**change) == status
    assert "add_rms_norm_fp8" in cw.last_error()


@pytest.mark.parametrize("change", [dict(ro=d_, x=d_, xs=72, r=None), dict(ro=d_, r=d_, rs=128, x=ctypes.c_void_p(8192))])
def test_norm_in_place_only_where_rows_are_contiguous(change):
    assert _norm(**change) == E and "rows that lie apart" in cw.last_error()


def test_norm_of_no_rows_launches_nothing():
    assert _norm(rows=0, x=None, r=None, o=None, s=None, ro=None) == cw.CW_OK


def _linear(x=d_, xs=d_, w=d_, ws=d_, b=d_, rows=4, n=64, k=64, o=d_):
    return cw.lib().cw_fp8_linear(x, xs, w, ws, b, rows, n, k, o, None)


@pytest.mark.parametrize("status,change", [
    (E, dict(rows=-1)), (E, dict(x=None)), (E, dict(xs=None)), (E, dict(w=None)), (E, dict(ws=None)), (E, dict(o=None)),
    (E, dict(x=odd)), (E, dict(w=odd)), (E, dict(b=odd)), (E, dict(o=odd)), (U, dict(k=24)), (U, dict(k=0)),
    (U, dict(n=24)), (U, dict(n=0)), (U, dict(k=2 ** 20 + 16)), (U, dict(n=2 ** 20 + 16)), (U, dict(rows=2 ** 22 + 1)),
])
def test_linear_refusals(status, change):
    assert _linear(**change) == status
    assert "fp8_linear" in cw.last_error()


def test_linear_of_no_rows_launches_nothing():
    assert _linear(rows=0, x=None, xs=None, o=None) == cw.CW_OK


def _append(q=d_, qs=512, k=d_, ks=128, v=d_, vs=128, rope=d_, n=64, qo=d_, k8=d_, v8=d_, sk=d_, sv=d_, bt=d_, stride=4,
            cud=d_, pld=d_, cu=i32(0, 3, 5), pl=i32(7, 20), batch=2, hq=8, hkv=2, d=64, bs=16, nb=9):
    return cw.lib().cw_rope_append_fp8(q, qs, k, ks, v, vs, rope, n, qo, k8, v8, sk, sv, bt, stride, cud, pld,
                                       None if cu is None else p32(cu), None if pl is None else p32(pl), batch, hq, hkv,
                                       d, bs, nb, None)


@pytest.mark.parametrize("status,change", [
    (E, dict(k=None)), (E, dict(v=None)), (E, dict(k8=None)), (E, dict(v8=None)), (E, dict(sk=None)), (E, dict(sv=None)),
    (E, dict(bt=None)), (E, dict(cud=None)), (E, dict(pld=None)), (E, dict(cu=None)), (E, dict(pl=None)),
    (E, dict(q=None)), (E, dict(qo=None)), (E, dict(rope=None)), (E, dict(hq=0)), (E, dict(hq=-1)), (E, dict(hkv=0)),
    (E, dict(nb=0)), (E, dict(batch=0)), (E, dict(stride=1)), (E, dict(pl=i32(-1, 0))), (E, dict(cu=i32(1, 3, 5))),
    (E, dict(cu=i32(0, 3, 2))), (E, dict(n=21)), (E, dict(ks=120)), (E, dict(vs=132)), (E, dict(qs=504)),
    (E, dict(k=odd)), (E, dict(k8=odd)), (E, dict(qo=odd)), (E, dict(rope=odd)), (U, dict(d=96)), (U, dict(bs=32)),
    (U, dict(hkv=65537, ks=2 ** 23, vs=2 ** 23)),
])
def test_append_refusals(status, change):
    assert _append(**change) == status
    assert cw.last_error()


def test_append_refuses_prompts_that_pass_32_bits():
    """The kernel counts tokens in 32 bits and drops the rows of such a request; the host says so instead."""
    big = 2 ** 31 - 34   # two rows behind it end at 2^31 - 32
    none = dict(q=None, qo=None, rope=None, n=0, stride=2 ** 27 + 4)
    assert _append(cu=i32(0, 3, 5), pl=i32(7, big), **none) == U and "tokens" in cw.last_error()
    assert _append(cu=i32(0, 2 ** 30, 2 ** 30 + 1), pl=i32(2 ** 30 - 16, 0), **none) == U
    assert _append(cu=i32(0, 0, 0), pl=i32(7, big), **none) == cw.CW_OK   # (a request without rows is not touched)


def test_append_of_no_rows_launches_nothing():
    assert _append(cu=i32(0, 0, 0), q=None, qo=None, k=None, v=None) == cw.CW_OK


def _prefill(q=d_, k8=d_, v8=d_, sk=d_, sv=d_, bt=d_, stride=4, cu=i32(0, 3, 5), pl=i32(7, 20), batch=2, hq=8, hkv=2, d=64,
             bs=16, nb=9, scale=0.1, plan="own", plan_dev=d_, out=d_):
    if isinstance(plan, str):
        plan = cw.suffix_prefill_plan(i32(0, 3, 5), i32(7, 20), 8, 2, 64)
    return cw.lib().cw_suffix_prefill_attn_fp8(q, k8, v8, sk, sv, bt, stride, p32(cu), p32(pl), batch, hq, hkv, d, bs, nb,
                                               scale, None if plan is None else p32(plan), plan_dev, out, None)


@pytest.mark.parametrize("status,change", [
    (E, dict(q=None)), (E, dict(k8=None)), (E, dict(v8=None)), (E, dict(sk=None)), (E, dict(sv=None)), (E, dict(bt=None)),
    (E, dict(out=None)), (E, dict(plan=None)), (E, dict(plan_dev=None)), (E, dict(hq=7)), (E, dict(hq=0)), (E, dict(nb=0)),
    (E, dict(batch=0)), (E, dict(stride=1)), (E, dict(scale=0.0)), (E, dict(scale=float("inf"))),
    (E, dict(pl=i32(8, 20))), (E, dict(pl=i32(-7, 20))), (E, dict(cu=i32(0, 2, 5))), (E, dict(hq=16)), (E, dict(q=odd)),
    (E, dict(out=odd)), (E, dict(v8=odd)), (U, dict(d=96)), (U, dict(bs=8)), (U, dict(hq=2 * 129)),
    (E, dict(plan=cw.suffix_prefill_plan(i32(0, 3, 5), i32(7, 20), 8, 2, 64, 2))),
])
def test_prefill_refusals(status, change):
    assert _prefill(**change) == status
    assert cw.last_error()


def _split(ws=d_, wb=1 << 20, splits=2, **kw):
    plan = cw.suffix_prefill_plan(i32(0, 3, 5), i32(7, 20), 8, 2, 64, splits)
    a = dict(q=d_, k8=d_, v8=d_, sk=d_, sv=d_, bt=d_, stride=4, cu=i32(0, 3, 5), pl=i32(7, 20), batch=2, hq=8, hkv=2, d=64,
             bs=16, nb=9, scale=0.1, plan_dev=d_, out=d_)
    assert set(kw) <= set(a)
    a.update(kw)
    return cw.lib().cw_suffix_prefill_attn_split_fp8(
        a["q"], a["k8"], a["v8"], a["sk"], a["sv"], a["bt"], a["stride"], p32(a["cu"]), p32(a["pl"]), a["batch"], a["hq"],
        a["hkv"], a["d"], a["bs"], a["nb"], a["scale"], p32(plan), a["plan_dev"], ws, wb, a["out"], None)


@pytest.mark.parametrize("status,change", [
    (E, dict(ws=None)), (E, dict(ws=odd)), (E, dict(wb=2 * 40 * 65 * 4 - 1)), (E, dict(q=None)), (E, dict(out=None)),
    (E, dict(plan_dev=None)), (E, dict(pl=i32(8, 20))), (E, dict(hq=16)), (E, dict(scale=-1.0)), (U, dict(d=96)),
])
def test_split_prefill_refusals(status, change):
    assert _split(**change) == status
    assert "suffix_prefill_attn_split_fp8" in cw.last_error()


def _decode(q=d_, k8=d_, v8=d_, sk=d_, sv=d_, bt=d_, stride=4, lens=d_, batch=2, hq=8, hkv=2, d=64, bs=16, nb=9, scale=0.1,
            splits=1, ws=None, wb=0, out=d_):
    return cw.lib().cw_decode_attn_fp8(q, k8, v8, sk, sv, bt, stride, lens, batch, hq, hkv, d, bs, nb, scale, splits, ws,
                                       wb, out, None)


@pytest.mark.parametrize("status,change", [
    (E, dict(q=None)), (E, dict(k8=None)), (E, dict(sv=None)), (E, dict(bt=None)), (E, dict(lens=None)),
    (E, dict(out=None)), (E, dict(batch=0)), (E, dict(stride=0)), (E, dict(hq=7)), (E, dict(hq=0)), (E, dict(hkv=0)),
    (E, dict(nb=0)), (E, dict(scale=-1.0)), (E, dict(scale=float("nan"))), (E, dict(splits=0)), (E, dict(splits=65)),
    (E, dict(splits=2)), (E, dict(splits=2, ws=d_, wb=2 * 16 * 65 * 4 - 1)), (E, dict(splits=2, ws=odd, wb=1 << 20)),
    (E, dict(q=odd)), (E, dict(out=odd)), (E, dict(k8=odd)), (U, dict(d=32)), (U, dict(bs=32)), (U, dict(hq=2 * 129)),
    (U, dict(stride=2 ** 27)), (U, dict(batch=2 ** 30, splits=1)), (U, dict(batch=2 ** 23, splits=1)),
])
def test_decode_refusals(status, change):
    assert _decode(**change) == status
    assert cw.last_error()


def test_decode_workspace_and_split_count():
    f = cw.decode_workspace_bytes
    assert f(4, 32, 128, 1) == 0
    assert f(4, 32, 128, 3) == 3 * 128 * 128 * 4 + 3 * 128 * 4
    for bad in ((0, 32, 128, 1), (4, 0, 128, 1), (4, 32, 96, 1), (4, 32, 128, 0), (4, 32, 128, 65)):
        with pytest.raises(cw.CwError):
            f(*bad)
    for b, hq, hkv, n in ((1, 32, 8, 1), (1, 32, 8, 200), (16, 32, 8, 1408), (64, 64, 8, 10368), (1, 4, 1, 10 ** 6)):
        s = cw.decode_split_count(b, hq, hkv, n)
        assert 1 <= s <= 64 and (s == 1 or n // s >= 256)


def test_split_count_keeps_runs_of_512_keys():
    for P, S, most in (([10000], [48], 19), ([700, 3], [64, 1], 1), ([0], [1], 1), ([5000, 5000], [64, 64], 9)):
        cu = np.concatenate([[0], np.cumsum(S)])
        meta = cw.BatchMeta(np.zeros((len(P), 700)), cu, P, 32, 8, 128, device=None)
        n = cw.split_count_fp8(meta)
        assert 1 <= n <= most and n <= cw.split_count(meta)


def test_python_argument_checks():
    """Shapes and types are refused by name before the library is called."""
    x, w = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU memory"):
        cw.add_rms_norm_fp8(x, w, 1e-5)
    f8 = torch.zeros(2, 64, dtype=cw.FP8)
    with pytest.raises(ValueError, match="x8 must be"):
        cw.fp8_linear(f8, x, torch.zeros(32, 48, dtype=cw.FP8), x)
    with pytest.raises(ValueError, match="x_scale must be"):
        cw.fp8_linear(f8, torch.zeros(2, 2), torch.zeros(32, 64, dtype=cw.FP8), x)
    with pytest.raises(ValueError, match="w_scale must be"):
        cw.fp8_linear(f8, torch.zeros(2, 1), torch.zeros(32, 64, dtype=cw.FP8), torch.zeros(2, 1))
    cache = cw.Fp8KvCache(4, 2, 64, device="cpu")
    assert cache.num_blocks == 4 and cache.k.dtype == cw.FP8 and cache.v_scale.shape == (4, 2)
    with pytest.raises(ValueError, match="k and v must both"):
        cw.Fp8KvCache.of(cache.k, cache.v[:2], cache.k_scale, cache.v_scale)
    with pytest.raises(ValueError, match="k_scale and v_scale"):
        cw.Fp8KvCache.of(cache.k, cache.v, cache.k_scale[:1], cache.v_scale)
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="block_table must be"):
        cw.decode_attn_fp8(q, cache, torch.zeros(3, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 0.1)
    with pytest.raises(ValueError, match="seq_lens must be"):
        cw.decode_attn_fp8(q, cache, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 0.1)
    meta = cw.BatchMeta(np.zeros((1, 4)), [0, 2], [5], 8, 2, 64, device=None)
    with pytest.raises(ValueError, match="k must be"):
        cw.rope_append_fp8(meta, q, q, cache)
    with pytest.raises(ValueError, match="q must be"):
        cw.suffix_prefill_attn_fp8(meta, q[:1], cache, 0.1)
    with pytest.raises(ValueError, match="no KV heads"):
        cw.decode_attn_fp8(q, cw.Fp8KvCache(4, 0, 64, device="cpu"), torch.zeros(2, 4, dtype=torch.int32),
                           torch.zeros(2, dtype=torch.int32), 0.1)
    with pytest.raises(TypeError, match="k must be a torch tensor"):
        cw._rows(None, torch.bfloat16, "k", 0)


def test_8_bit_sources_are_built_with_nan_honoured():
    """The header says where NaN codes go; the build's default lets the compiler assume that there are none."""
    from paper_2606_19667_amd import build
    sources = [s for s in build.HIP_SOURCES if "fp8" in s]
    assert len(sources) == 3
    for s in sources:
        honor = [f for f in build.HIP_FLAGS + build.EXTRA_FLAGS.get(s, []) if f.endswith("honor-nans")]
        assert honor[-1] == "-fhonor-nans", s
