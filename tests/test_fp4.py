"""The 4-bit cache without a GPU: pins of its oracle, and the refusals of the calls."""
import copy
import ctypes
import pickle
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import fp4 as F
from oracle import projection as OP
from paper_2606_19667_amd import cw

E, U = cw.CW_EINVAL, cw.CW_EUNSUPPORTED


# ---------------------------------------------------------------- oracle
def test_values_from_the_format():
    """Sign, two exponent bits with bias 1, one mantissa bit; exponent 0 is subnormal."""
    for c in range(16):
        e, m = (c >> 1) & 3, c & 1
        v = (2 + m) * 2.0 ** (e - 2) if e else m * 0.5
        assert F.value(c) == (-v if c & 8 else v)


@pytest.mark.parametrize("x,code", [(0.0, 0), (-0.0, 8), (0.25, 0), (0.2500001, 1), (0.75, 2), (0.7499999, 1), (1.25, 2), (1.75, 4),
                                    (2.5, 4), (3.5, 6), (5.0, 6), (5.0000001, 7), (6.0, 7), (7.0, 7), (100.0, 7), (-0.75, 10),
                                    (-2.6, 13), (-6.5, 15)])
def test_code_of_hand_worked(x, code):
    assert F.code_of(x) == code
    row = np.zeros(32)
    row[3], row[4] = 6.0, x if abs(x) <= 7 else 7.0
    codes, scales = F.round_rows(row)
    assert scales[0] == 127 and codes[4] == code


def test_exponent_closed_forms():
    for amax, e in ((0.0, -100), (7.0, 0), (np.nextafter(7.0, 8), 1), (3.5, -1), (3.5000001, 0), (1e-40, -100),
                    (2.0 ** 127, 125), (7.0 * 2.0 ** 125, 125), (2.0 ** 127.99, 125)):
        assert F.exponent_for(amax) == e


def test_round_rows_is_nearest_and_within_a_step():
    g = np.random.default_rng(1)
    x = g.standard_normal((40, 96)) * np.exp(2 * g.standard_normal((40, 1)))
    codes, scales = F.round_rows(x)
    v = F.values_of(codes, scales)
    s = np.repeat(np.exp2(scales.astype(float) - 127), 32, axis=1)
    for i in range(40):
        for d in range(96):
            assert F.code_of(x[i, d] / s[i, d]) == codes[i, d]
    assert (np.abs(v - x) <= s + 1e-300).all()   # the largest step is 2, and 7 is 1 from 6
    top = np.abs(x).reshape(40, 3, 32).max(-1)
    e = scales.astype(int) - 127
    assert (top <= 7 * np.exp2(e.astype(float))).all() and (top > 7 * np.exp2(e - 1.0)).all()


def test_groups_with_infinite_or_nan_values():
    x = np.ones((4, 64))
    x[0, 5], x[1, 40], x[2, 63], x[3, 0] = np.nan, np.inf, -np.inf, 2.0 ** 128
    codes, scales = F.round_rows(x)
    assert scales.tolist() == [[255, 125], [125, 255], [125, 255], [255, 125]]   # (1 <= 7 * 2^-2)
    assert not codes[0, :32].any() and codes[0, 32] == 6
    assert np.isnan(F.values_of(codes, scales)[1, 32:]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_every_place_of_a_page_is_used_once(D):
    seen = np.zeros(17 * D, int)
    for t in range(16):
        for d in range(D):
            for at in (F.key_byte, F.value_byte):
                seen[at(D, t, d)] += 1          # two codes a byte
        for d in range(0, D, 32):
            for at in (F.key_scale_byte, F.value_scale_byte):
                seen[at(D, t, d)] += 2
    assert (seen == 2).all()


@pytest.mark.parametrize("D", [64, 128])
def test_store_and_unpack(D):
    g = np.random.default_rng(2)
    k, v = g.standard_normal((2, 16, D))
    page = g.integers(0, 256, 17 * D, dtype=np.uint8)
    kept = page.copy()
    for t in (0, 5, 6, 15):
        F.store(page, D, t, k[t], v[t])
    for (codes, scales), (old_c, old_s), x in zip(F.unpack(page, D), F.unpack(kept, D), (k, v)):
        for t in range(16):
            c, s = F.round_rows(x[t]) if t in (0, 5, 6, 15) else (old_c[t], old_s[t])
            assert np.array_equal(codes[t], c) and np.array_equal(scales[t], s)


def test_append_and_logical_rows():
    g = np.random.default_rng(3)
    pages = g.integers(0, 255, (5, 2, 17 * 64), dtype=np.uint8)
    k, v = g.standard_normal((2, 9, 2, 64))
    bt = [[4, 0], [2, -1]]
    after = F.append(pages, k, v, bt, [0, 4, 9], [14, 13])
    kr, vr = F.logical_rows(after, bt[0], 14, 4)
    assert np.array_equal(kr, F.values_of(*F.round_rows(k[:4]))) and np.array_equal(vr, F.values_of(*F.round_rows(v[:4])))
    kr, vr = F.logical_rows(after, bt[1], 13, 5)
    assert np.array_equal(kr[:3], F.values_of(*F.round_rows(k[4:7]))) and not kr[3:].any() and not vr[3:].any()
    assert np.array_equal(after[[1, 3]], pages[[1, 3]])
    assert np.array_equal(F.logical_rows(after, bt[0], 0, 14)[0], F.logical_rows(pages, bt[0], 0, 14)[0])


def test_rotate_is_the_projections_rotation_and_multiplication_of_complex_numbers():
    g = np.random.default_rng(4)
    x = g.standard_normal((3, 2, 64))
    pos = np.array([0, 5, 1000])
    ang = pos[:, None] * 10000.0 ** (-np.arange(32) / 32)
    full = np.stack([np.cos(ang), np.sin(ang)], -1)
    z = (x[..., :32] + 1j * x[..., 32:]) * np.exp(1j * ang)[:, None]
    got = F.rotate(x, full, False)
    assert np.allclose(got, np.concatenate([z.real, z.imag], -1), atol=1e-12)
    assert np.allclose(got, OP.rope(x, pos, 10000.0), atol=1e-9)
    part = F.rotate(x, full[:, :16], True)
    z = (x[..., :32:2] + 1j * x[..., 1:32:2]) * np.exp(1j * ang[:, :16])[:, None]
    assert np.allclose(part[..., :32:2], z.real) and np.allclose(part[..., 1:32:2], z.imag)
    assert np.array_equal(part[..., 32:], x[..., 32:])


@pytest.mark.parametrize("s,codes,scale", [
    # 1.25 + d, -(2.5 - d) and 7 - d of d = 2^-60: 1.5, -2, and 6 at scale 1
    (-2.0 ** -20, [3, 12, 7], 127),
    # 1.25 - d, -(2.5 + d) and 7 + d, which needs the scale 2: halves just below 0.625, above 1.25, above 3.5
    (2.0 ** -20, [1, 11, 6], 128),
    # the ties themselves go to the even code
    (0.0, [2, 12, 7], 127),
])
def test_exact_codes_of_hand_worked(s, codes, scale):
    """Borders of codes and of a scale with a product beside them that lies below the 53 bits of a double."""
    tiny = 2.0 ** -40
    row = np.zeros(32)
    row[:6] = [1.25, tiny, -2.5, tiny, 7.0, -tiny]
    cos_sin = np.stack([np.ones(3), np.full(3, s)], -1)
    turned = F.exact_rotation(row, cos_sin, True)
    assert turned[0] == Fraction(5, 4) - Fraction(tiny) * Fraction(s) and turned[1] == Fraction(tiny) + Fraction(5, 4) * Fraction(s)
    assert F.rotate(row[None, None], cos_sin[None], True)[0, 0, 0] == 1.25   # (what 64 bits make of it)
    got, scales = F.exact_codes(turned)
    assert got[:6:2].tolist() == codes and scales.tolist() == [scale]


def test_exact_codes_are_those_of_64_bits_where_these_hold_the_values():
    g = np.random.default_rng(5)
    x = g.choice([0.0, 0.25, 0.75, -1.25, 2.5, 5.0, 7.0, 3.3, -0.1], (6, 1, 64)) * 2.0 ** g.integers(-4, 5, (6, 1, 1))
    ang = np.stack([g.choice([0.5, 1.0], (6, 16)), g.choice([0.0, -0.25, 2.0 ** -12], (6, 16))], -1)
    for interleaved in (False, True):
        turned = F.rotate(x, ang, interleaved)
        want, scales = F.round_rows(turned)
        for i in range(6):
            exact = F.exact_rotation(x[i, 0], ang[i], interleaved)
            assert [float(u) for u in exact] == turned[i, 0].tolist()
            got, e = F.exact_codes(exact)
            assert np.array_equal(got, np.where(want[i, 0] == 8, 0, want[i, 0])) and np.array_equal(e, scales[i, 0])


# ---------------------------------------------------------------- refusals
d_ = ctypes.c_void_p(4096)
odd = ctypes.c_void_p(4104)
i32 = lambda *v: np.array(v, np.int32)
p32 = lambda a: a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def _append(q=d_, qs=512, k=d_, ks=128, v=d_, vs=128, rope=d_, n=64, rd=64, il=0, qo=ctypes.c_void_p(65536), pages=d_, bt=d_,
            stride=4, cud=d_, pld=d_, cu=i32(0, 3, 5), pl=i32(7, 20), batch=2, hq=8, hkv=2, d=64, bs=16, nb=9):
    return cw.lib().cw_rope_append_fp4(q, qs, k, ks, v, vs, rope, n, rd, il, qo, pages, bt, stride, cud, pld,
                                       None if cu is None else p32(cu), None if pl is None else p32(pl), batch, hq, hkv,
                                       d, bs, nb, None)


@pytest.mark.parametrize("status,change", [
    (E, dict(k=None)), (E, dict(v=None)), (E, dict(pages=None)), (E, dict(bt=None)), (E, dict(cud=None)),
    (E, dict(pld=None)), (E, dict(cu=None)), (E, dict(pl=None)), (E, dict(q=None)), (E, dict(qo=None)),
    (E, dict(rope=None)), (E, dict(hq=0)), (E, dict(hq=-1)), (E, dict(hkv=0)), (E, dict(nb=0)), (E, dict(batch=0)),
    (E, dict(stride=1)), (E, dict(pl=i32(-1, 0))), (E, dict(cu=i32(1, 3, 5))), (E, dict(cu=i32(0, 3, 2))),
    (E, dict(n=21)), (E, dict(rd=0)), (E, dict(rd=24)), (E, dict(rd=80)), (E, dict(rd=-16)), (E, dict(il=2)),
    (E, dict(ks=120)), (E, dict(vs=132)), (E, dict(qs=504)), (E, dict(qs=1024, qo=d_)),
    (E, dict(k=odd)), (E, dict(v=odd)), (E, dict(q=odd)), (E, dict(pages=odd)), (E, dict(qo=odd)), (E, dict(rope=odd)),
    (U, dict(d=96)), (U, dict(bs=32)), (U, dict(hkv=65537, ks=2 ** 23, vs=2 ** 23)),
])
def test_append_refusals(status, change):
    assert _append(**change) == status
    assert cw.last_error()


def test_append_refuses_prompts_that_pass_32_bits():
    big = 2 ** 31 - 34   # two rows behind it end at 2^31 - 32
    none = dict(q=None, qo=None, rope=None, n=0, stride=2 ** 27 + 4)
    assert _append(cu=i32(0, 3, 5), pl=i32(7, big), **none) == U and "tokens" in cw.last_error()
    assert _append(cu=i32(0, 2 ** 30, 2 ** 30 + 1), pl=i32(2 ** 30 - 16, 0), **none) == U
    assert _append(cu=i32(0, 0, 0), pl=i32(7, big), **none) == cw.CW_OK   # (a request without rows is not touched)


def test_append_of_no_rows_launches_nothing():
    assert _append(cu=i32(0, 0, 0), q=None, qo=None, k=None, v=None) == cw.CW_OK


def _rows(pages=d_, bt=d_, stride=4, cud=d_, fd=d_, cu=i32(0, 3, 5), first=i32(7, 20), batch=2, hkv=2, d=64, bs=16, nb=9,
          k=d_, v=d_):
    return cw.lib().cw_cache_rows_fp4(pages, bt, stride, cud, fd, None if cu is None else p32(cu),
                                      None if first is None else p32(first), batch, hkv, d, bs, nb, k, v, None)


@pytest.mark.parametrize("status,change", [
    (E, dict(pages=None)), (E, dict(bt=None)), (E, dict(cud=None)), (E, dict(fd=None)), (E, dict(cu=None)),
    (E, dict(first=None)), (E, dict(hkv=0)), (E, dict(nb=0)), (E, dict(batch=0)), (E, dict(stride=1)),
    (E, dict(first=i32(-1, 0))), (E, dict(cu=i32(0, 3, 2))), (E, dict(k=odd)), (E, dict(v=odd)), (E, dict(pages=odd)),
    (U, dict(d=96)), (U, dict(bs=32)), (U, dict(hkv=65537)),
    (U, dict(first=i32(7, 2 ** 31 - 34), stride=2 ** 27 + 4)),
])
def test_rows_refusals(status, change):
    assert _rows(**change) == status
    assert cw.last_error()


def test_rows_of_nothing_launch_nothing():
    assert _rows(cu=i32(0, 0, 0), k=None, v=None) == cw.CW_OK
    assert _rows(k=None, v=None) == cw.CW_OK


def _prefill(q=d_, pages=d_, bt=d_, stride=4, cu=i32(0, 3, 5), pl=i32(7, 20), batch=2, hq=8, hkv=2, d=64, bs=16, nb=9,
             scale=0.1, plan="own", plan_dev=d_, out=d_):
    if isinstance(plan, str):
        plan = cw.suffix_prefill_plan(i32(0, 3, 5), i32(7, 20), 8, 2, 64)
    return cw.lib().cw_suffix_prefill_attn_fp4(q, pages, bt, stride, p32(cu), p32(pl), batch, hq, hkv, d, bs, nb, scale,
                                               None if plan is None else p32(plan), plan_dev, out, None)


@pytest.mark.parametrize("status,change", [
    (E, dict(q=None)), (E, dict(pages=None)), (E, dict(bt=None)), (E, dict(out=None)), (E, dict(plan=None)),
    (E, dict(plan_dev=None)), (E, dict(hq=7)), (E, dict(hq=0)), (E, dict(nb=0)), (E, dict(batch=0)), (E, dict(stride=1)),
    (E, dict(scale=0.0)), (E, dict(scale=float("inf"))), (E, dict(pl=i32(8, 20))), (E, dict(pl=i32(-7, 20))),
    (E, dict(cu=i32(0, 2, 5))), (E, dict(hq=16)), (E, dict(q=odd)), (E, dict(out=odd)), (E, dict(pages=odd)),
    (U, dict(d=96)), (U, dict(bs=8)), (U, dict(hq=2 * 129)),
    (E, dict(plan=cw.suffix_prefill_plan(i32(0, 3, 5), i32(7, 20), 8, 2, 64, 2))),
])
def test_prefill_refusals(status, change):
    assert _prefill(**change) == status
    assert cw.last_error()


def _split(ws=d_, wb=1 << 20, splits=2, **kw):
    plan = cw.suffix_prefill_plan(i32(0, 3, 5), i32(7, 20), 8, 2, 64, splits)
    a = dict(q=d_, pages=d_, bt=d_, stride=4, cu=i32(0, 3, 5), pl=i32(7, 20), batch=2, hq=8, hkv=2, d=64, bs=16, nb=9,
             scale=0.1, plan_dev=d_, out=d_)
    assert set(kw) <= set(a)
    a.update(kw)
    return cw.lib().cw_suffix_prefill_attn_split_fp4(
        a["q"], a["pages"], a["bt"], a["stride"], p32(a["cu"]), p32(a["pl"]), a["batch"], a["hq"], a["hkv"], a["d"],
        a["bs"], a["nb"], a["scale"], p32(plan), a["plan_dev"], ws, wb, a["out"], None)


@pytest.mark.parametrize("status,change", [
    (E, dict(ws=None)), (E, dict(ws=odd)), (E, dict(wb=2 * 40 * 65 * 4 - 1)), (E, dict(q=None)), (E, dict(out=None)),
    (E, dict(plan_dev=None)), (E, dict(pl=i32(8, 20))), (E, dict(hq=16)), (E, dict(scale=-1.0)), (U, dict(d=96)),
])
def test_split_prefill_refusals(status, change):
    assert _split(**change) == status
    assert "suffix_prefill_attn_split_fp4" in cw.last_error()


def _decode(q=d_, pages=d_, bt=d_, stride=4, lens=d_, batch=2, hq=8, hkv=2, d=64, bs=16, nb=9, scale=0.1, splits=1, ws=None,
            wb=0, out=d_):
    return cw.lib().cw_decode_attn_fp4(q, pages, bt, stride, lens, batch, hq, hkv, d, bs, nb, scale, splits, ws, wb, out,
                                       None)


@pytest.mark.parametrize("status,change", [
    (E, dict(q=None)), (E, dict(pages=None)), (E, dict(bt=None)), (E, dict(lens=None)), (E, dict(out=None)),
    (E, dict(batch=0)), (E, dict(stride=0)), (E, dict(hq=7)), (E, dict(hq=0)), (E, dict(hkv=0)), (E, dict(nb=0)),
    (E, dict(scale=-1.0)), (E, dict(scale=float("nan"))), (E, dict(splits=0)), (E, dict(splits=65)), (E, dict(splits=2)),
    (E, dict(splits=2, ws=d_, wb=2 * 16 * 65 * 4 - 1)), (E, dict(splits=2, ws=odd, wb=1 << 20)), (E, dict(q=odd)),
    (E, dict(out=odd)), (E, dict(pages=odd)), (U, dict(d=32)), (U, dict(bs=32)), (U, dict(hq=2 * 129)),
    (U, dict(stride=2 ** 27)), (U, dict(stride=2 ** 27 - 256)), (U, dict(batch=2 ** 30, splits=1)),
    (U, dict(batch=2 ** 23, splits=1)), (U, dict(batch=2 ** 30, hkv=2 ** 16, hq=2 ** 23, splits=64, ws=d_, wb=2 ** 40)),
])
def test_decode_refusals(status, change):
    assert _decode(**change) == status
    assert cw.last_error()


def test_decode_workspace_and_split_counts():
    f = cw.decode_workspace_bytes_fp4
    assert f(4, 32, 128, 1) == 0
    assert f(4, 32, 128, 3) == 3 * 128 * 128 * 4 + 3 * 128 * 4
    for bad in ((0, 32, 128, 1), (4, 0, 128, 1), (4, 32, 96, 1), (4, 32, 128, 0), (4, 32, 128, 65)):
        with pytest.raises(cw.CwError):
            f(*bad)
    with pytest.raises(cw.CwError, match="too large"):   # (its bytes would pass 64 bits)
        f(2 ** 31 - 1, 2 ** 31 - 1, 128, 64)
    for b, hq, hkv, n in ((1, 32, 8, 1), (1, 32, 8, 200), (16, 32, 8, 1408), (64, 64, 8, 10368), (1, 4, 1, 10 ** 6)):
        assert 1 <= cw.decode_split_count_fp4(b, hq, hkv, n) <= 64
    assert cw.decode_split_count_fp4(1, 32, 8, 1) == 1
    for P, S, most in (([10000], [48], 39), ([0], [1], 1), ([5000, 5000], [64, 64], 19)):
        meta = cw.BatchMeta(np.zeros((len(P), 700)), np.concatenate([[0], np.cumsum(S)]), P, 32, 8, 128, device=None)
        assert 1 <= cw.split_count_fp4(meta) <= most


def test_python_argument_checks():
    """Shapes and types are refused by name before the library is called."""
    cache = cw.Fp4KvCache(4, 2, 64, device="cpu")
    assert cache.num_blocks == 4 and cache.num_kv_heads == 2 and cache.head_dim == 64
    assert cache.pages.dtype == torch.uint8 and cw.Fp4KvCache.of(cache.pages).pages is cache.pages
    for bad in (cache.pages[0], cache.pages[..., :-1]):
        with pytest.raises(ValueError, match="pages must be"):
            cw.Fp4KvCache.of(bad)
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    kv = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q must be"):
        cw.decode_attn_fp4(q[0], cache, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 0.1)
    with pytest.raises(ValueError, match="block_table must be"):
        cw.decode_attn_fp4(q, cache, torch.zeros(3, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 0.1)
    with pytest.raises(ValueError, match="seq_lens must be"):
        cw.decode_attn_fp4(q, cache, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 0.1)
    with pytest.raises(ValueError, match="no KV heads"):
        cw.decode_attn_fp4(q, cw.Fp4KvCache(4, 0, 64, device="cpu"), torch.zeros(2, 4, dtype=torch.int32),
                           torch.zeros(2, dtype=torch.int32), 0.1)
    meta = cw.BatchMeta(np.zeros((1, 4)), [0, 2], [5], 8, 2, 64, device=None)
    with pytest.raises(ValueError, match="k must be"):
        cw.rope_append_fp4(meta, q, kv, cache)
    with pytest.raises(ValueError, match="rope must be"):
        cw.rope_append_fp4(meta, kv, kv, cache, rope=torch.zeros(64, 32))
    with pytest.raises(ValueError, match="q_out without q"):
        cw.rope_append_fp4(meta, kv, kv, cache, rope=torch.zeros(64, 32, 2), q_out=q)
    with pytest.raises(ValueError, match="GPU memory"):
        cw.rope_append_fp4(meta, kv, kv, cache)
    with pytest.raises(ValueError, match="GPU memory"):
        cw.cache_rows_fp4(meta, cache)
    with pytest.raises(ValueError, match="q must be"):
        cw.suffix_prefill_attn_fp4(meta, q[:1], cache, 0.1)
    with pytest.raises(ValueError, match="q must be"):
        cw.suffix_prefill_attn_split_fp4(meta, q[:1], cache, 0.1)
    with pytest.raises(ValueError, match="out must have"):
        cw.suffix_prefill_attn_fp4(meta, q, cache, 0.1, out=q[:1])


def test_4_bit_sources_are_built_with_nan_honoured():
    """The header says where NaN scales go; the build's default lets the compiler assume that there are none."""
    from paper_2606_19667_amd import build
    sources = [s for s in build.HIP_SOURCES if "fp4" in s]
    assert len(sources) == 2
    for s in sources:
        honor = [f for f in build.HIP_FLAGS + build.EXTRA_FLAGS.get(s, []) if f.endswith("honor-nans")]
        assert honor[-1] == "-fhonor-nans", s


def test_the_join_of_runs_is_built_with_nan_honoured():
    """The decode's runs, and the prefill's where they are many, are joined by a kernel of another source: a NaN
    log-sum-exp has to make its row NaN there too."""
    import os
    from paper_2606_19667_amd import build
    homes = []
    for s in build.HIP_SOURCES:
        with open(os.path.join(build.CSRC, s)) as fh:
            if "cw_status cw::decode_join(" in fh.read():
                homes.append(s)
    assert len(homes) == 1
    honor = [f for f in build.HIP_FLAGS + build.EXTRA_FLAGS.get(homes[0], []) if f.endswith("honor-nans")]
    assert honor[-1] == "-fhonor-nans", homes


@pytest.mark.parametrize("again", [copy.copy, copy.deepcopy, lambda m: pickle.loads(pickle.dumps(m))], ids=["copy", "deepcopy", "pickle"])
def test_copies_of_a_used_batch_hand_over_their_own_arrays(again):
    """What a call keeps of a batch's host arrays goes into the library as their address: a copy of the batch, or one
    that another process gets, has to hand over the whole of its own."""
    def address(p):   # (arrays that cannot be written have a pointer, others an object on their memory)
        return ctypes.addressof(p.contents if isinstance(p, ctypes.POINTER(ctypes.c_int32)) else p)

    for writable in (True, False):
        meta = cw.BatchMeta(np.zeros((3, 4)), [0, 2, 5, 9], [5, 0, 7], 8, 2, 64, device=None)
        names = ("cu_host", "plen_host", "plan_host")
        for name in names:
            getattr(meta, name).flags.writeable = writable
            meta._field(name)
        other = again(meta)
        for m in (meta, other):
            for name in names:
                assert address(m._field(name)) == getattr(m, name).ctypes.data, (name, writable)
        other.cu_host = np.array([0, 1, 2, 3], np.int32)   # (and the other one does not follow)
        assert address(other._field("cu_host")) == other.cu_host.ctypes.data
        assert address(meta._field("cu_host")) == meta.cu_host.ctypes.data
