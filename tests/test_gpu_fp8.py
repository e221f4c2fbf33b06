"""GPU parity of the 8-bit layer path against its fp64 oracle (oracle.fp8 and, for
attention over the values a cache stands for, oracle.attention).

Bounds, derived from the roundings (eps/2 of bf16 is 2^-8, a half step of e4m3
is oracle.fp8.step(x) / 2):

* norm: h is compared by its bits. A scale is max|h w| / 448 (one rounding each) times
  the inverse root: a sum of squares of at most 64 terms a thread and 10
  additions over threads, all positive, is off by at most 74 * 2^-24, half of that after the
  root; 2^-16 leaves a factor. A code is the e4m3 value nearest to y / scale up to
  the quotient's own rounding: half a step and 2^-20 of the quotient.
* linear: the output's rounding, 2^-8 |y|; fp32 sums of K products and K / 128 partial sums in
  any order, (K + K / 128 + 4) 2^-23 of the sum of their magnitudes; and what the 8-bit matrix
  instruction cuts: of 8 consecutive products it keeps 13 bits below the exponent of the
  largest (measured: 2^16 + 2^3 is exact in a group, of 2^16 + 2^2 the second is lost, beside
  a product of another group it is not), so 7 products lose up to 2^-13 of the largest each.
  The cuts have either sign: their rms is 3^-1/2 of that, and adds by squares. The rms over an
  output of many rows is held to that plus the rounding's, 12^-1/2 steps = 2^-8.79 |y|, taken
  as 2^-8.5.
* append: q as an output rounding plus 3 * 2^-24 of the products' magnitudes; a
  code half a step plus that. Values that are not rotated and kept rows: equal.
* attention: with A = sum p|v| / sum p, the probabilities' rounding to bf16 before the product
  gives 2^-8 A; the row's sum of the same rounded values (prefill) 2^-8 |o| <= 2^-8 A;
  fp32 scores of magnitude below 64 and the exponential 2^-12 A; the output 2^-8 |o|.
"""
import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import fp8 as F
from paper_2606_19667_amd import cw

pytestmark = pytest.mark.gpu

BS = 16
B8 = 2.0 ** -8
NAN8 = 0x7F


def _say(msg):
    print(msg, flush=True)


def _gen(seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g) * std).to(torch.bfloat16)


def _f64(t):
    return t.detach().float().cpu().double().numpy()


def _codes(t):
    return t.detach().view(torch.uint8).cpu().numpy()


def _bits(t):
    return t.detach().contiguous().view(torch.int16).cpu()


def _within(got, exp, bound, what):
    err = np.abs(got - exp)
    _say(f"{what}: n={err.size} max_err={err.max() if err.size else 0:.3e} "
         f"worst_margin={(err - bound).max() if err.size else -1:.3e}")
    assert np.isfinite(got).all(), what
    assert (err <= bound).all(), (what, float((err - bound).max()))


# ---------------------------------------------------------------- norm
def _check_norm(x, r, w, eps, out8, scales, h, what):
    hx = (x.float() + r.float()).to(torch.bfloat16) if r is not None else x
    assert torch.equal(_bits(h), _bits(hx)), what
    y, s = F.add_rms_norm(_f64(hx), None, _f64(w), eps)
    _within(_f64(scales), s, 2.0 ** -16 * s, what + " scales")
    ratio = y / np.repeat(s, 128, axis=1)[:, :y.shape[1]]
    _within(F.decode(_codes(out8)), ratio, F.step(ratio) / 2 + 2.0 ** -20 * np.abs(ratio), what + " codes")


@pytest.mark.parametrize("rows,hidden", [(1, 16), (3, 80), (5, 512), (7, 528), (2, 1024), (9, 1040), (3, 2048), (4, 2064),
                                         (2001, 1024), (1537, 528), (33, 4096), (5, 4992), (2, 8192), (1, 8208), (3, 16384)])
@pytest.mark.parametrize("residual", [True, False])
def test_norm(rows, hidden, residual):
    _say(f"norm {rows} x {hidden} residual={residual}")
    g = _gen(rows * 7 + hidden)
    x = _normal(g, rows, hidden).cuda()
    r = _normal(g, rows, hidden, std=3.0).cuda() if residual else None
    w = (1 + 0.3 * torch.randn(hidden, generator=g)).to(torch.bfloat16).cuda()
    out8, scales, h = cw.add_rms_norm_fp8(x, w, 1e-5, residual=r)
    assert (h is x) == (not residual)
    _check_norm(x, r, w, 1e-5, out8, scales, h, f"norm {rows}x{hidden}")


def test_norm_strided_rows_and_in_place():
    g = _gen(3)
    odd = _normal(g, 6, 700).cuda()
    res, w = _normal(g, 6, 272).cuda(), _normal(g, 272).cuda()
    with pytest.raises(cw.CwError, match="multiples of 8"):   # rows 700 elements apart are not 16-byte aligned
        cw.add_rms_norm_fp8(odd[:, 8:8 + 272], w, 1e-6, residual=res)
    wide = _normal(g, 6, 704).cuda()
    x = wide[:, 8:8 + 272]
    keep = wide.clone()
    r0 = res.clone()
    out8, scales, h = cw.add_rms_norm_fp8(x, w, 1e-6, residual=res, residual_out=res)
    assert h is res
    _check_norm(x, r0, w, 1e-6, out8, scales, h, "strided, into the residual")
    assert torch.equal(_bits(wide), _bits(keep))
    first = (out8.view(torch.uint8).clone(), scales.clone())
    x2, r2 = x.contiguous(), r0.clone()
    o2, s2, h2 = cw.add_rms_norm_fp8(x2, w, 1e-6, residual=r2, residual_out=x2)
    assert h2 is x2 and torch.equal(_bits(h2), _bits(h)) and torch.equal(_bits(r2), _bits(r0))
    assert torch.equal(o2.view(torch.uint8), first[0]) and torch.equal(s2, first[1])


def test_norm_of_rows_below_the_smallest_scale():
    """max|h w| below 2^-100: zeros with scale 1."""
    x = (_normal(_gen(6), 3, 256).double() * 2.0 ** -104).to(torch.bfloat16).cuda()
    out8, scales, _ = cw.add_rms_norm_fp8(x, torch.ones(256, dtype=torch.bfloat16).cuda(), 1e-5)
    assert not F.decode(_codes(out8)).any() and (scales == 1).all()


@pytest.mark.parametrize("hidden", [256, 4096])
def test_norm_of_the_largest_values(hidden):
    x = (_normal(_gen(8), 4, hidden).double().clamp(-3, 3) * 1e38).to(torch.bfloat16).cuda()
    w = _normal(_gen(9), hidden).cuda()
    _check_norm(x, None, w, 1e-5, *cw.add_rms_norm_fp8(x, w, 1e-5), "values of 1e38")


def test_norm_extreme_rows():
    """Zeros, rows whose squares leave fp32, tiny rows, one infinity, one NaN, a NaN weight."""
    g = _gen(4)
    x = _normal(g, 8, 400)
    x[0] = 0
    x[1] *= 1e30
    x[2] *= 1e38
    x[3] *= 1e-30
    x[4, 7] = float("inf")
    x[5, 300] = float("nan")
    x[6, 128:256] = 0
    w = _normal(g, 400)
    w[390] = float("nan")
    xd, wd = x.cuda(), w.cuda()
    out8, scales, _ = cw.add_rms_norm_fp8(xd, wd, 1e-5)
    torch.cuda.synchronize()
    val, s = F.decode(_codes(out8)), _f64(scales)
    # (row 2 has an infinity: its largest draw is above 3.39, and 3.39e38 is bf16's largest value)
    assert torch.isinf(x[2]).any()
    for r in (2, 4, 5):
        assert np.isnan(val[r]).all() and (s[r] == 1).all()
    assert np.isnan(val[:, 390]).all()
    assert not val[0, :384].any() and (s[0] == 1).all()
    # (row 3 is tiny beside eps, but 1e-30 is above 2^-100 = 7.9e-31: it is coded like any other)
    assert not val[6, 128:256].any() and s[6, 1] == 1
    w0 = w.clone()
    w0[390] = 0
    y, es = F.add_rms_norm(_f64(x), None, _f64(w0), 1e-5)
    for r in (1, 3, 7):
        _within(s[r], es[r], 2.0 ** -16 * es[r], f"row {r} scales")
        ratio = (y[r] / np.repeat(es[r], 128)[:400])
        keep = np.arange(400) != 390
        _within(val[r][keep], ratio[keep], (F.step(ratio) / 2 + 2.0 ** -20 * np.abs(ratio))[keep], f"row {r} codes")


# ---------------------------------------------------------------- linear
def _quantised(g, n, k, spread=1.0):
    """e4m3 [n, k] and fp32 scales [n or blocks, blocks of 128]."""
    return (torch.randn(n, k, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)


def _scales(g, n, k, lo=-12, hi=2):
    return torch.exp2(torch.rand(n, -(-k // 128), generator=g) * (hi - lo) + lo)


def _check_linear(rows, hidden, feats, bias, seed):
    g = _gen(seed)
    x8, w8 = _quantised(g, rows, hidden), _quantised(g, feats, hidden)
    xs, ws = _scales(g, rows, hidden), _scales(g, -(-feats // 128), hidden)
    b = _normal(g, feats, std=50.0) if bias else None
    got = cw.fp8_linear(x8.cuda(), xs.cuda(), w8.cuda(), ws.cuda(), None if b is None else b.cuda())
    assert got.shape == (rows, feats) and got.dtype == torch.bfloat16
    exp, mag = F.linear(_f64(x8), _f64(xs), _f64(w8), _f64(ws), None if b is None else _f64(b))
    terms = hidden + hidden / 128 + 4
    cut, cut2 = F.linear_cut(_f64(x8), _f64(xs), _f64(w8), _f64(ws))
    _within(_f64(got), exp, B8 * np.abs(exp) + terms * 2.0 ** -23 * mag + 7 * 2.0 ** -13 * cut,
            f"linear {rows}x{hidden}x{feats}")
    if exp.size >= 10000:
        rms, most = (float(np.sqrt((v ** 2).mean())) for v in (_f64(got) - exp, exp))
        assert rms <= 2.0 ** -8.5 * most + float(np.sqrt(7 / 3 * cut2.mean())) * 2.0 ** -13


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 63, 64, 65, 127, 129, 200, 300])
@pytest.mark.parametrize("hidden,feats", [(16, 16), (144, 304), (256, 128), (1040, 48), (512, 656)])
def test_linear(rows, hidden, feats):
    _say(f"linear {rows} x {hidden} x {feats}")
    _check_linear(rows, hidden, feats, (rows + feats) % 2 == 0, rows * 1000 + hidden)


@pytest.mark.parametrize("rows,hidden,feats", [(1, 4096, 6144), (16, 4096, 6144), (40, 3584, 4608), (96, 4096, 1024),
                                               (300, 2064, 2064), (1100, 384, 2320), (700, 128, 4608)])
def test_linear_model_sizes(rows, hidden, feats):
    _say(f"linear {rows} x {hidden} x {feats}")
    _check_linear(rows, hidden, feats, rows % 2 == 0, rows + feats)


def test_linear_rows_alone_equal_rows_in_a_batch():
    """A row's bits do not depend on the rows beside it, whatever tile the batch takes."""
    g = _gen(9)
    K, N, T = 4096, 1536, 2100
    x8, xs = _quantised(g, T, K).cuda(), _scales(g, T, K).cuda()
    w8, ws = _quantised(g, N, K).cuda(), _scales(g, N // 128, K).cuda()
    all_rows = cw.fp8_linear(x8, xs, w8, ws)
    for n in (1, 7, 16, 31, 48, 64, 100, 128, 200, 256, 500, 1000):
        part = cw.fp8_linear(x8[:n].contiguous(), xs[:n].contiguous(), w8, ws)
        assert torch.equal(_bits(part), _bits(all_rows[:n])), n
    one = cw.fp8_linear(x8[777:778], xs[777:778], w8, ws)
    assert torch.equal(_bits(one[0]), _bits(all_rows[777]))


@pytest.mark.parametrize("rows,hidden,feats", [(4099, 400, 6160), (2100, 2064, 4112), (5000, 1040, 1040),
                                               (16000, 272, 400), (2000, 4112, 6160)])
def test_linear_many_rows(rows, hidden, feats):
    """Large tiles, with several tiles a workgroup, cut rows, features and columns: sampled rows against
    fp64, and all rows' bits equal to those of the same rows in calls of 96."""
    _say(f"linear {rows} x {hidden} x {feats}")
    g = _gen(rows)
    x8, w8 = _quantised(g, rows, hidden), _quantised(g, feats, hidden)
    xs, ws = _scales(g, rows, hidden), _scales(g, -(-feats // 128), hidden)
    b = _normal(g, feats, std=50.0)
    dev = [t.cuda() for t in (x8, xs, w8, ws, b)]
    buf = torch.full((rows + 300, feats), 3.0, dtype=torch.bfloat16, device="cuda")
    got = cw.fp8_linear(*dev, out=buf[:rows])
    torch.cuda.synchronize()
    assert (buf[rows:] == 3).all()
    for t in range(0, rows, 96):
        part = cw.fp8_linear(dev[0][t:t + 96], dev[1][t:t + 96], *dev[2:])
        assert torch.equal(part.view(torch.int16), got[t:t + 96].view(torch.int16)), t
    pick = [0, 1, 255, 256, 1023, rows - 257, rows - 2, rows - 1]
    exp, mag = F.linear(_f64(x8[pick]), _f64(xs[pick]), _f64(w8), _f64(ws), _f64(b))
    cut = F.linear_cut(_f64(x8[pick]), _f64(xs[pick]), _f64(w8), _f64(ws))[0]
    _within(_f64(got[pick]), exp, B8 * np.abs(exp) + (hidden + hidden / 128 + 4) * 2.0 ** -23 * mag + 7 * 2.0 ** -13 * cut,
            "sampled rows")


def test_linear_nan_code_stays_in_its_row():
    g = _gen(10)
    x8 = _quantised(g, 40, 256)
    x8.view(torch.uint8)[11, 130] = NAN8
    w8, xs, ws = _quantised(g, 144, 256), _scales(g, 40, 256), _scales(g, 2, 256)
    got = _f64(cw.fp8_linear(x8.cuda(), xs.cuda(), w8.cuda(), ws.cuda()))
    assert np.isnan(got[11]).all() and np.isfinite(np.delete(got, 11, axis=0)).all()


def test_linear_into_rows_of_a_larger_buffer():
    """Rows behind the last one of `out` keep their bytes."""
    g = _gen(11)
    buf = torch.full((70, 48), 3.0, dtype=torch.bfloat16, device="cuda")
    x8, w8 = _quantised(g, 50, 96).cuda(), _quantised(g, 48, 96).cuda()
    cw.fp8_linear(x8, _scales(g, 50, 96).cuda(), w8, _scales(g, 1, 96).cuda(), out=buf[:50])
    assert (buf[50:] == 3).all() and not (buf[:50] == 3).all()


# ---------------------------------------------------------------- a cache and its batch
class Batch:
    """A ragged batch over an 8-bit cache with random placement and NaN behind every prompt."""

    def __init__(self, hq, hkv, D, P, S, seed, extra=3, spread=2.0, held=None):
        self.hq, self.hkv, self.D, self.P, self.S = hq, hkv, D, list(P), list(S)
        self.L = [p + s for p, s in zip(P, S)]
        self.cu = np.concatenate([[0], np.cumsum(S)]).astype(np.int32)
        self.T = int(self.cu[-1])
        g = self.g = _gen(seed)
        nblk = [-(-n // BS) for n in self.L]
        self.nb, self.stride = sum(nblk) + extra, max(1, max(nblk))
        order = torch.randperm(self.nb, generator=g).numpy()
        self.bt, o = np.full((len(P), self.stride), -1, np.int32), 0
        for r, n in enumerate(nblk):
            self.bt[r, :n] = order[o:o + n]
            o += n
        held = self.L if held is None else held   # tokens in the cache at the start
        codes = [torch.randint(0, 256, (self.nb, hkv, BS, D), generator=g, dtype=torch.uint8) for _ in range(2)]
        self.scale = [torch.exp2(torch.randn(self.nb, hkv, generator=g) * spread - 7) for _ in range(2)]
        x = [torch.randn(self.nb, hkv, BS, D, generator=g).mul(100).clamp(-448, 448).to(cw.FP8).view(torch.uint8)
             for _ in range(2)]
        for r, n in enumerate(held):
            for j in range(-(-n // BS)):
                k = min(BS, n - j * BS)
                for c, v in zip(codes, x):
                    c[self.bt[r, j], :, :k] = v[self.bt[r, j], :, :k]
                    c[self.bt[r, j], :, k:] = NAN8
        self.codes = codes
        self.cache = cw.Fp8KvCache.of(*(c.cuda().view(cw.FP8) for c in codes), *(s.cuda() for s in self.scale))

    def meta(self):
        return cw.BatchMeta(self.bt, self.cu, self.P, self.hq, self.hkv, self.D)

    def rows(self, which, r):
        """Request r's keys (0) or values (1) as the starting cache holds them, [L, Hkv, D]."""
        return F.logical_rows(F.decode(self.codes[which].numpy()), self.scale[which].double().numpy(), self.bt[r],
                              self.L[r])

    def queries(self, n=None):
        return _normal(self.g, self.T if n is None else n, self.hq, self.D)


# ---------------------------------------------------------------- append
def _check_append(b, q, k, v, rope, q_out, what, base=None):
    pos = np.concatenate([np.arange(p, p + s) for p, s in zip(b.P, b.S)]) if b.T else np.zeros(0, int)

    def turned(u):
        """(rotated, sum of the products' magnitudes)"""
        u = _f64(u)
        if rope is None:
            return u, np.abs(u) * 0
        c, s = (_f64(rope)[pos][:, None, :, i] for i in (0, 1))
        x, y = u[..., :b.D // 2], u[..., b.D // 2:]
        rot = np.concatenate([x * c - y * s, y * c + x * s], -1)
        mag = np.concatenate([np.abs(x * c) + np.abs(y * s), np.abs(y * c) + np.abs(x * s)], -1)
        return rot, mag

    if q is not None:
        rot, mag = turned(q)
        _within(_f64(q_out), rot, B8 * np.abs(rot) + 3 * 2.0 ** -24 * mag, what + " q")
    for name, which, new in (("k", 0, k), ("v", 1, v)):
        rows, mag = turned(new) if which == 0 else (_f64(new), None)
        before, scale = F.decode(b.codes[which].numpy()), b.scale[which].double().numpy()
        values, scales = F.append(before, scale, rows, b.bt, b.cu, b.P)
        got = F.decode(_codes(getattr(b.cache, name)))
        gs = _f64(getattr(b.cache, name + "_scale"))
        assert np.array_equal(gs, scales), what
        if which == 1 or rope is None:
            assert np.array_equal(got, values, equal_nan=True), what
            continue
        # rotated keys: nearest code up to the rotation's fp32 error
        exact = np.full(got.shape, np.nan)
        slack = np.zeros(got.shape)
        mask = np.zeros(got.shape, bool)
        for r in range(len(b.P)):
            for i in range(b.S[r]):
                t = b.P[r] + i
                blk = b.bt[r, t // BS]
                if 0 <= blk < b.nb:
                    at = (blk, slice(None), t % BS)
                    exact[at] = rows[b.cu[r] + i] / scales[blk][:, None]
                    slack[at] = 3 * 2.0 ** -24 * mag[b.cu[r] + i] / scales[blk][:, None]
                    mask[at] = True
        assert np.array_equal(got[~mask], values[~mask], equal_nan=True), what
        _within(got[mask], exact[mask], (F.step(exact) / 2 + slack)[mask], what + " k")


APPEND_CASES = [
    # hq, hkv, D, prefix lengths, suffix lengths
    (4, 1, 64, [0], [1]),
    (4, 1, 64, [64], [32]),
    (8, 2, 128, [0, 5, 16, 31, 47], [1, 1, 1, 1, 1]),
    (7, 7, 64, [3, 0, 16, 40], [17, 0, 16, 50]),
    (28, 4, 128, [100, 15, 0, 1], [29, 2, 33, 1]),
    (32, 8, 128, [13] * 70, [1] * 70),
    (16, 4, 64, [0, 1, 2, 3], [200, 100, 15, 14]),
]


@pytest.mark.parametrize("hq,hkv,D,P,S", APPEND_CASES)
def test_append(hq, hkv, D, P, S):
    _say(f"append {hq}/{hkv} D={D} P={P[:5]} S={S[:5]}")
    b = Batch(hq, hkv, D, P, S, seed=sum(P) + hq, held=P)
    qkv = _normal(b.g, b.T, (hq + 2 * hkv) * D, std=2.0).cuda()
    q, k, v = (x.view(b.T, -1, D) for x in qkv.split([hq * D, hkv * D, hkv * D], 1))
    rope = torch.from_numpy(cw.rope_table(max(b.L) + 1, D, 10000.0)).cuda()
    q_out = cw.rope_append_fp8(b.meta(), k, v, b.cache, q=q, rope=rope)
    torch.cuda.synchronize()
    _check_append(b, q, k, v, rope, q_out, f"append {hq}/{hkv}")


def test_append_without_rotation_values_and_growth():
    """Unrotated keys: every code is the oracle's. Rows of rising size raise the scale of a
    block token by token; infinities, NaN and zeros; one head of tiny values."""
    b = Batch(4, 2, 64, [0], [1], seed=5, held=[0], extra=2)
    meta_bt = b.bt
    codes, scale = [c.numpy().copy() for c in b.codes], [s.double().numpy() for s in b.scale]
    val = [F.decode(c) for c in codes]
    rng = np.random.default_rng(0)
    for t in range(16):
        k = (rng.normal(size=(1, 2, 64)) * 1.7 ** t).astype(np.float32)
        v = (rng.normal(size=(1, 2, 64)) * 2.0 ** (-t)).astype(np.float32)
        k[0, 1] *= 1e-33
        if t == 3:
            k[0, 0, 5], k[0, 0, 6], v[0, 1, 0] = np.inf, np.nan, -np.inf
        if t == 9:
            v[:] = 0
        kt, vt = (torch.from_numpy(x).to(torch.bfloat16) for x in (k, v))
        meta = cw.BatchMeta(meta_bt, [0, 1], [t], 4, 2, 64)
        assert cw.rope_append_fp8(meta, kt.cuda(), vt.cuda(), b.cache) is None
        for i, x in enumerate((kt, vt)):
            val[i], scale[i] = F.append(val[i], scale[i], _f64(x), meta_bt, [0, 1], [t])
        for i, (c, s) in enumerate(((b.cache.k, b.cache.k_scale), (b.cache.v, b.cache.v_scale))):
            assert np.array_equal(_f64(s), scale[i]), t
            assert np.array_equal(F.decode(_codes(c)), val[i], equal_nan=True), t


def test_append_drops_blocks_outside_the_pool():
    b = Batch(8, 2, 128, [10, 20], [30, 20], seed=6, held=[10, 20])
    b.bt[0, 1], b.bt[1, 2] = -1, b.nb
    meta = b.meta()
    k, v = _normal(b.g, b.T, 2, 128), _normal(b.g, b.T, 2, 128)
    cw.rope_append_fp8(meta, k.cuda(), v.cuda(), b.cache)
    torch.cuda.synchronize()
    _check_append(b, None, k, v, None, None, "foreign blocks")


@pytest.mark.parametrize("D", [64, 128])
def test_append_into_blocks_whose_scale_is_no_power_of_two(D):
    """Rows that follow others in a block of any scale: quotients (and, where the scale is raised, products of the
    earlier codes) a rounding away from halfway between two codes go to the nearest code, not to the even one."""
    halves = [t for t in (F.decode(np.arange(0x20, 0x70, 5)) + F.decode(np.arange(0x21, 0x71, 5))) / 2]
    near = [np.float32(1 / t) for t in halves] + [np.float32(t / 1.125) for t in halves]
    scales = [f(x) for x in near for f in (lambda x: np.nextafter(x, np.float32(0)), np.float32,
                                           lambda x: np.nextafter(x, np.float32(9e9)))]
    n = len(scales)
    g = _gen(93)
    signs = (torch.randint(0, 2, (n, 1, D), generator=g) * 2 - 1).float()
    rows = torch.exp2(torch.randint(-4, 5, (n, 1, D), generator=g).float()) * signs
    for grow in (False, True):
        codes = [torch.randint(0, 256, (n, 1, BS, D), generator=g, dtype=torch.uint8) for _ in range(2)]
        for c in codes:   # earlier codes 1.125 and others; behind the new row NaN
            c[:, :, :7, ::2] = 0x39
            c[:, :, 8:] = NAN8
        scale = [torch.tensor(np.array(scales)).view(n, 1).clone() for _ in range(2)]
        cache = cw.Fp8KvCache.of(*(c.cuda().view(cw.FP8) for c in codes), *(x.cuda() for x in scale))
        new = rows.clone()
        if grow:   # the scale becomes the smallest power of two above it, times 4
            up = torch.exp2(torch.floor(torch.log2(scale[0].double())) + 3).float()
            new[:, :, :1] = (up * 448).view(n, 1, 1).flip(0)   # (request r writes block n - 1 - r)
        new = new.to(torch.bfloat16)
        bt = np.arange(n, dtype=np.int32)[::-1].copy()[:, None]
        meta = cw.BatchMeta(bt, np.arange(n + 1), [7] * n, 1, 1, D)
        cw.rope_append_fp8(meta, new.cuda(), (-new).cuda(), cache)
        for c, s, x, got, gs in ((codes[0], scale[0], new, cache.k, cache.k_scale),
                                 (codes[1], scale[1], -new, cache.v, cache.v_scale)):
            values, es = F.append(F.decode(c.numpy()), s.double().numpy(), x, bt, np.arange(n + 1), [7] * n)
            assert np.array_equal(_f64(gs), es) and (es > s.double().numpy()).all() == grow
            assert np.array_equal(F.decode(_codes(got)), values, equal_nan=True), grow


def test_append_captured_and_replayed_with_growing_prefixes():
    """A decode step's append in a HIP graph: each replay reads the prefix lengths and the
    table from device memory and equals an eager call at those lengths."""
    P = [14, 0, 31]
    b, e = (Batch(8, 2, 64, [p + 6 for p in P], [1, 1, 1], seed=7, held=P) for _ in range(2))
    rope = torch.from_numpy(cw.rope_table(64, 64, 10000.0)).cuda()
    meta = cw.BatchMeta(b.bt, [0, 1, 2, 3], P, 8, 2, 64)
    q, k, v = (torch.empty(3, h, 64, dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2))
    q_out = torch.empty_like(q)
    for t in (q, k, v):
        t.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        cw.rope_append_fp8(meta, k, v, b.cache, q=q, rope=rope, q_out=q_out)
    for step in range(5):
        new = [_normal(b.g, *t.shape).cuda() for t in (q, k, v)]
        for t, x in zip((q, k, v), new):
            t.copy_(x)
        meta.plen.copy_(torch.tensor([p + step for p in P], dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        em = cw.BatchMeta(e.bt, [0, 1, 2, 3], [p + step for p in P], 8, 2, 64)
        eq = cw.rope_append_fp8(em, new[1], new[2], e.cache, q=new[0], rope=rope)
        torch.cuda.synchronize()
        assert torch.equal(_bits(q_out), _bits(eq)), step
        for n in ("k", "v"):
            assert np.array_equal(_codes(getattr(b.cache, n)), _codes(getattr(e.cache, n))), step
            assert torch.equal(getattr(b.cache, n + "_scale"), getattr(e.cache, n + "_scale")), step


# ---------------------------------------------------------------- prefill attention
def _check_attention(got, q, k, v, prefix, scale, what):
    exp = OA.suffix_prefill_attention(q, k, v, prefix, scale)
    mag = OA.suffix_prefill_attention(q, k, np.abs(v), prefix, scale)
    _within(got, exp, (2 * B8 + 2.0 ** -12) * mag + B8 * np.abs(exp), what)


PREFILL_CASES = [
    (4, 1, 64, [64], [32]),
    (1, 1, 128, [0], [1]),
    (8, 8, 64, [0, 5, 0, 33], [1, 70, 0, 15]),
    (8, 2, 128, [16, 100, 0, 63], [65, 1, 130, 64]),
    (28, 4, 128, [0, 17, 200], [40, 37, 5]),
    (16, 1, 64, [3, 129], [20, 64]),
    (128, 1, 64, [31], [5]),
    (12, 4, 128, [500, 0], [90, 257]),
    (5, 1, 128, [47], [100]),
]


@pytest.mark.parametrize("hq,hkv,D,P,S", PREFILL_CASES)
def test_prefill(hq, hkv, D, P, S):
    _say(f"prefill {hq}/{hkv} D={D} P={P} S={S}")
    b = Batch(hq, hkv, D, P, S, seed=hq + sum(S), spread=0.5)
    q = b.queries()
    qd = q.cuda()
    out = torch.full_like(qd, 9.0)
    got = cw.suffix_prefill_attn_fp8(b.meta(), qd, b.cache, D ** -0.5, out=out)
    torch.cuda.synchronize()
    assert got is out
    for r in range(len(P)):
        rows = slice(b.cu[r], b.cu[r + 1])
        if S[r]:
            _check_attention(_f64(out[rows]), _f64(q[rows]), b.rows(0, r), b.rows(1, r), P[r], D ** -0.5,
                             f"prefill {hq}/{hkv} r{r}")


@pytest.mark.parametrize("D", [64, 128])
def test_prefill_scales_of_any_size(D):
    """Scales that differ by 2^20 between blocks and are no powers of two, rising scores that
    move the exponent base at every step, and a block outside the pool."""
    b = Batch(8, 2, D, [400], [70], seed=12, spread=0.0)
    rng = np.random.default_rng(1)
    for r, which in ((0, 0), (0, 1)):
        s = b.scale[which]
        for j in range(b.stride):
            s[b.bt[0, j]] = float(2.0 ** -7 * (1 + j / 8) * rng.uniform(0.9, 1.1)) if which == 0 else \
                float(2.0 ** rng.uniform(-14, 6))
    b.bt[0, 5] = -1
    b.bt[0, 9] = b.nb + 100
    cache = cw.Fp8KvCache.of(b.cache.k, b.cache.v, *(s.cuda() for s in b.scale))
    q = b.queries()
    out = cw.suffix_prefill_attn_fp8(b.meta(), q.cuda(), cache, D ** -0.5)
    torch.cuda.synchronize()
    _check_attention(_f64(out), _f64(q), b.rows(0, 0), b.rows(1, 0), 400, D ** -0.5, f"scales D={D}")


def test_prefill_nan_code_reaches_only_rows_that_see_it():
    b = Batch(4, 1, 64, [20], [40], seed=13, spread=0.0)
    b.codes[0][b.bt[0, 2], 0, 3, 7] = NAN8      # key 35
    cache = cw.Fp8KvCache.of(b.codes[0].cuda().view(cw.FP8), b.cache.v, b.cache.k_scale, b.cache.v_scale)
    out = _f64(cw.suffix_prefill_attn_fp8(b.meta(), b.queries().cuda(), cache, 0.125))
    assert np.isfinite(out[:15]).all() and np.isnan(out[15:]).all()


def test_prefill_leaves_other_rows_and_foreign_plans():
    """Rows of `out` behind the batch keep their bytes; a device plan of another batch computes nothing."""
    b = Batch(8, 2, 128, [30], [50], seed=14, spread=0.0)
    meta, q = b.meta(), b.queries().cuda()
    buf = torch.full((60, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    cw.suffix_prefill_attn_fp8(meta, q, b.cache, 0.1, out=buf[:50])
    torch.cuda.synchronize()
    assert (buf[50:] == 5).all() and not (buf[:50] == 5).all()
    meta.plan = cw.BatchMeta(b.bt, b.cu, [14], 8, 2, 128).plan
    buf.fill_(5.0)
    cw.suffix_prefill_attn_fp8(meta, q, b.cache, 0.1, out=buf[:50])
    torch.cuda.synchronize()
    assert (buf == 5).all()


@pytest.mark.parametrize("D,hq,hkv,P,S", [(128, 32, 8, 1000, 700), (64, 16, 4, 2000, 333), (128, 28, 4, 77, 1500)])
def test_prefill_long_sampled_rows(D, hq, hkv, P, S):
    _say(f"prefill long D={D}")
    b = Batch(hq, hkv, D, [P, 16], [S, 100], seed=15, spread=0.5)
    q = b.queries()
    out = _f64(cw.suffix_prefill_attn_fp8(b.meta(), q.cuda(), b.cache, D ** -0.5))
    k, v, qf = b.rows(0, 0), b.rows(1, 0), _f64(q)
    for i in (0, 1, 63, 64, S // 2, S - 2, S - 1):
        L = P + i + 1
        _check_attention(out[i:i + 1], qf[i:i + 1], k[:L], v[:L], P + i, D ** -0.5, f"row {i}")


@pytest.mark.parametrize("hq,hkv,D,P,S", [(4, 1, 64, [9001, 0, 4096], [70, 33, 16]), (2, 2, 128, [4100, 8175], [20, 3]),
                                          (128, 2, 64, [4030, 60, 4159, 17], [70, 9, 1, 66])])
def test_prefill_of_more_keys_than_a_run_of_table_words(hq, hkv, D, P, S):
    """Prompts of 63 to 142 steps of 64 keys: the kernel takes table words and scales 64 steps at a time."""
    _say(f"prefill {hq}/{hkv} D={D} P={P} S={S}")
    b = Batch(hq, hkv, D, P, S, seed=61, spread=0.5)
    q = b.queries()
    out = cw.suffix_prefill_attn_fp8(b.meta(), q.cuda(), b.cache, D ** -0.5)
    torch.cuda.synchronize()
    for r in range(len(P)):
        rows = slice(b.cu[r], b.cu[r + 1])
        _check_attention(_f64(out[rows]), _f64(q[rows]), b.rows(0, r), b.rows(1, r), P[r], D ** -0.5, f"r{r}")


SPLIT_CASES = [
    (8, 2, 128, [1000, 0, 63], [17, 5, 1]),
    (28, 4, 128, [700, 40], [40, 3]),
    (4, 1, 64, [5000, 3, 4100], [9, 70, 64]),
    (128, 2, 64, [130], [5]),
]


@pytest.mark.parametrize("hq,hkv,D,P,S", SPLIT_CASES)
@pytest.mark.parametrize("splits", [None, 1, 2, 7, 64])
def test_prefill_split(hq, hkv, D, P, S, splits):
    """Runs of keys, some of them empty (short prompts) or unseen by some rows, joined."""
    _say(f"split prefill {hq}/{hkv} D={D} P={P} S={S} x{splits}")
    b = Batch(hq, hkv, D, P, S, seed=71 + hq, spread=0.5)
    q, meta = b.queries(), b.meta()
    n = cw.split_count_fp8(meta) if splits is None else splits
    ws = torch.full((cw.split_workspace_bytes(meta, n) + 64,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN
    out = torch.full((b.T + 3, hq, D), 9.0, dtype=torch.bfloat16, device="cuda")
    cw.suffix_prefill_attn_split_fp8(meta, q.cuda(), b.cache, D ** -0.5, num_splits=splits, workspace=ws, out=out[:b.T])
    torch.cuda.synchronize()
    assert (out[b.T:] == 9).all() and (ws[-64:] == 0xFF).all()
    for r in range(len(P)):
        rows = slice(b.cu[r], b.cu[r + 1])
        _check_attention(_f64(out[rows]), _f64(q[rows]), b.rows(0, r), b.rows(1, r), P[r], D ** -0.5, f"r{r}")


def test_prefill_split_nan_and_capture():
    """A NaN key code reaches the rows that see it, whichever run holds it; two captured calls with workspaces
    that they allocate themselves, replayed with other queries between eager calls, have the eager bits."""
    b = Batch(4, 1, 64, [600], [40], seed=72, spread=0.0)
    b.codes[0][b.bt[0, 38], 0, 7, 7] = NAN8      # key 615
    cache = cw.Fp8KvCache.of(b.codes[0].cuda().view(cw.FP8), b.cache.v, b.cache.k_scale, b.cache.v_scale)
    out = _f64(cw.suffix_prefill_attn_split_fp8(b.meta(), b.queries().cuda(), cache, 0.125, num_splits=4))
    assert np.isfinite(out[:15]).all() and np.isnan(out[15:]).all()
    meta = b.meta()
    sets = []
    for n in (3, 5):
        meta.split_plan(n)   # (its copy to the device is not for a graph)
        q = torch.zeros(40, 4, 64, dtype=torch.bfloat16, device="cuda")
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            got = cw.suffix_prefill_attn_split_fp8(meta, q, b.cache, 0.125, num_splits=n)
        sets.append((n, q, graph, got))
    for step in range(4):
        want = []
        for n, q, _, _ in sets:
            q.copy_(b.queries().cuda())
            want.append(cw.suffix_prefill_attn_split_fp8(meta, q, b.cache, 0.125, num_splits=n))
        torch.cuda.synchronize()
        for s in sets:
            s[2].replay()
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            assert torch.equal(_bits(s[3]), _bits(w)), step


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("D", [64, 128])
def test_prefill_ends_beside_values_out_of_range(D, splits):
    """One head's value scales are 2^126, so its rows' sums leave fp32 and its outputs are no numbers; one of
    its query rows is NaN. The call ends, the NaN row is NaN, and the other head's rows are right."""
    _say(f"out of range D={D} splits={splits}")
    b = Batch(8, 2, D, [70], [40], seed=81, spread=0.0)
    b.scale[1][:, 1] = 2.0 ** 126
    cache = cw.Fp8KvCache.of(b.cache.k, b.cache.v, b.cache.k_scale, b.scale[1].cuda())
    q = b.queries()
    q[3, 4:] = float("nan")
    meta, qd = b.meta(), q.cuda()
    got = _f64(cw.suffix_prefill_attn_fp8(meta, qd, cache, D ** -0.5) if splits == 1 else
               cw.suffix_prefill_attn_split_fp8(meta, qd, cache, D ** -0.5, num_splits=splits))
    assert np.isnan(got[3, 4:]).all()
    _check_attention(got[:, :4], _f64(q[:, :4]), b.rows(0, 0)[:, :1], b.rows(1, 0)[:, :1], 70, D ** -0.5, f"D={D}")


@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("hq,hkv,D,key", [(8, 2, 128, 5), (8, 2, 128, 270), (14, 2, 64, 270), (2, 2, 64, 620), (2, 2, 64, 19)])
def test_prefill_nan_value_codes(hq, hkv, D, key, splits):
    """A NaN value code of one KV head makes its column NaN in that head's rows that see it. What else it
    may reach are the same column and head in earlier rows, at most 256 / (Hq / Hkv) + 62 tokens before."""
    P, S, col = 20, 700, 9
    b = Batch(hq, hkv, D, [P, 33], [S, 10], seed=91, spread=0.0)
    codes = b.codes[1].clone()
    codes[b.bt[0, key // BS], 1, key % BS, col] = NAN8
    cache = cw.Fp8KvCache.of(b.cache.k, codes.cuda().view(cw.FP8), b.cache.k_scale, b.cache.v_scale)
    meta, q = b.meta(), b.queries().cuda()

    def run(c):
        return _f64(cw.suffix_prefill_attn_fp8(meta, q, c, D ** -0.5) if splits == 0 else
                    cw.suffix_prefill_attn_split_fp8(meta, q, c, D ** -0.5, num_splits=splits))

    out, clean = run(cache), run(b.cache)
    sees = np.arange(S) + P >= key
    far = np.arange(S) + P < key - (256 // (hq // hkv) + 62)
    nan = np.isnan(out)
    assert nan[:S][sees, hq // 2:, col].all() and not nan[:S][far].any() and not nan[S:].any()
    nan[:S, hq // 2:, col] = False
    assert not nan.any()
    keep = ~np.isnan(out)
    assert np.array_equal(out[keep], clean[keep])


@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_tiny_scales(D):
    """Positive scales down to fp32's smallest: such values are nothing beside the others (value scales
    below 2^-100 count as 2^-100 in the calls over suffix rows: at most 448 * 2^-100 off)."""
    b = Batch(8, 2, D, [200], [70], seed=92, spread=0.0)
    tiny = [1e-39, 2.0 ** -149, 2.0 ** -127, 2.0 ** -126, 2.0 ** -101]
    for j, t in enumerate(tiny):
        b.scale[0][b.bt[0, 2 * j]] = t
        b.scale[1][b.bt[0, 2 * j + 1]] = t
        b.scale[1][b.bt[0, 2 * j], 1] = t
    cache = cw.Fp8KvCache.of(b.cache.k, b.cache.v, *(s.cuda() for s in b.scale))
    q = b.queries()
    meta, qd = b.meta(), q.cuda()
    for out in (cw.suffix_prefill_attn_fp8(meta, qd, cache, D ** -0.5),
                cw.suffix_prefill_attn_split_fp8(meta, qd, cache, D ** -0.5, num_splits=3)):
        _check_attention(_f64(out), _f64(q), b.rows(0, 0), b.rows(1, 0), 200, D ** -0.5, f"tiny scales D={D}")
    lens = torch.tensor([270], dtype=torch.int32).cuda()
    for n in (1, 3):
        out = cw.decode_attn_fp8(qd[-1:], cache, torch.from_numpy(b.bt).cuda(), lens, D ** -0.5, num_splits=n)
        _check_attention(_f64(out), _f64(q[-1:]), b.rows(0, 0), b.rows(1, 0), 269, D ** -0.5, "decode")


# ---------------------------------------------------------------- decode attention
def _check_decode(b, lens, q, out, scale, what):
    for r, n in enumerate(lens):
        n = min(max(n, 0), b.stride * BS)
        if n == 0:
            assert not _f64(out[r]).any(), what
            continue
        k, v = b.rows(0, r)[:n], b.rows(1, r)[:n]
        _check_attention(_f64(out[r:r + 1]), _f64(q[r:r + 1]), k, v, n - 1, scale, f"{what} r{r} len {n}")


DECODE_CASES = [
    (4, 1, 64, [1, 2, 15, 16, 17]),
    (8, 8, 128, [31, 32, 33, 0, 64]),
    (8, 2, 128, [127, 128, 129, 130, 1]),
    (28, 4, 128, [300, 5, 1000]),
    (16, 1, 64, [511, 513, 90]),
    (20, 1, 128, [260, 33]),
    (128, 1, 64, [129]),
    (64, 8, 128, [700]),
]


@pytest.mark.parametrize("hq,hkv,D,lens", DECODE_CASES)
@pytest.mark.parametrize("splits", [1, 2, 5, 64])
def test_decode(hq, hkv, D, lens, splits):
    _say(f"decode {hq}/{hkv} D={D} lens={lens} splits={splits}")
    b = Batch(hq, hkv, D, lens, [0] * len(lens), seed=hq + sum(lens), spread=0.5)
    q = b.queries(len(lens))
    bt, sl = torch.from_numpy(b.bt).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    out = torch.full((len(lens), hq, D), 4.0, dtype=torch.bfloat16, device="cuda")
    got = cw.decode_attn_fp8(q.cuda(), b.cache, bt, sl, D ** -0.5, num_splits=splits, out=out)
    torch.cuda.synchronize()
    assert got is out
    _check_decode(b, lens, q, out, D ** -0.5, f"decode {hq}/{hkv} x{splits}")


def test_decode_default_splits_and_long_sequence():
    b = Batch(32, 8, 128, [5000, 17], [0, 0], seed=21, spread=0.5)
    q = b.queries(2)
    out = cw.decode_attn_fp8(q.cuda(), b.cache, torch.from_numpy(b.bt).cuda(),
                             torch.tensor([5000, 17], dtype=torch.int32).cuda(), 128 ** -0.5)
    _check_decode(b, [5000, 17], q, out, 128 ** -0.5, "default splits")


@pytest.mark.parametrize("splits", [1, 3])
def test_decode_lengths_out_of_range_and_foreign_blocks(splits):
    """A length beyond the table counts as the table's; a negative one as 0; blocks outside the pool
    are zero keys and values."""
    b = Batch(8, 2, 64, [100, 64, 80], [0] * 3, seed=22, spread=0.0)
    b.L = [b.stride * BS] * 3
    for r in range(3):   # every table entry names a block of whole rows, or none
        b.bt[r] = np.arange(b.stride) % b.nb
    b.codes = [(torch.randn(b.nb, 2, BS, 64, generator=b.g) * 100).clamp(-448, 448).to(cw.FP8).view(torch.uint8)
               for _ in range(2)]
    b.bt[2, 1], b.bt[2, 3] = -5, b.nb
    cache = cw.Fp8KvCache.of(*(c.cuda().view(cw.FP8) for c in b.codes), b.cache.k_scale, b.cache.v_scale)
    lens = [10 ** 9, -3, 75]
    q = b.queries(3)
    out = cw.decode_attn_fp8(q.cuda(), cache, torch.from_numpy(b.bt).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                             0.125, num_splits=splits)
    torch.cuda.synchronize()
    _check_decode(b, lens, q, out, 0.125, "out of range")


@pytest.mark.parametrize("splits", [1, 4])
@pytest.mark.parametrize("key,sees", [(0, True), (299, True), (300, False)])
def test_decode_nan_codes(splits, key, sees):
    """A NaN key code makes its KV head's outputs NaN, a NaN value code its column; behind the length neither does."""
    b = Batch(8, 2, 64, [320, 40], [0, 0], seed=24, spread=0.0)
    q, lens = b.queries(2).cuda(), torch.tensor([300, 40], dtype=torch.int32).cuda()
    bt = torch.from_numpy(b.bt).cuda()
    for which in (0, 1):
        codes = [c.clone() for c in b.codes]
        codes[which][b.bt[0, key // BS], 1, key % BS, 9] = NAN8
        cache = cw.Fp8KvCache.of(*(c.cuda().view(cw.FP8) for c in codes), b.cache.k_scale, b.cache.v_scale)
        out = _f64(cw.decode_attn_fp8(q, cache, bt, lens, 0.125, num_splits=splits))
        bad = np.zeros(out.shape, bool)
        if sees:
            bad[0, 4:, slice(None) if which == 0 else 9] = True
        assert np.array_equal(np.isnan(out), bad), which


def test_decode_captured_replays_follow_growing_lengths():
    """Two captured decode calls with workspaces of their own, replayed in turn with other lengths
    and queries, equal eager calls each time."""
    lens = [40, 200, 7]
    b = Batch(8, 2, 128, [n + 60 for n in lens], [0] * 3, seed=23, spread=0.5)
    bt = torch.from_numpy(b.bt).cuda()
    sets = []
    for _ in range(2):
        q = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda")
        sl = torch.ones(3, dtype=torch.int32, device="cuda")
        ws = torch.empty(cw.decode_workspace_bytes(3, 8, 128, 4), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            cw.decode_attn_fp8(q, b.cache, bt, sl, 128 ** -0.5, num_splits=4, workspace=ws, out=out)
        sets.append((q, sl, ws, out, graph))
    for step in range(4):
        want = []
        for i, (q, sl, ws, out, graph) in enumerate(sets):
            q.copy_(b.queries(3).cuda())
            sl.copy_(torch.tensor([n + 7 * step + i for n in lens], dtype=torch.int32))
            want.append(cw.decode_attn_fp8(q, b.cache, bt, sl, 128 ** -0.5, num_splits=4))
        torch.cuda.synchronize()
        for s in sets:
            s[4].replay()
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            assert torch.equal(_bits(s[3]), _bits(w)), step


# ---------------------------------------------------------------- together
def test_layer_prefill_then_decode_steps():
    """A layer as it is used: norm, projection, append, prefill attention, then three decode steps on
    another stream than the default. Each call is checked against its oracle on the values that
    the calls before it left."""
    hq, hkv, D, hidden = 8, 2, 64, 256
    P, S = [16, 0, 5], [20, 33, 1]
    steps = 3
    b = Batch(hq, hkv, D, [p + s + steps for p, s in zip(P, S)], [0] * 3, seed=31, spread=0.0, held=P)
    g = b.g
    feats = (hq + 2 * hkv) * D
    w8, ws = _quantised(g, feats, hidden).cuda(), (_scales(g, feats // 128, hidden, -12, -11)).cuda()
    bias, weight = _normal(g, feats, std=0.1).cuda(), (1 + 0.1 * torch.randn(hidden, generator=g)).to(torch.bfloat16).cuda()
    rope = torch.from_numpy(cw.rope_table(64, D, 10000.0)).cuda()
    stream = torch.cuda.Stream()
    lens = list(P)
    for step in range(1 + steps):
        n = S if step == 0 else [1, 1, 1]
        T = sum(n)
        x, r = _normal(g, T, hidden).cuda(), _normal(g, T, hidden).cuda()
        before = [c.clone() for c in (b.cache.k.view(torch.uint8), b.cache.v.view(torch.uint8))]
        sb = [s.clone() for s in (b.cache.k_scale, b.cache.v_scale)]
        meta = cw.BatchMeta(b.bt, np.concatenate([[0], np.cumsum(n)]), lens, hq, hkv, D)
        seq = torch.tensor([a + c for a, c in zip(lens, n)], dtype=torch.int32).cuda()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            x8, xs, h = cw.add_rms_norm_fp8(x, weight, 1e-5, residual=r)
            qkv = cw.fp8_linear(x8, xs, w8, ws, bias)
            q, k, v = (t.view(T, -1, D) for t in qkv.split([hq * D, hkv * D, hkv * D], 1))
            qr = cw.rope_append_fp8(meta, k, v, b.cache, q=q, rope=rope)
            if step == 0:
                out = cw.suffix_prefill_attn_fp8(meta, qr, b.cache, D ** -0.5)
            else:
                out = cw.decode_attn_fp8(qr, b.cache, meta.bt, seq, D ** -0.5)
        stream.synchronize()
        what = f"step {step}"
        _check_norm(x, r, weight, 1e-5, x8, xs, h, what)
        exp, mag = F.linear(_f64(x8), _f64(xs), _f64(w8), _f64(ws), _f64(bias))
        cut = F.linear_cut(_f64(x8), _f64(xs), _f64(w8), _f64(ws))[0]
        _within(_f64(qkv), exp, B8 * np.abs(exp) + (hidden + 6) * 2.0 ** -23 * mag + 7 * 2.0 ** -13 * cut, what + " qkv")
        old = (b.codes, b.scale, b.P, b.S, b.L, b.cu, b.T)
        b.codes, b.scale = [c.cpu() for c in before], [s.cpu() for s in sb]
        b.P, b.S, b.cu, b.T = lens, n, np.concatenate([[0], np.cumsum(n)]), T
        _check_append(b, q, k, v, rope, qr, what)
        b.codes = [c.view(torch.uint8).cpu() for c in (b.cache.k, b.cache.v)]
        b.scale = [s.cpu() for s in (b.cache.k_scale, b.cache.v_scale)]
        b.L = [a + c for a, c in zip(lens, n)]
        for i in range(3):
            rows = slice(b.cu[i], b.cu[i + 1])
            _check_attention(_f64(out[rows]), _f64(qr[rows]), b.rows(0, i), b.rows(1, i), lens[i], D ** -0.5, what)
        lens = [a + c for a, c in zip(lens, n)]


def _layer_inputs(seed, P, S, hq=8, hkv=2, D=64, hidden=272):
    """A layer's weights, a cache with room, and one call's static inputs."""
    b = Batch(hq, hkv, D, [p + s for p, s in zip(P, S)], [0] * len(P), seed=seed, spread=0.0, held=P)
    g, feats, T = b.g, (hq + 2 * hkv) * D, sum(S)
    meta = cw.BatchMeta(b.bt, np.concatenate([[0], np.cumsum(S)]), P, hq, hkv, D)
    seq = torch.tensor([p + s for p, s in zip(P, S)], dtype=torch.int32).cuda()
    w8, ws = _quantised(g, feats, hidden).cuda(), _scales(g, feats // 128, hidden, -12, -11).cuda()
    weight, rope = torch.ones(hidden, dtype=torch.bfloat16, device="cuda"), torch.from_numpy(cw.rope_table(128, D, 10000.0)).cuda()
    x, r = torch.zeros(2, T, hidden, dtype=torch.bfloat16, device="cuda").unbind(0)

    def run(cache, stream=None):
        x8, xs, h = cw.add_rms_norm_fp8(x, weight, 1e-5, residual=r, stream=stream)
        qkv = cw.fp8_linear(x8, xs, w8, ws, stream=stream)
        q, k, v = (t.view(T, -1, D) for t in qkv.split([hq * D, hkv * D, hkv * D], 1))
        qr = cw.rope_append_fp8(meta, k, v, cache, q=q, rope=rope, stream=stream)
        out = cw.suffix_prefill_attn_fp8(meta, qr, cache, D ** -0.5, stream=stream)
        last = qr[(meta.cu[1:] - 1).long()] if stream is None else None
        return [x8.view(torch.uint8), xs, h, qr, out] + (
            [] if last is None else [cw.decode_attn_fp8(last, cache, meta.bt, seq, D ** -0.5, num_splits=3)])

    return b, x, r, run


def _copy_of(cache):
    return cw.Fp8KvCache.of(cache.k.clone(), cache.v.clone(), cache.k_scale.clone(), cache.v_scale.clone())


def test_layer_captured_and_replayed():
    """The five calls in one captured graph, replayed with other hidden states between eager runs on a copy
    of the cache: every replay has the eager run's bits, in its results and in the cache."""
    b, x, r, run = _layer_inputs(51, [20, 0, 37], [9, 17, 1])
    twin = _copy_of(b.cache)
    run(_copy_of(b.cache))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        got = run(b.cache)
    for step in range(4):
        for t in (x, r):
            t.copy_(_normal(b.g, *t.shape).cuda())
        want = [t.clone() for t in run(twin)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, e) in enumerate(zip(got, want)):
            assert torch.equal(a.view(torch.uint8), e.view(torch.uint8)), (step, i)
        for n in ("k", "v", "k_scale", "v_scale"):
            assert torch.equal(getattr(b.cache, n).view(torch.uint8), getattr(twin, n).view(torch.uint8)), (step, n)


def test_layer_on_given_streams():
    """With stream=: two layers' calls on two streams at once equal the ones on the current stream, and what
    the calls allocate comes from their stream's memory."""
    sets = [_layer_inputs(seed, [20, 0, 37], [40, 117, 1]) for seed in (52, 53)]
    for b, x, r, _ in sets:
        for t in (x, r):
            t.copy_(_normal(b.g, *t.shape).cuda())
    want = [run(_copy_of(b.cache)) for b, _, _, run in sets]
    caches = [_copy_of(b.cache) for b, *_ in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [run(c, stream=s) for (*_, run), c, s in zip(sets, caches, streams)]
    torch.cuda.synchronize()
    for g, w, s in zip(got, want, streams):
        for i, (a, e) in enumerate(zip(g, w)):
            assert torch.equal(a.view(torch.uint8), e.view(torch.uint8)), i
            seg = [m for m in torch.cuda.memory_snapshot()
                   if m["address"] <= a.data_ptr() < m["address"] + m["total_size"]]
            assert [m["stream"] for m in seg] == [s.cuda_stream], i


def test_blocks_beyond_32_bit_offsets():
    """Blocks at the end of a cache of 5.7 GB a tensor: append, prefill (whole and in runs) and decode have the
    bits that they have in a small one."""
    nb, hkv, D, hq, S = 600000, 5, 128, 15, [300, 70]
    g = _gen(94)
    big = np.full((2, 25), -1, np.int32)
    small = big.copy()
    order = torch.randperm(26, generator=g).numpy()
    ids = np.concatenate([np.arange(nb - 20, nb), [0, 1, 2 ** 18 - 1, 2 ** 18, 2 ** 18 + 1, nb // 2]])[order]
    for r, (a, n) in enumerate(((0, 19), (19, 5))):
        big[r, :n], small[r, :n] = ids[a:a + n], np.arange(a, a + n)
    rope = torch.from_numpy(cw.rope_table(512, D, 10000.0)).cuda()
    qkv = _normal(g, sum(S), (hq + 2 * hkv) * D).cuda()
    q, k, v = (t.view(sum(S), -1, D) for t in qkv.split([hq * D, hkv * D, hkv * D], 1))
    lens = torch.tensor(S, dtype=torch.int32).cuda()
    res = []
    for n, table in ((nb, big), (26, small)):
        cache = cw.Fp8KvCache(n, hkv, D)
        meta = cw.BatchMeta(table, np.concatenate([[0], np.cumsum(S)]), [0, 0], hq, hkv, D)
        qr = cw.rope_append_fp8(meta, k, v, cache, q=q, rope=rope)
        out = [qr, cw.suffix_prefill_attn_fp8(meta, qr, cache, 0.088),
               cw.suffix_prefill_attn_split_fp8(meta, qr, cache, 0.088, num_splits=3)]
        out += [cw.decode_attn_fp8(qr[:2], cache, meta.bt, lens, 0.088, num_splits=m) for m in (1, 4)]
        full = torch.from_numpy(np.concatenate([table[0, :18], table[1, :4]])).cuda().long()   # whole blocks
        out += [c.view(torch.uint8)[full] for c in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
        res.append(out)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(*res)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i


def test_decode_calls_at_once_on_two_streams():
    """Two calls at the same time with workspaces that they allocate themselves."""
    b = Batch(8, 2, 128, [900, 300], [0, 0], seed=54, spread=0.5)
    bt = torch.from_numpy(b.bt).cuda()
    qs = [b.queries(2).cuda() for _ in range(2)]
    sl = [torch.tensor(n, dtype=torch.int32).cuda() for n in ([900, 300], [850, 1])]
    want = [cw.decode_attn_fp8(q, b.cache, bt, n, 128 ** -0.5, num_splits=5) for q, n in zip(qs, sl)]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[cw.decode_attn_fp8(q, b.cache, bt, n, 128 ** -0.5, num_splits=5, stream=s) for _ in range(8)]
           for q, n, s in zip(qs, sl, streams)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(_bits(t), _bits(w)) for t in g)


def test_batches_with_no_rows():
    """Batches whose requests are all empty launch nothing; the cache keeps its bytes."""
    b = Batch(8, 2, 64, [20, 0], [0, 0], seed=55)
    before = b.cache.k.view(torch.uint8).clone()
    none = torch.empty(0, 8, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    rope = torch.from_numpy(cw.rope_table(64, 64, 10000.0)).cuda()
    assert cw.rope_append_fp8(b.meta(), kv, kv, b.cache, q=none, rope=rope).shape == none.shape
    assert cw.suffix_prefill_attn_fp8(b.meta(), none, b.cache, 0.1).shape == none.shape
    x8, xs, h = cw.add_rms_norm_fp8(none.view(0, 512), torch.ones(512, dtype=torch.bfloat16, device="cuda"), 1e-5)
    w8, ws = _quantised(b.g, 48, 512).cuda(), _scales(b.g, 1, 512).cuda()
    assert cw.fp8_linear(x8, xs, w8, ws).shape == (0, 48)
    torch.cuda.synchronize()
    assert torch.equal(before, b.cache.k.view(torch.uint8))


def test_python_refusals_on_the_gpu():
    b = Batch(8, 2, 64, [20], [4], seed=41)
    k = _normal(b.g, 4, 2, 64).cuda()
    with pytest.raises(cw.CwError, match="rope is required"):
        cw.rope_append_fp8(b.meta(), k, k, b.cache, q=b.queries().cuda())
    with pytest.raises(ValueError, match="KV heads"):
        cw.rope_append_fp8(b.meta(), k, k, cw.Fp8KvCache(4, 2, 128))
    with pytest.raises(ValueError, match="row must be contiguous"):
        cw.rope_append_fp8(b.meta(), k.transpose(1, 2).contiguous().transpose(1, 2), k, b.cache)
    with pytest.raises(ValueError, match="rows overlap"):
        cw.rope_append_fp8(b.meta(), k[:1].expand(4, 2, 64), k, b.cache)
    with pytest.raises(TypeError, match="float8"):
        cw.fp8_linear(k.view(8, 64), torch.ones(8, 1).cuda(), k.view(8, 64), torch.ones(1, 1).cuda())
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="GPU memory"):
        cw.add_rms_norm_fp8(x, torch.zeros(64, dtype=torch.bfloat16), 1e-5)
    with pytest.raises(cw.CwError, match="hidden must be a multiple"):
        cw.add_rms_norm_fp8(torch.zeros(2, 24, dtype=torch.bfloat16, device="cuda"),
                            torch.zeros(24, dtype=torch.bfloat16, device="cuda"), 1e-5)
    with pytest.raises(cw.CwError, match="workspace"):
        cw.decode_attn_fp8(_normal(b.g, 1, 8, 64).cuda(), b.cache, torch.from_numpy(b.bt).cuda(),
                           torch.ones(1, dtype=torch.int32).cuda(), 0.1, num_splits=2,
                           workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
