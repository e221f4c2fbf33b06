"""GPU parity of the calls over the 4-bit cache against their fp64 oracle (oracle.fp4 and, for
attention over the values a cache stands for, oracle.attention).

Bounds, derived from the roundings (eps/2 of bf16 is 2^-8):

* append: pages are compared byte by byte with the oracle's, which rounds the rotation in 64 bits
  (or, beside borders that these do not resolve, in rational arithmetic): the call's codes are those of exact arithmetic. q is an output rounding, 2^-8 |q|, plus the
  rotation's: 2^-24 of a product and of the sum, taken as 2^-22 of the products' magnitudes.
* rows: exact.
* attention: with A = sum p|v| / sum p, the probabilities' rounding to bf16 before the product
  gives 2^-8 A; the row's sum of the same rounded values 2^-8 |o| <= 2^-8 A; fp32 scores of
  magnitude below 64 and the exponential 2^-12 A; the output 2^-8 |o|.
"""
import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import fp4 as F
from paper_2606_19667_amd import cw

pytestmark = pytest.mark.gpu

BS = 16
B8 = 2.0 ** -8


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


def _bits(t):
    return t.detach().view(torch.int16)


def _within(got, exp, bound, what):
    bad = ~(np.abs(got - exp) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0].tolist()}: " \
                          f"{got[bad][0]} against {exp[bad][0]}, bound {np.broadcast_to(bound, bad.shape)[bad][0]}"


class Batch:
    """A ragged batch over a 4-bit cache with random placement, random codes, scales of about 1 (times
    2^+-spread) and NaN scales behind every prompt."""

    def __init__(self, hq, hkv, D, P, S, seed, extra=3, spread=1, held=None):
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
        pages = torch.randint(0, 256, (self.nb, hkv, 17 * D), generator=g, dtype=torch.uint8).numpy()
        pages[:, :, 16 * D:] = torch.randint(125 - spread, 126 + spread, (self.nb, hkv, D), generator=g,
                                             dtype=torch.uint8).numpy()
        for r, n in enumerate(held):
            for j in range(-(-n // BS)):
                for t in range(min(BS, n - j * BS), BS):
                    for d in range(0, D, 32):
                        for at in (F.key_scale_byte, F.value_scale_byte):
                            pages[self.bt[r, j], :, at(D, t, d)] = 255
        self.host(pages)

    def host(self, pages):
        self.pages = pages
        self.cache = cw.Fp4KvCache.of(torch.from_numpy(pages.copy()).cuda())

    def set_scale(self, which, r, t, g, group, byte):
        """Plants one scale byte of request r's token t."""
        at = (F.key_scale_byte, F.value_scale_byte)[which](self.D, t % BS, 32 * group)
        pages = self.pages.copy()
        pages[self.bt[r, t // BS], g, at] = byte
        self.host(pages)

    def meta(self):
        return cw.BatchMeta(self.bt, self.cu, self.P, self.hq, self.hkv, self.D)

    def rows(self, r, n=None):
        """Request r's (keys, values) as the cache at the start holds them, [L, Hkv, D]."""
        return F.logical_rows(self.pages, self.bt[r], 0, self.L[r] if n is None else n)

    def queries(self, n=None):
        return _normal(self.g, self.T if n is None else n, self.hq, self.D)

    def positions(self):
        return np.concatenate([np.arange(p, p + s) for p, s in zip(self.P, self.S)]) if self.T else np.zeros(0, int)


# ---------------------------------------------------------------- append
def _check_append(b, q, k, v, rope, interleaved, q_out, what):
    turn = (lambda u: _f64(u)) if rope is None else \
        (lambda u: F.rotate(_f64(u), _f64(rope)[b.positions()], interleaved))
    if q is not None:
        exp = turn(q)
        big = np.abs(_f64(q)).max(-1, keepdims=True) * (0 if rope is None else 2 * np.abs(_f64(rope)).max())
        _within(_f64(q_out), exp, B8 * np.abs(exp) + 2.0 ** -22 * big, what + " q")
    want = F.append(b.pages, turn(k), _f64(v), b.bt, b.cu, b.P)
    got = b.cache.pages.cpu().numpy()
    bad = np.argwhere(got != want)
    assert not len(bad), f"{what}: {len(bad)} bytes of {got.size}, first at {bad[0].tolist()}"


def _append_inputs(b, std=2.0):
    n = b.hq + 2 * b.hkv
    qkv = _normal(b.g, b.T, n * b.D, std=std).cuda()
    return (x.view(b.T, -1, b.D) for x in qkv.split([b.hq * b.D, b.hkv * b.D, b.hkv * b.D], 1))


def _table(n, rotary, base=10000.0):
    return torch.from_numpy(cw.rope_table(n, rotary, base)).cuda()


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
@pytest.mark.parametrize("part,interleaved", [(1, False), (1, True), (0.5, False), (0.75, True), (0.25, False), (0, False)])
def test_append(hq, hkv, D, P, S, part, interleaved):
    rotary = max(16, int(part * D)) if part else 0
    _say(f"append {hq}/{hkv} D={D} P={P[:5]} S={S[:5]} rotary={rotary} interleaved={interleaved}")
    b = Batch(hq, hkv, D, P, S, seed=sum(P) + hq, held=P)
    q, k, v = _append_inputs(b)
    rope = _table(max(b.L) + 1, rotary) if part else None
    q_out = cw.rope_append_fp4(b.meta(), k, v, b.cache, q=q if part else None, rope=rope, interleaved=interleaved)
    torch.cuda.synchronize()
    _check_append(b, q if part else None, k, v, rope, interleaved, q_out, f"append {hq}/{hkv}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_values_beside_borders(D, interleaved):
    """Keys that the rotation brings as near to a border of two codes (or of two scales: 7 times a power of two)
    as 2^-30 of it, which fp32 cannot hold: each falls on its side."""
    b = Batch(2, 2, D, [3], [40], seed=61, held=[3])
    _, _, v = _append_inputs(b)
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0, -0.25, -5.0, -2.5])
    k = borders[torch.randint(0, 13, (40, 2, D), generator=b.g)]
    k[:, :, ::32] = torch.where(torch.rand(40, 2, D // 32, generator=b.g) < 0.5, 6.0, 7.0)
    k = (k * torch.exp2(torch.randint(-3, 4, (40, 1, 1), generator=b.g).float())).to(torch.bfloat16).cuda()
    n = D // 2
    rope = torch.ones(43, n, 2)
    rope[:, :, 1] = torch.randint(-1, 2, (43, n), generator=b.g) * torch.exp2(-torch.randint(26, 40, (43, n), generator=b.g).float())
    rope = rope.cuda()
    cw.rope_append_fp4(b.meta(), k, v, b.cache, rope=rope, interleaved=interleaved)
    torch.cuda.synchronize()
    _check_append(b, None, k, v, rope, interleaved, None, "borders")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("size", [0, -96, 100])
def test_append_values_beside_borders_below_64_bits(D, interleaved, size):
    """Keys next to a border of two codes, or of two scales, by as little as 2^-230 of it: a double holds 2^-53. The
    codes are those of rational arithmetic. (`size`: the keys' power of two.)"""
    n, T = D // 2, 10
    b = Batch(1, 1, D, [3], [T], seed=68, held=[3])
    _, _, v = _append_inputs(b)
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -1.25, -2.5, -5.0, 0.75])
    near = borders[torch.randint(0, 12, (T, 1, n), generator=b.g)]
    near[:, :, ::16] = torch.where(torch.rand(T, 1, n // 16, generator=b.g) < 0.5, 6.0, 7.0)
    far = torch.exp2(-torch.randint(20, 126 + min(size, 0), (T, 1, n), generator=b.g).float())   # (times 2^size a bf16 value)
    far = far * torch.randint(-1, 2, (T, 1, n), generator=b.g)
    first = torch.rand(T, 1, n, generator=b.g) < 0.5   # the column of a pair that is beside a border
    cols = [torch.where(first, near, far), torch.where(first, far, near)]
    k = (torch.stack(cols, -1).flatten(2) if interleaved else torch.cat(cols, -1)) * 2.0 ** size
    k = k.to(torch.bfloat16).cuda()
    rope = torch.ones(T + 3, n, 2)
    rope[:, :, 1] = torch.exp2(-torch.randint(20, 105, (T + 3, n), generator=b.g).float()) * \
        (2 * torch.randint(0, 2, (T + 3, n), generator=b.g) - 1)
    cw.rope_append_fp4(b.meta(), k, v, b.cache, rope=rope.cuda(), interleaved=interleaved)
    torch.cuda.synchronize()
    pages = b.cache.pages.cpu().numpy()
    for t in range(T):
        exact = F.exact_rotation(_f64(k)[t, 0], _f64(rope)[t + 3], interleaved)
        codes, scales = F.exact_codes(exact)
        got, at = (x[(t + 3) % BS] for x in F.unpack(pages[b.bt[0, (t + 3) // BS], 0], D)[0])
        got = np.where(got == 8, 0, got)   # (minus zero is zero)
        assert np.array_equal(at, scales), (t, at, scales)
        off = np.flatnonzero(got != codes)
        assert not len(off), f"token {t}: {len(off)} of {D}, column {off[0]} is {got[off[0]]}, should be {codes[off[0]]}"


def test_append_products_that_leave_fp32():
    """A table of more than 1 (scaled angles): both products of a pair leave fp32, their difference does not, their sum does."""
    b = Batch(2, 2, 128, [0], [20], seed=69, held=[0])
    _, k, v = _append_inputs(b)
    k.copy_(((torch.rand(k.shape, generator=b.g) * 0.02 + 0.97) * 3.3e38).to(torch.bfloat16))
    rope = torch.tensor([1.2, 1.3]).expand(20, 64, 2).contiguous()
    rope[10:] = torch.tensor([1.3, -1.2])   # (the other column of a pair)
    rope = rope.cuda()
    cw.rope_append_fp4(b.meta(), k, v, b.cache, rope=rope)
    torch.cuda.synchronize()
    turned = F.rotate(_f64(k), _f64(rope), False)
    assert (np.abs(turned[:10, :, :64]) < 2.0 ** 127).all() and (np.abs(turned[:10, :, 64:]) > 2.0 ** 128).all()
    _check_append(b, None, k, v, rope, False, None, "beyond fp32")


def test_append_cancelling_rotations():
    """Pairs whose products nearly cancel: 24 bits of each product are not enough for the difference's codes."""
    b = Batch(2, 2, 128, [0], [64], seed=62, held=[0])
    _, k, v = _append_inputs(b)
    k[:, :, 64:] = k[:, :, :64]
    ang = torch.rand(64, 64, generator=b.g) * 2e-3 + np.pi / 4
    rope = torch.stack([ang.cos(), ang.sin()], -1).cuda()
    cw.rope_append_fp4(b.meta(), k, v, b.cache, rope=rope)
    torch.cuda.synchronize()
    _check_append(b, None, k, v, rope, False, None, "cancelling")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rotate", [False, True])
def test_append_values_of_any_size(D, rotate):
    """Rows from bf16's smallest to its largest values, zeros, infinities and NaN: the last two make the scale of
    their 32 columns (and of their pair's) NaN."""
    b = Batch(2, 2, D, [5], [70], seed=63, held=[5])
    _, k, v = _append_inputs(b, std=1.0)
    for t in (k, v):
        size = torch.exp2(torch.randint(-133, 127, (70, 2, D // 32), generator=b.g).float()).repeat_interleave(32, 2)
        x = (t.float().cpu() * size).clamp(-3.38e38, 3.38e38)
        x[:4] = 0.0
        x[4] = -0.0
        x[5, 0, 7], x[6, 1, 33], x[7, 0, D - 1] = float("nan"), float("inf"), -float("inf")
        x[8], x[9] = 3.38e38, 1e-40
        t.copy_(x.to(torch.bfloat16))
    if rotate:   # (sums of two of the largest leave fp32)
        k.copy_((k.float() / 2).to(torch.bfloat16))
    rope = _table(80, D) if rotate else None
    cw.rope_append_fp4(b.meta(), k, v, b.cache, rope=rope)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        _check_append(b, None, k, v, rope, False, None, "any size")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("part,interleaved", [(1, False), (0.5, False), (1, True)])
def test_append_queries_of_any_size(D, part, interleaved):
    """Queries from bf16's smallest to near its largest values, infinities and NaN: what the formula gives of them."""
    b = Batch(4, 2, D, [5], [70], seed=64, held=[5])
    q, k, v = _append_inputs(b)
    size = torch.exp2(torch.randint(-133, 120, (70, 4, D // 32), generator=b.g).float()).repeat_interleave(32, 2)
    x = q.float().cpu() * size
    x[5, 0, 7], x[6, 1, 33], x[7, 0, D - 1], x[8, 3, 0] = float("nan"), float("inf"), -float("inf"), float("inf")
    q.copy_(x.to(torch.bfloat16))
    rope = _table(80, int(part * D))
    got = _f64(cw.rope_append_fp4(b.meta(), k, v, b.cache, q=q, rope=rope, interleaved=interleaved))
    cos_sin = _f64(rope)[b.positions()]
    with np.errstate(invalid="ignore"):
        exp = F.rotate(_f64(q), cos_sin, interleaved)
        # |x c| + |w s|: the rotation of magnitudes by (|c|, -|s|) has it in a pair's first column, by (|c|, |s|) in its second
        mag = [F.rotate(np.abs(_f64(q)), np.stack([np.abs(cos_sin[..., 0]), s * np.abs(cos_sin[..., 1])], -1), interleaved)
               for s in (-1, 1)]
    whole = np.isfinite(exp)
    assert (~whole).sum() >= 4 and np.array_equal(got[~whole], exp[~whole], equal_nan=True)
    # output's rounding, of its smallest steps too; product and sum, half a unit of 2^-23 each
    _within(got[whole], exp[whole], B8 * np.abs(exp[whole]) + 2.0 ** -23 * np.maximum(*mag)[whole] + 2.0 ** -133, f"D={D}")


def test_append_drops_blocks_outside_the_pool_and_long_tables():
    b = Batch(4, 2, 64, [10, 3], [40, 30], seed=64, held=[10, 3])
    b.bt[0, 1], b.bt[1, 0], b.bt[1, 2] = -7, b.nb, 2 ** 31 - 1
    q, k, v = _append_inputs(b)
    rope = _table(64, 64)
    q_out = cw.rope_append_fp4(b.meta(), k, v, b.cache, q=q, rope=rope)
    torch.cuda.synchronize()
    _check_append(b, q, k, v, rope, False, q_out, "foreign blocks")


def test_append_of_two_requests_into_one_block():
    """Tokens of one block by two requests, in different slots."""
    b = Batch(4, 2, 128, [0, 6], [6, 5], seed=65, held=[0, 0])
    b.bt[1] = b.bt[0]
    q, k, v = _append_inputs(b)
    rope = _table(32, 128)
    q_out = cw.rope_append_fp4(b.meta(), k, v, b.cache, q=q, rope=rope)
    torch.cuda.synchronize()
    _check_append(b, q, k, v, rope, False, q_out, "shared block")


def test_append_in_place_queries_and_rows_of_a_larger_buffer():
    b = Batch(8, 2, 64, [7], [33], seed=66, held=[7])
    wide = _normal(b.g, 40, 3, 2, 64).cuda()
    k, v = wide[3:36, 0], wide[3:36, 2]
    q = b.queries().cuda()
    keep, rope = q.clone(), _table(64, 32)
    assert cw.rope_append_fp4(b.meta(), k, v, b.cache, q=q, rope=rope, interleaved=True, q_out=q) is q
    torch.cuda.synchronize()
    _check_append(b, keep, k, v, rope, True, q, "in place")


def test_append_captured_and_replayed_with_growing_prefixes():
    """A decode step's append in a HIP graph: each replay reads the prefix lengths and the table from device
    memory and leaves the bytes of an eager call at those lengths."""
    P = [14, 0, 31]
    b, e = (Batch(8, 2, 64, [p + 6 for p in P], [1, 1, 1], seed=7, held=P) for _ in range(2))
    rope = _table(64, 64)
    meta = cw.BatchMeta(b.bt, [0, 1, 2, 3], P, 8, 2, 64)
    q, k, v = (torch.zeros(3, h, 64, dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2))
    q_out = torch.empty_like(q)
    rows = [torch.empty_like(k) for _ in range(2)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        cw.rope_append_fp4(meta, k, v, b.cache, q=q, rope=rope, q_out=q_out)
        cw.cache_rows_fp4(meta, b.cache, *rows)
    for step in range(5):
        new = [_normal(b.g, *t.shape).cuda() for t in (q, k, v)]
        for t, x in zip((q, k, v), new):
            t.copy_(x)
        meta.plen.copy_(torch.tensor([p + step for p in P], dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        em = cw.BatchMeta(e.bt, [0, 1, 2, 3], [p + step for p in P], 8, 2, 64)
        eq = cw.rope_append_fp4(em, new[1], new[2], e.cache, q=new[0], rope=rope)
        er = cw.cache_rows_fp4(em, e.cache)
        torch.cuda.synchronize()
        assert torch.equal(_bits(q_out), _bits(eq)), step
        assert torch.equal(b.cache.pages, e.cache.pages), step
        assert all(torch.equal(_bits(a), _bits(c)) for a, c in zip(rows, er)), step


# ---------------------------------------------------------------- rows
ROWS_CASES = [
    (1, 64, [0], [1]),
    (2, 128, [0, 5, 16, 33], [1, 40, 0, 15]),
    (7, 64, [3, 0], [17, 300]),
    (8, 128, [15] * 70, [2] * 70),
    (5, 128, [100], [64]),
]


@pytest.mark.parametrize("hkv,D,P,S", ROWS_CASES)
def test_rows(hkv, D, P, S):
    _say(f"rows {hkv} D={D} P={P[:4]} S={S[:4]}")
    b = Batch(hkv, hkv, D, P, S, seed=40 + hkv, spread=90)
    got = [torch.full((b.T + 2, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cw.cache_rows_fp4(b.meta(), b.cache, got[0][:b.T], got[1][:b.T])
    torch.cuda.synchronize()
    for r in range(len(P)):
        want = F.logical_rows(b.pages, b.bt[r], P[r], S[r])
        for g, w in zip(got, want):
            assert np.array_equal(_f64(g[b.cu[r]:b.cu[r + 1]]), w), r
    assert (got[0][b.T:] == 7).all() and (got[1][b.T:] == 7).all()


def test_rows_nan_scales_foreign_blocks_and_one_of_the_two():
    b = Batch(2, 2, 64, [0], [60], seed=47)
    b.set_scale(0, 0, 20, 1, 1, 255)
    b.set_scale(1, 0, 21, 0, 0, 255)
    b.bt[0, 3] = b.nb
    k, v = cw.cache_rows_fp4(b.meta(), b.cache)
    wk, wv = F.logical_rows(b.pages, b.bt[0], 0, 60)
    assert np.isnan(wk[20, 1, 32:]).all() and not wk[48:].any()
    assert np.array_equal(_f64(k), wk, equal_nan=True) and np.array_equal(_f64(v), wv, equal_nan=True)
    one = torch.zeros_like(k)
    m = b.meta()
    st = cw.lib().cw_cache_rows_fp4(b.cache.pages.data_ptr(), m.bt.data_ptr(), m.bt_stride, m.cu.data_ptr(), m.plen.data_ptr(),
                                    m._hp(m.cu_host), m._hp(m.plen_host), 1, 2, 64, 16, b.nb, None, one.data_ptr(), None)
    torch.cuda.synchronize()
    assert st == cw.CW_OK and torch.equal(_bits(one), _bits(v))


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
    (28, 4, 128, [77], [1100]),
    (4, 1, 64, [9001, 0, 4096], [70, 33, 16]),
    (2, 2, 128, [4100, 8175], [20, 3]),
]


@pytest.mark.parametrize("hq,hkv,D,P,S", PREFILL_CASES)
def test_prefill(hq, hkv, D, P, S):
    _say(f"prefill {hq}/{hkv} D={D} P={P} S={S}")
    b = Batch(hq, hkv, D, P, S, seed=hq + sum(S))
    q = b.queries()
    qd = q.cuda()
    out = torch.full((b.T + 3, hq, D), 9.0, dtype=torch.bfloat16, device="cuda")
    got = cw.suffix_prefill_attn_fp4(b.meta(), qd, b.cache, D ** -0.5, out=out[:b.T])
    torch.cuda.synchronize()
    assert got.data_ptr() == out.data_ptr() and (out[b.T:] == 9).all()
    for r in range(len(P)):
        if S[r]:
            rows = slice(b.cu[r], b.cu[r + 1])
            _check_attention(_f64(out[rows]), _f64(q[rows]), *b.rows(r), P[r], D ** -0.5, f"prefill {hq}/{hkv} r{r}")


def _run_prefill(meta, q, cache, scale, splits):
    return _f64(cw.suffix_prefill_attn_fp4(meta, q, cache, scale) if splits == 0 else
                cw.suffix_prefill_attn_split_fp4(meta, q, cache, scale, num_splits=splits))


@pytest.mark.parametrize("splits", [0, 1, 3, 12])
@pytest.mark.parametrize("hq,hkv,D,key", [(8, 2, 128, 5), (8, 2, 128, 270), (14, 2, 64, 270), (2, 2, 64, 620), (2, 2, 64, 19)])
def test_prefill_nan_scales(hq, hkv, D, key, splits):
    """A NaN scale of one KV head's key makes that head's rows that see it NaN, and nothing else; one of a value its
    32 columns of them. What else that may reach are the same columns and head in earlier rows, at most
    256 / (Hq / Hkv) + 62 tokens before."""
    P, S = 20, 700
    b = Batch(hq, hkv, D, [P, 33], [S, 10], seed=91)
    start, meta, q = b.pages, b.meta(), b.queries().cuda()
    clean = _run_prefill(meta, q, b.cache, D ** -0.5, splits)
    sees = np.arange(S) + P >= key
    b.set_scale(0, 0, key, 1, 0, 255)
    nan = np.isnan(_run_prefill(meta, q, b.cache, D ** -0.5, splits))
    assert nan[:S][sees, hq // 2:].all() and not nan[:S][~sees].any() and not nan[:S, :hq // 2].any() and not nan[S:].any()
    b.host(start)
    b.set_scale(1, 0, key, 1, 1, 255)
    out = _run_prefill(meta, q, b.cache, D ** -0.5, splits)
    far = np.arange(S) + P < key - (256 // (hq // hkv) + 62)
    nan = np.isnan(out)
    assert nan[:S][sees, hq // 2:, 32:64].all() and not nan[:S][far].any() and not nan[S:].any()
    keep = ~nan
    nan[:S, hq // 2:, 32:64] = False
    assert not nan.any()
    assert np.array_equal(out[keep], clean[keep])


@pytest.mark.parametrize("splits", [0, 3, 11])
@pytest.mark.parametrize("D", [64, 128])
def test_prefill_scores_that_grow_by_orders(D, splits):
    """Keys whose scales grow along the prompt: the softmax base moves, several times in a row's steps; and shrink:
    later keys add nothing. One step's keys dominate whatever the order."""
    for name, slope in (("grow", 1), ("shrink", -1)):
        b = Batch(8, 2, D, [300], [150], seed=77, spread=0)
        pages = b.pages.copy()
        for j in range(b.stride):
            e = 119 + (j * 12 // b.stride if slope > 0 else 12 - j * 12 // b.stride)
            region = pages[b.bt[0, j], :, 16 * D:16 * D + D // 2]
            region[region != 255] = e
        b.host(pages)
        q = b.queries()
        out = _run_prefill(b.meta(), q.cuda(), b.cache, D ** -0.5, splits)
        # scores reach 128 * 6 * 2^4 * 4 / 8: their fp32 sums' error is 2^-24 times D of them; the bound counts it
        k, v = b.rows(0)
        exp = OA.suffix_prefill_attention(_f64(q), k, v, 300, D ** -0.5)
        mag = OA.suffix_prefill_attention(_f64(q), k, np.abs(v), 300, D ** -0.5)
        score = np.abs(_f64(q)).max() * np.abs(k).max() * D * D ** -0.5
        # a probability below 2^-126 of the base's (whose own is 1, so the row's sum is 1 at least) is zero in fp32
        lost = len(k) * 2.0 ** -126 * np.abs(v).max()
        _within(out, exp, (2 * B8 + 2.0 ** -12 + 2 * score * 2.0 ** -22) * mag + B8 * np.abs(exp) + lost, name)


@pytest.mark.parametrize("splits", [0, 3, 11])
@pytest.mark.parametrize("D", [64, 128])
def test_prefill_ends_beside_values_out_of_range(D, splits):
    """One head's values are near 2^126, so its rows' sums may leave fp32; one of its query rows is NaN. The call
    ends, the NaN row is NaN, and the other head's rows are right."""
    b = Batch(8, 2, D, [70], [40], seed=81)
    pages = b.pages.copy()
    region = pages[:, 1, 16 * D + D // 2:]
    region[region != 255] = 252
    b.host(pages)
    q = b.queries()
    q[3, 4:] = float("nan")
    got = _run_prefill(b.meta(), q.cuda(), b.cache, D ** -0.5, splits)
    assert np.isnan(got[3, 4:]).all()
    k, v = b.rows(0)
    _check_attention(got[:, :4], _f64(q[:, :4]), k[:, :1], v[:, :1], 70, D ** -0.5, f"D={D}")


def test_prefill_foreign_blocks_and_foreign_plans():
    """Blocks outside the pool are zero keys and values, each with score 0; a plan of another batch computes nothing."""
    b = Batch(8, 2, 128, [100], [60], seed=82)
    b.bt[0, 2], b.bt[0, 7] = -4, b.nb
    q = b.queries()
    meta = b.meta()
    out = cw.suffix_prefill_attn_fp4(meta, q.cuda(), b.cache, 0.09)
    k, v = b.rows(0)
    assert not k[32:48].any() and not v[112:128].any()
    _check_attention(_f64(out), _f64(q), k, v, 100, 0.09, "foreign blocks")
    other = cw.BatchMeta(b.bt, [0, 60], [99], 8, 2, 128)
    meta.plan = other.plan
    out = torch.full_like(out, 5.0)
    cw.suffix_prefill_attn_fp4(meta, q.cuda(), b.cache, 0.09, out=out)
    torch.cuda.synchronize()
    assert (out == 5).all()


SPLIT_CASES = [
    (8, 2, 128, [1000], [30]),
    (8, 2, 64, [2000, 0, 77], [20, 40, 0]),
    (28, 4, 128, [700, 40], [40, 3]),
    (4, 1, 64, [5000, 3, 4100], [9, 70, 64]),
    (128, 2, 64, [130], [5]),
    (64, 4, 64, [700, 50], [260, 41]),
]


@pytest.mark.parametrize("hq,hkv,D,P,S", SPLIT_CASES)
@pytest.mark.parametrize("splits", [None, 1, 2, 7, 9, 64])
def test_prefill_split(hq, hkv, D, P, S, splits):
    """Runs of keys, some of them empty (short prompts) or unseen by some rows, joined."""
    _say(f"split prefill {hq}/{hkv} D={D} P={P} S={S} x{splits}")
    b = Batch(hq, hkv, D, P, S, seed=71 + hq)
    q, meta = b.queries(), b.meta()
    n = cw.split_count_fp4(meta) if splits is None else splits
    ws = torch.full((cw.split_workspace_bytes(meta, n) + 64,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN
    out = torch.full((b.T + 3, hq, D), 9.0, dtype=torch.bfloat16, device="cuda")
    cw.suffix_prefill_attn_split_fp4(meta, q.cuda(), b.cache, D ** -0.5, num_splits=splits, workspace=ws, out=out[:b.T])
    torch.cuda.synchronize()
    assert (out[b.T:] == 9).all() and (ws[-64:] == 0xFF).all()
    for r in range(len(P)):
        if S[r]:
            rows = slice(b.cu[r], b.cu[r + 1])
            _check_attention(_f64(out[rows]), _f64(q[rows]), *b.rows(r), P[r], D ** -0.5, f"r{r}")


# ---------------------------------------------------------------- decode attention
def _check_decode(b, lens, q, out, scale, what):
    for r, n in enumerate(lens):
        n = min(max(n, 0), b.stride * BS)
        if n == 0:
            assert not _f64(out[r]).any(), what
            continue
        _check_attention(_f64(out[r:r + 1]), _f64(q[r:r + 1]), *b.rows(r, n), n - 1, scale, f"{what} r{r} len {n}")


DECODE_CASES = [
    (4, 1, 64, [1, 2, 15, 16, 17]),
    (8, 8, 128, [31, 32, 33, 0, 64]),
    (8, 2, 128, [127, 128, 129, 130, 1]),
    (28, 4, 128, [300, 5, 1000]),
    (16, 1, 64, [511, 513, 90]),
    (20, 1, 128, [260, 33]),
    (128, 1, 64, [129]),
    (64, 8, 128, [700]),
    (4, 1, 128, [4500, 2049, 1023]),
]


@pytest.mark.parametrize("hq,hkv,D,lens", DECODE_CASES)
@pytest.mark.parametrize("splits", [1, 2, 5, 64])
def test_decode(hq, hkv, D, lens, splits):
    _say(f"decode {hq}/{hkv} D={D} lens={lens} splits={splits}")
    b = Batch(hq, hkv, D, lens, [0] * len(lens), seed=hq + sum(lens))
    q = b.queries(len(lens))
    bt, sl = torch.from_numpy(b.bt).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    out = torch.full((len(lens) + 1, hq, D), 4.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((cw.decode_workspace_bytes_fp4(len(lens), hq, D, splits) + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    cw.decode_attn_fp4(q.cuda(), b.cache, bt, sl, D ** -0.5, num_splits=splits, workspace=ws, out=out[:-1])
    torch.cuda.synchronize()
    assert (out[-1] == 4).all() and (ws[-64:] == 0xFF).all()
    _check_decode(b, lens, q, out, D ** -0.5, f"decode {hq}/{hkv} x{splits}")


def test_decode_default_splits_and_long_sequence():
    b = Batch(32, 8, 128, [5000, 17], [0, 0], seed=21)
    q = b.queries(2)
    out = cw.decode_attn_fp4(q.cuda(), b.cache, torch.from_numpy(b.bt).cuda(),
                             torch.tensor([5000, 17], dtype=torch.int32).cuda(), 128 ** -0.5)
    _check_decode(b, [5000, 17], q, out, 128 ** -0.5, "default splits")


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("D", [64, 128])
def test_decode_scores_that_grow_by_orders(D, splits):
    for name, slope in (("grow", 1), ("shrink", -1)):
        b = Batch(8, 2, D, [900], [0], seed=78, spread=0)
        pages = b.pages.copy()
        for j in range(b.stride):
            e = 119 + (j * 12 // b.stride if slope > 0 else 12 - j * 12 // b.stride)
            region = pages[b.bt[0, j], :, 16 * D:16 * D + D // 2]
            region[region != 255] = e
        b.host(pages)
        q = b.queries(1)
        out = cw.decode_attn_fp4(q.cuda(), b.cache, torch.from_numpy(b.bt).cuda(), torch.tensor([900], dtype=torch.int32).cuda(),
                                 D ** -0.5, num_splits=splits)
        k, v = b.rows(0)
        exp = OA.suffix_prefill_attention(_f64(q), k, v, 899, D ** -0.5)
        mag = OA.suffix_prefill_attention(_f64(q), k, np.abs(v), 899, D ** -0.5)
        score = np.abs(_f64(q)).max() * np.abs(k).max() * D * D ** -0.5
        lost = len(k) * 2.0 ** -126 * np.abs(v).max()   # (as for the prefill)
        _within(_f64(out), exp, (2 * B8 + 2.0 ** -12 + 2 * score * 2.0 ** -22) * mag + B8 * np.abs(exp) + lost, name)


def _large_values(D, pattern, step, times, power=96):
    """A batch of one request whose values reach 2^power and whose scores (base 2, queries of ones, a softmax scale of
    ln 2) are pattern[i % len] in the i-th `step` keys, the pattern `times` times (but for the last 5 keys)."""
    n = step * times * len(pattern) - 5
    b = Batch(8, 2, D, [n], [0], seed=79, spread=0)
    pages = b.pages.copy()
    g = np.random.default_rng(80)
    parts = {0: (0, 0), 22: (16, 6), 24: (24, 0), 26: (24, 2), 28: (24, 4)}   # values at the scale 4
    for t in range(n):
        key = np.zeros(D)
        key[:2] = parts[pattern[t // step % len(pattern)]]
        for h in range(2):
            value = g.choice([2.0 ** power, 2.0 ** power, 2.0 ** (power - 1), -2.0 ** (power - 2)], D)
            value[::3] = 2.0 ** power
            F.store(pages[b.bt[0, t // BS], h], D, t % BS, key, value)
    b.host(pages)
    k, v = b.rows(0)
    assert np.array_equal(k[:, 0].sum(-1), np.array([pattern[t // step % len(pattern)] for t in range(n)]))
    assert np.abs(v).max() == 2.0 ** power
    return b, n


LN2 = float(np.log(2.0))


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pattern", [(0, 26, 26), (0, 24, 24, 26), (0, 24, 24), (0, 22, 22, 22), (0, 22), (28, 0, 28)])
def test_decode_values_of_2_to_96_behind_a_base_that_stays(D, splits, pattern):
    """Values up to 2^96 stay in range however far scores have risen above the first chunk's: sums in which every
    key counts up to 2^26 times the base's are within the rule by which the base moves, or move it. The largest
    sum of weights, over all lanes and waves, times 2^96 has to stay below 2^128. (A wave's chunks are the pattern.)"""
    b, n = _large_values(D, pattern, 32, 4 * splits)
    q = torch.ones(1, 8, D, dtype=torch.bfloat16)
    out = cw.decode_attn_fp4(q.cuda(), b.cache, torch.from_numpy(b.bt).cuda(), torch.tensor([n], dtype=torch.int32).cuda(),
                             LN2, num_splits=splits)
    _check_attention(_f64(out), _f64(q), *b.rows(0), n - 1, LN2, f"D={D} {pattern}")


@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pattern", [(0, 24, 24), (0, 24, 24, 26), (28, 0, 28)])
def test_prefill_values_of_2_to_96_behind_a_base_that_stays(D, splits, pattern):
    b, n = _large_values(D, pattern, 64, 4)
    b.P, b.S, b.T, b.cu = [n - 6], [6], 6, np.array([0, 6], np.int32)
    q = torch.ones(6, 8, D, dtype=torch.bfloat16)
    out = _run_prefill(b.meta(), q.cuda(), b.cache, LN2, splits)
    _check_attention(out, _f64(q), *b.rows(0), n - 6, LN2, f"D={D} {pattern}")


@pytest.mark.parametrize("splits", [1, 3])
def test_decode_lengths_out_of_range_and_foreign_blocks(splits):
    """A length beyond the table counts as the table's; a negative one as 0; blocks outside the pool are zero keys
    and values."""
    b = Batch(8, 2, 64, [100, 64, 80], [0] * 3, seed=22)
    b.L = [b.stride * BS] * 3
    for r in range(3):   # every table entry names a block of whole rows, or none
        b.bt[r] = np.arange(b.stride) % b.nb
    pages = b.pages.copy()
    pages[:, :, 16 * 64:][pages[:, :, 16 * 64:] == 255] = 124
    b.host(pages)
    b.bt[2, 1], b.bt[2, 3] = -5, b.nb
    lens = [10 ** 9, -3, 75]
    q = b.queries(3)
    out = cw.decode_attn_fp4(q.cuda(), b.cache, torch.from_numpy(b.bt).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                             0.125, num_splits=splits)
    torch.cuda.synchronize()
    _check_decode(b, lens, q, out, 0.125, "out of range")


@pytest.mark.parametrize("splits", [1, 4])
@pytest.mark.parametrize("key,sees", [(0, True), (299, True), (300, False)])
def test_decode_nan_scales(splits, key, sees):
    """A NaN scale of keys makes its KV head's outputs NaN, one of values its columns; behind the length neither does."""
    b = Batch(8, 2, 64, [320, 40], [0, 0], seed=24)
    q, lens = b.queries(2).cuda(), torch.tensor([300, 40], dtype=torch.int32).cuda()
    bt, start = torch.from_numpy(b.bt).cuda(), b.pages
    for which in (0, 1):
        b.host(start)
        b.set_scale(which, 0, key, 1, 1, 255)
        out = _f64(cw.decode_attn_fp4(q, b.cache, bt, lens, 0.125, num_splits=splits))
        bad = np.zeros(out.shape, bool)
        if sees:
            bad[0, 4:, slice(None) if which == 0 else slice(32, 64)] = True
        assert np.array_equal(np.isnan(out), bad), which


def test_decode_captured_replays_follow_growing_lengths():
    """Two captured decode calls with workspaces of their own, replayed in turn with other lengths and queries,
    equal eager calls each time."""
    lens = [40, 200, 7]
    b = Batch(8, 2, 128, [n + 60 for n in lens], [0] * 3, seed=23)
    bt = torch.from_numpy(b.bt).cuda()
    sets = []
    for _ in range(2):
        q = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda")
        sl = torch.ones(3, dtype=torch.int32, device="cuda")
        ws = torch.empty(cw.decode_workspace_bytes_fp4(3, 8, 128, 4), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            cw.decode_attn_fp4(q, b.cache, bt, sl, 128 ** -0.5, num_splits=4, workspace=ws, out=out)
        sets.append((q, sl, ws, out, graph))
    for step in range(4):
        want = []
        for i, (q, sl, ws, out, graph) in enumerate(sets):
            q.copy_(b.queries(3).cuda())
            sl.copy_(torch.tensor([n + 7 * step + i for n in lens], dtype=torch.int32))
            want.append(cw.decode_attn_fp4(q, b.cache, bt, sl, 128 ** -0.5, num_splits=4))
        torch.cuda.synchronize()
        for s in sets:
            s[4].replay()
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            assert torch.equal(_bits(s[3]), _bits(w)), step


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("D,rotary,interleaved", [(64, 64, False), (128, 64, True)])
def test_prompt_then_decode_steps(D, rotary, interleaved):
    """A layer as it is used: append, prefill attention, then three decode steps, on another stream than the default;
    at last the rows taken back. Each call is checked against its oracle on what the calls before it left."""
    hq, hkv = 8, 2
    P, S, steps = [16, 0, 5], [20, 33, 1], 3
    b = Batch(hq, hkv, D, [p + s + steps for p, s in zip(P, S)], [0] * 3, seed=31, held=P)
    rope = _table(64, rotary)
    stream = torch.cuda.Stream()
    lens = list(P)
    for step in range(1 + steps):
        n = S if step == 0 else [1, 1, 1]
        b.P, b.S, b.cu, b.T = lens, n, np.concatenate([[0], np.cumsum(n)]).astype(np.int32), sum(n)
        b.L = [a + c for a, c in zip(lens, n)]
        q, k, v = _append_inputs(b, std=1.0)
        meta = b.meta()
        seq = torch.tensor(b.L, dtype=torch.int32).cuda()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            qr = cw.rope_append_fp4(meta, k, v, b.cache, q=q, rope=rope, interleaved=interleaved)
            if step == 0:
                out = cw.suffix_prefill_attn_fp4(meta, qr, b.cache, D ** -0.5)
            else:
                out = cw.decode_attn_fp4(qr, b.cache, meta.bt, seq, D ** -0.5)
        stream.synchronize()
        what = f"step {step}"
        _check_append(b, q, k, v, rope, interleaved, qr, what)
        b.pages = b.cache.pages.cpu().numpy()
        for i in range(3):
            rows = slice(b.cu[i], b.cu[i + 1])
            _check_attention(_f64(out[rows]), _f64(qr[rows]), *b.rows(i), lens[i], D ** -0.5, what)
        lens = list(b.L)
    whole = cw.BatchMeta(b.bt, np.concatenate([[0], np.cumsum(lens)]), [0] * 3, hq, hkv, D)
    k, v = cw.cache_rows_fp4(whole, b.cache)
    for i in range(3):
        at = slice(whole.cu_host[i], whole.cu_host[i + 1])
        for got, want in zip((k, v), b.rows(i)):
            assert np.array_equal(_f64(got[at]), want)


def _layer(seed, P, S, hq=8, hkv=2, D=64):
    """A cache with room, one call's static inputs, and a layer's calls over them."""
    b = Batch(hq, hkv, D, P, S, seed=seed, held=P)
    meta, rope = b.meta(), _table(max(b.L) + 8, D)
    meta.split_plan(3)   # (its copy to the device is not for a graph)
    seq = torch.tensor(b.L, dtype=torch.int32).cuda()
    qkv = torch.zeros(b.T, (hq + 2 * hkv) * D, dtype=torch.bfloat16, device="cuda")
    q, k, v = (t.view(b.T, -1, D) for t in qkv.split([hq * D, hkv * D, hkv * D], 1))

    def run(cache, stream=None):
        qr = cw.rope_append_fp4(meta, k, v, cache, q=q, rope=rope, stream=stream)
        out = [qr, cw.suffix_prefill_attn_fp4(meta, qr, cache, D ** -0.5, stream=stream),
               cw.suffix_prefill_attn_split_fp4(meta, qr, cache, D ** -0.5, num_splits=3, stream=stream),
               *cw.cache_rows_fp4(meta, cache, stream=stream)]
        if stream is None:
            last = qr[(meta.cu[1:] - 1).long()]
            out.append(cw.decode_attn_fp4(last, cache, meta.bt, seq, D ** -0.5, num_splits=3))
        return out

    return b, qkv, run


def test_layer_captured_and_replayed():
    """The calls in one captured graph, replayed with other inputs between eager runs on a copy of the cache: every
    replay has the eager run's bits, in its results and in the cache."""
    b, qkv, run = _layer(51, [20, 0, 37], [9, 17, 1])
    twin = cw.Fp4KvCache.of(b.cache.pages.clone())
    run(cw.Fp4KvCache.of(b.cache.pages.clone()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        got = run(b.cache)
    for step in range(4):
        qkv.copy_(_normal(b.g, *qkv.shape).cuda())
        want = [t.clone() for t in run(twin)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, e) in enumerate(zip(got, want)):
            assert torch.equal(_bits(a), _bits(e)), (step, i)
        assert torch.equal(b.cache.pages, twin.pages), step


def test_layer_on_given_streams():
    """With stream=: two layers' calls on two streams at once equal the ones on the current stream, and what the
    calls allocate comes from their stream's memory."""
    sets = [_layer(seed, [20, 0, 37], [40, 117, 1]) for seed in (52, 53)]
    for b, qkv, _ in sets:
        qkv.copy_(_normal(b.g, *qkv.shape).cuda())
    want = [run(cw.Fp4KvCache.of(b.cache.pages.clone())) for b, _, run in sets]
    caches = [cw.Fp4KvCache.of(b.cache.pages.clone()) for b, *_ in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [run(c, stream=s) for (*_, run), c, s in zip(sets, caches, streams)]
    torch.cuda.synchronize()
    for g, w, s in zip(got, want, streams):
        for i, (a, e) in enumerate(zip(g, w)):
            assert torch.equal(_bits(a), _bits(e)), i
            seg = [m for m in torch.cuda.memory_snapshot()
                   if m["address"] <= a.data_ptr() < m["address"] + m["total_size"]]
            assert [m["stream"] for m in seg] == [s.cuda_stream], i


def test_rows_alone_equal_rows_in_a_batch():
    """A request's codes do not depend on the rest of the batch, nor on how its tokens are cut into calls."""
    b = Batch(4, 2, 128, [5, 0], [50, 33], seed=56, held=[5, 0])
    q, k, v = _append_inputs(b)
    rope = _table(64, 128)
    start = b.cache.pages.clone()
    cw.rope_append_fp4(b.meta(), k, v, b.cache, q=q, rope=rope)
    one = cw.Fp4KvCache.of(start)
    for r in range(2):
        for a in range(0, b.S[r], 7):
            e = min(b.S[r], a + 7)
            rows = slice(b.cu[r] + a, b.cu[r] + e)
            meta = cw.BatchMeta(b.bt[r:r + 1], [0, e - a], [b.P[r] + a], 4, 2, 128)
            cw.rope_append_fp4(meta, k[rows], v[rows], one, rope=rope)
    assert torch.equal(one.pages, b.cache.pages)


def test_blocks_beyond_32_bit_offsets():
    """Blocks at the end of a cache of 6.5 GB: append, rows, prefill (whole and in runs) and decode have the bits
    that they have in a small one."""
    nb, hkv, D, hq, S = 600000, 5, 128, 15, [300, 70]
    g = _gen(94)
    big = np.full((2, 25), -1, np.int32)
    small = big.copy()
    order = torch.randperm(26, generator=g).numpy()
    ids = np.concatenate([np.arange(nb - 20, nb), [0, 1, 2 ** 18 - 1, 2 ** 18, 2 ** 18 + 1, nb // 2]])[order]
    for r, (a, n) in enumerate(((0, 19), (19, 5))):
        big[r, :n], small[r, :n] = ids[a:a + n], np.arange(a, a + n)
    rope = _table(512, D)
    qkv = _normal(g, sum(S), (hq + 2 * hkv) * D).cuda()
    q, k, v = (t.view(sum(S), -1, D) for t in qkv.split([hq * D, hkv * D, hkv * D], 1))
    lens = torch.tensor(S, dtype=torch.int32).cuda()
    res = []
    for n, table in ((nb, big), (26, small)):
        cache = cw.Fp4KvCache(n, hkv, D)
        meta = cw.BatchMeta(table, np.concatenate([[0], np.cumsum(S)]), [0, 0], hq, hkv, D)
        qr = cw.rope_append_fp4(meta, k, v, cache, q=q, rope=rope)
        out = [qr, cw.suffix_prefill_attn_fp4(meta, qr, cache, 0.088),
               cw.suffix_prefill_attn_split_fp4(meta, qr, cache, 0.088, num_splits=3), *cw.cache_rows_fp4(meta, cache)]
        out += [cw.decode_attn_fp4(qr[:2], cache, meta.bt, lens, 0.088, num_splits=m) for m in (1, 4)]
        full = torch.from_numpy(np.concatenate([table[0, :18], table[1, :4]])).cuda().long()   # whole blocks
        out.append(cache.pages[full])
        res.append(out)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(*res)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_appends_of_more_rows_than_caches_hold_equal_their_parts(D, interleaved):
    """8,200 rows of 8,192 query columns (273 MB or more with what is written) in a call have the bits of a call for each request."""
    hq, hkv, P, S = 8192 // D, 2, [3, 16], [4100, 4100]
    stride = (16 + 4100 + 15) // 16
    bt = np.arange(2 * stride, dtype=np.int32).reshape(2, stride)[:, ::-1].copy()
    g = torch.Generator(device="cuda").manual_seed(95)
    qkv = torch.randn(8200, (hq + 2 * hkv) * D, generator=g, device="cuda").to(torch.bfloat16)
    q, k, v = (x.view(8200, -1, D) for x in qkv.split([hq * D, hkv * D, hkv * D], 1))
    rope = _table(4200, D)
    caches = [cw.Fp4KvCache.of(torch.zeros(2 * stride, hkv, 17 * D, dtype=torch.uint8, device="cuda")) for _ in range(2)]
    whole = cw.rope_append_fp4(cw.BatchMeta(bt, [0, 4100, 8200], P, hq, hkv, D), k, v, caches[0], q=q, rope=rope,
                               interleaved=interleaved)
    for r in range(2):
        rows = slice(4100 * r, 4100 * (r + 1))
        part = cw.rope_append_fp4(cw.BatchMeta(bt[r:r + 1], [0, 4100], P[r:r + 1], hq, hkv, D), k[rows], v[rows],
                                  caches[1], q=q[rows], rope=rope, interleaved=interleaved)
        assert torch.equal(_bits(part), _bits(whole[rows]))
    assert torch.equal(caches[0].pages, caches[1].pages)


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("D", [64, 128])
def test_decode_with_a_table_of_more_than_caches_hold(D, splits):
    """A table that could name 272 MB of pages or more: the bits that the table of the sequences' own blocks gives."""
    b = Batch(12, 4, D, [700, 33, 5], [0, 0, 0], seed=96)
    wide = np.full((3, 21000), -1, np.int32)
    wide[:, :b.bt.shape[1]] = b.bt
    q, lens = b.queries(3).cuda(), torch.tensor([700, 33, 0], dtype=torch.int32).cuda()
    got, want = (cw.decode_attn_fp4(q, b.cache, torch.from_numpy(np.ascontiguousarray(x)).cuda(), lens, D ** -0.5,
                                    num_splits=splits) for x in (wide, b.bt))
    assert torch.equal(_bits(got), _bits(want)) and not want[2].any() and not want.isnan().any()


def test_decode_calls_at_once_on_two_streams():
    """Two calls at the same time with workspaces that they allocate themselves."""
    b = Batch(8, 2, 128, [900, 300], [0, 0], seed=54)
    bt = torch.from_numpy(b.bt).cuda()
    qs = [b.queries(2).cuda() for _ in range(2)]
    sl = [torch.tensor(n, dtype=torch.int32).cuda() for n in ([900, 300], [850, 1])]
    want = [cw.decode_attn_fp4(q, b.cache, bt, n, 128 ** -0.5, num_splits=5) for q, n in zip(qs, sl)]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[cw.decode_attn_fp4(q, b.cache, bt, n, 128 ** -0.5, num_splits=5, stream=s) for _ in range(8)]
           for q, n, s in zip(qs, sl, streams)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(_bits(t), _bits(w)) for t in g)


def test_batches_with_no_rows():
    """Batches whose requests are all empty launch nothing; the cache keeps its bytes."""
    b = Batch(8, 2, 64, [20, 0], [0, 0], seed=55)
    before = b.cache.pages.clone()
    none = torch.empty(0, 8, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert cw.rope_append_fp4(b.meta(), kv, kv, b.cache, q=none, rope=_table(64, 64)).shape == none.shape
    assert cw.suffix_prefill_attn_fp4(b.meta(), none, b.cache, 0.1).shape == none.shape
    assert cw.suffix_prefill_attn_split_fp4(b.meta(), none, b.cache, 0.1).shape == none.shape
    assert cw.cache_rows_fp4(b.meta(), b.cache)[1].shape == kv.shape
    torch.cuda.synchronize()
    assert torch.equal(before, b.cache.pages)


def test_python_refusals_on_the_gpu():
    b = Batch(8, 2, 64, [20], [4], seed=41)
    k = _normal(b.g, 4, 2, 64).cuda()
    with pytest.raises(cw.CwError, match="rope is required"):
        cw.rope_append_fp4(b.meta(), k, k, b.cache, q=b.queries().cuda())
    with pytest.raises(cw.CwError, match="rotary_dim"):
        cw.rope_append_fp4(b.meta(), k, k, b.cache, rope=torch.zeros(64, 12, 2, device="cuda"))
    with pytest.raises(ValueError, match="KV heads"):
        cw.rope_append_fp4(b.meta(), k, k, cw.Fp4KvCache(4, 2, 128))
    with pytest.raises(ValueError, match="row must be contiguous"):
        cw.rope_append_fp4(b.meta(), k.transpose(1, 2).contiguous().transpose(1, 2), k, b.cache)
    with pytest.raises(TypeError, match="k_rows"):
        cw.cache_rows_fp4(b.meta(), b.cache, k_rows=k.float())
    with pytest.raises(ValueError, match="k_rows must be"):
        cw.cache_rows_fp4(b.meta(), b.cache, k_rows=k[:2])
    with pytest.raises(TypeError, match="cache.pages"):
        cw.decode_attn_fp4(_normal(b.g, 1, 8, 64).cuda(), cw.Fp4KvCache.of(b.cache.pages.view(torch.int8)),
                           torch.from_numpy(b.bt).cuda(), torch.ones(1, dtype=torch.int32).cuda(), 0.1)
    with pytest.raises(cw.CwError, match="workspace"):
        cw.decode_attn_fp4(_normal(b.g, 1, 8, 64).cuda(), b.cache, torch.from_numpy(b.bt).cuda(),
                           torch.ones(1, dtype=torch.int32).cuda(), 0.1, num_splits=2,
                           workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
