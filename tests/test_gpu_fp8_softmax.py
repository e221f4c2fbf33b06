"""The running softmax of the attention calls over the 8-bit cache, where its base has to move: scores
that rise by tens to hundreds of powers of two along a sequence, or that stay level until the sum is
large. Each case asserts on the host that its inputs move the base.

Scores are made through column 0: key j has the value `profile[j]` there, a query row `factor /
(softmax_scale log2 e)`, so that its base-2 scores are factor * profile[j] and some noise from the
other columns.

Bounds, with A = sum p|v| / sum p: the probabilities' rounding to bf16 before the product 2^-8 A, that of
the row's sum of the same values (prefill) 2^-8 A, the exponential and the rest 2^-12 A, the output
2^-8 |o| (eps/2 of bf16 is 2^-8). A score is off by at most (D + 4) 2^-24 of its products' magnitudes
(fp32 sums) and, with its base, by four roundings of the largest base-2 score, 2^-22 of it; as a
factor of p that is e^delta, on both sums: 2 (e^delta - 1) A.
"""
import math

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import fp8 as F
from paper_2606_19667_amd import cw

pytestmark = pytest.mark.gpu

BS, STEP, CHUNK = 16, 64, 32
FACTORS = (1.0, 0.01, 0.25, -1.0, 0.0)
LOG2E = 1.0 / math.log(2.0)


def _f64(t):
    return t.detach().float().cpu().double().numpy()


class Cache:
    """One request's keys and values in blocks of random places; keys of KV head g rise by `profile`."""

    def __init__(self, profile, hkv, D, seed):
        self.D, self.hkv, self.n = D, hkv, len(profile)
        g = self.g = torch.Generator(device="cpu")
        g.manual_seed(seed)
        nblk = -(-self.n // BS)
        self.bt = torch.randperm(nblk + 3, generator=g)[:nblk].to(torch.int32).numpy()[None]
        k = torch.randn(nblk * BS, hkv, D, generator=g) * 0.25
        k[:, :, 0] = 0
        k[:self.n, :, 0] = torch.tensor(profile, dtype=torch.float32)[:, None]
        v = torch.randn(nblk * BS, hkv, D, generator=g)
        scale = [torch.exp2(torch.randint(lo, hi, (nblk + 3, hkv), generator=g).float()) for lo, hi in ((0, 3), (-9, 3))]
        at = torch.from_numpy(self.bt[0]).long()
        self.codes = []
        for x, unit in ((k, scale[0][at][:, :, None, None]), (v, 2.0 ** -7)):   # (values of blocks differ in size)
            c = torch.full((nblk + 3, hkv, BS, D), 0x7F, dtype=torch.uint8)
            c[at] = (x.view(nblk, BS, hkv, D).transpose(1, 2) / unit).clamp(-448, 448).to(cw.FP8).view(torch.uint8)
            for t in range(self.n, nblk * BS):   # NaN behind the last token
                c[at[t // BS], :, t % BS] = 0x7F
            self.codes.append(c)
        self.scale = scale
        self.cache = cw.Fp8KvCache.of(*(c.cuda().view(cw.FP8) for c in self.codes), *(s.cuda() for s in scale))
        self.k, self.v = (F.logical_rows(F.decode(c.numpy()), s.double().numpy(), self.bt[0], self.n)
                          for c, s in zip(self.codes, scale))

    def queries(self, factors, hq):
        """bf16 rows [len(factors), hq, D]; factors are the rows', or a list per row the heads'."""
        q = torch.randn(len(factors), hq, self.D, generator=self.g) * 0.2
        q[..., 0] = torch.tensor(factors, dtype=torch.float32).view(len(factors), -1) * math.log(2.0) * math.sqrt(self.D)
        return q.to(torch.bfloat16)

    def scores(self, q, sees):
        """Base-2 scores [rows, hq, n], -inf where row i does not see key j (sees[i] keys)."""
        s = np.einsum("rghd,jgd->rghj", q.reshape(len(q), self.hkv, -1, self.D), self.k).reshape(len(q), -1, self.n)
        s = s * (LOG2E * self.D ** -0.5)
        return np.where(np.arange(self.n) < np.asarray(sees)[:, None, None], s, -np.inf)

    def check(self, got, q, prefix, what):
        scale = self.D ** -0.5
        n = prefix + len(q)
        k, v = self.k[:n], self.v[:n]
        exp = OA.suffix_prefill_attention(q, k, v, prefix, scale)
        mag = OA.suffix_prefill_attention(q, k, np.abs(v), prefix, scale)
        qg = np.abs(q).reshape(len(q), self.hkv, -1, self.D)
        most = np.einsum("rghd,jgd->rghj", qg, np.abs(k)).max(-1).reshape(len(q), -1) * (scale * LOG2E)
        delta = math.log(2.0) * ((self.D + 4) * 2.0 ** -24 + 2.0 ** -22) * most
        bound = (2.0 ** -7 + 2.0 ** -12 + 2 * np.expm1(delta))[..., None] * mag + 2.0 ** -8 * np.abs(exp)
        err = np.abs(got - exp)
        print(f"{what}: max_err={err.max():.3e} worst_margin={(err - bound).max():.3e}", flush=True)
        assert np.isfinite(got).all(), what
        assert (err <= bound).all(), (what, float((err - bound).max()))


def _moves(scores, first, last):
    """How often a row's base moves over the steps first .. last - 1 of 64 keys: the base is the first step's
    maximum until the sum of powers of two passes 2^30."""
    base, total, moves = None, 0.0, 0
    for j in range(first, last):
        x = scores[j * STEP:(j + 1) * STEP]
        if base is None:
            base = x.max() if np.isfinite(x.max()) else 0.0
        add = float(np.exp2(np.minimum(x - base, 1000.0)).sum())
        if total + add > 2.0 ** 30:
            to = max(x.max(), base + math.log2(total) if total > 1 else base)
            total, base, moves = total * 2.0 ** (base - to), to, moves + 1
            add = float(np.exp2(x - base).sum())
        total += add
    return moves


RISING = [0, 60, 144, 144, 416, 96, 0, 40, 112, 240, 416, 448]
LEVEL = [0] + [22] * 23
PROFILES = {"rising": RISING, "level": LEVEL}


@pytest.mark.parametrize("name", sorted(PROFILES))
@pytest.mark.parametrize("hq,hkv,D", [(4, 1, 128), (4, 2, 64), (7, 1, 128), (1, 1, 64)])
@pytest.mark.parametrize("splits", [0, 1, 2, 3])
def test_prefill_base_moves(name, hq, hkv, D, splits):
    """Rows whose base moves in several steps beside rows of the same wave whose base stays; without runs
    (0) and with."""
    print(f"prefill base {name} {hq}/{hkv} D={D} splits={splits}", flush=True)
    profile = np.repeat(PROFILES[name], STEP)
    S = 45
    c = Cache(profile, hkv, D, seed=len(profile) + hq + D)
    P = c.n - S
    q = c.queries([FACTORS[i % 5] for i in range(S)], hq)
    qf = _f64(q)
    s = c.scores(qf, P + 1 + np.arange(S))
    steps = len(PROFILES[name])
    runs = max(splits, 1)
    cuts = [steps * i // runs for i in range(runs + 1)]
    moves = np.array([[[_moves(s[i, h], a, b) for a, b in zip(cuts, cuts[1:])] for h in range(hq)] for i in range(S)])
    still = [i for i in range(S) if FACTORS[i % 5] in (0.01, 0.0)]
    if name == "rising":
        assert (moves[::5].max(-1) >= (3 if runs == 1 else 1)).all() and (moves[still] == 0).all()
    elif runs == 1:   # (a run of its own starts at its scores' level)
        assert (moves[::5] >= 1).all() and (moves[still] == 0).all()
    meta = cw.BatchMeta(c.bt, [0, S], [P], hq, hkv, D)
    out = (cw.suffix_prefill_attn_fp8(meta, q.cuda(), c.cache, D ** -0.5) if splits == 0 else
           cw.suffix_prefill_attn_split_fp8(meta, q.cuda(), c.cache, D ** -0.5, num_splits=splits))
    torch.cuda.synchronize()
    c.check(_f64(out), qf, P, f"prefill base {name}")


LAZY = 8.0   # the base of a decode call's wave moves when a score passes it by more
CLIMB = [0, 12, 40, 40, 30, 104, 208, 208, 16, 48, 0, 9, 80, 240, 320, 448]


@pytest.mark.parametrize("hq,hkv,D", [(4, 1, 128), (10, 2, 64), (40, 2, 128), (1, 1, 64)])
@pytest.mark.parametrize("splits", [1, 2])
@pytest.mark.parametrize("cut", [0, 77])
def test_decode_base_moves(hq, hkv, D, splits, cut):
    """Heads whose scores rise by 9 to 200 powers of two over the chunks of a wave, beside heads that stay."""
    print(f"decode base {hq}/{hkv} D={D} splits={splits} cut={cut}", flush=True)
    profile = np.repeat(CLIMB, 4 * CHUNK)[:16 * 4 * CHUNK - cut]
    c = Cache(profile, hkv, D, seed=hq + D + cut)
    f = [FACTORS[h % 5] for h in range(hq)]
    q = c.queries([f], hq)
    qf = _f64(q)
    s = c.scores(qf, [c.n])[0]
    chunks = -(-c.n // CHUNK)
    for split in range(splits):
        a, b = chunks * split // splits, chunks * (split + 1) // splits
        for wave in range(4):
            tops = [s[:, j * CHUNK:(j + 1) * CHUNK].max(1) for j in range(a + wave, b, 4)]
            assert len(tops) >= 8 - bool(cut)
            rises = sum(t[0] > np.max([u[0] for u in tops[:i]]) + LAZY for i, t in enumerate(tops) if i)
            assert rises >= 2, (split, wave)
    bt, n = torch.from_numpy(c.bt).cuda(), torch.tensor([c.n], dtype=torch.int32).cuda()
    out = cw.decode_attn_fp8(q.cuda(), c.cache, bt, n, D ** -0.5, num_splits=splits)
    torch.cuda.synchronize()
    c.check(_f64(out), qf, c.n - 1, "decode base")
