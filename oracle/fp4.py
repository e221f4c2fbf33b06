"""fp64 reference for the 4-bit KV cache: e2m1 values, the scale of 32 columns, a page's
bytes, the rotation of part of a head, and the append.

TEST INFRASTRUCTURE ONLY (see the package docstring).

* e2m1 is the OCP format: sign, 2 exponent bits (bias 1), 1 mantissa bit, no infinity and
  no NaN; the magnitudes are 0, 0.5, 1, 1.5, 2, 3, 4, 6.
* A scale is 2^(c - 127) for a byte c; c = 255 makes its 32 values NaN.
* Rounding is to nearest, ties to the even code; what is larger is 6.
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
GROUP = 32
MIN_EXP, MAX_EXP = -100, 125
BS = 16


def value(code: int) -> float:
    return -VALUES[code - 8] if code >= 8 else VALUES[code]


def code_of(x: float) -> int:
    """The code of the value nearest to x, ties to the even code; the sign bit is x's."""
    a = abs(x)
    best = min(range(8), key=lambda c: (abs(a - VALUES[c]), c % 2))
    return best + (8 if math.copysign(1.0, x) < 0 else 0)


def exponent_for(amax: float) -> int:
    """The smallest e in [-100, 125] with amax <= 7 * 2^e."""
    e = MIN_EXP
    while e < MAX_EXP and amax > 7.0 * 2.0 ** e:
        e += 1
    return e


_TABLE = np.array(VALUES)


def round_rows(x):
    """(codes uint8 [..., D], scale bytes uint8 [..., D / 32]) of rows of 64-bit values."""
    x = np.asarray(x, dtype=np.float64)
    groups = x.reshape(x.shape[:-1] + (-1, GROUP))
    with np.errstate(invalid="ignore"):
        amax = np.abs(groups).max(-1)
    bad = ~np.isfinite(groups).all(-1) | ~(amax < 2.0 ** 128)
    exp = np.vectorize(exponent_for, otypes=[np.int64])(np.where(bad, 0.0, amax))
    y = np.where(bad[..., None], 0.0, groups) / np.exp2(exp.astype(np.float64))[..., None]
    off = np.abs(np.abs(y)[..., None] - _TABLE)
    # nearest, then the even code: an odd code loses where it is as near
    order = np.lexsort(np.broadcast_arrays(np.arange(8) % 2, off), axis=-1)
    code = order[..., 0].astype(np.uint8) | (np.signbit(y).astype(np.uint8) << 3)
    code = np.where(bad[..., None], 0, code).astype(np.uint8)
    return code.reshape(x.shape), np.where(bad, 255, exp + 127).astype(np.uint8)


def values_of(codes, scales):
    """Values of codes [..., D] with scale bytes [..., D / 32]."""
    c = np.asarray(codes).astype(np.int64)
    v = np.where(c >= 8, -1.0, 1.0) * _TABLE[c & 7]
    s = np.asarray(scales).astype(np.float64)
    s = np.where(s == 255, np.nan, np.exp2(s - 127))
    return v * np.repeat(s, GROUP, axis=-1)


# ------------------------------------------------------------- pages
def key_byte(D, t, d):
    return t * (D // 2) + d // 2


def value_byte(D, t, d):
    wide = D // 16
    return 8 * D + ((t // 4 * 16 + d // wide) * 4 + t % 4) * (D // 32) + d % wide // 2


def key_scale_byte(D, t, d):
    return 16 * D + t * (D // 32) + d // 32


def value_scale_byte(D, t, d):
    return 16 * D + D // 2 + d // 32 * 16 + t


def _places(D):
    t, d = np.meshgrid(np.arange(BS), np.arange(D), indexing="ij")
    return t, d


def unpack(pages, D):
    """((key codes, key scales), (value codes, value scales)) of pages [..., 17 D]: codes [..., 16, D]
    and scale bytes [..., 16, D / 32]."""
    t, d = _places(D)
    ts, ds = t[:, ::GROUP], d[:, ::GROUP]
    out = []
    for code_at, scale_at in ((key_byte, key_scale_byte), (value_byte, value_scale_byte)):
        out.append(((pages[..., code_at(D, t, d)] >> (4 * (d % 2)).astype(np.uint8)) & 15,
                    pages[..., scale_at(D, ts, ds)]))
    return tuple(out)


def store(page, D, t, key_row, value_row):
    """Writes token t's codes and scales of one page [17 D] (rows of 64-bit values [D])."""
    for row, code_at, scale_at in ((key_row, key_byte, key_scale_byte), (value_row, value_byte, value_scale_byte)):
        codes, scales = round_rows(row)
        even = np.arange(0, D, 2)   # (both codes of a byte are the token's)
        page[code_at(D, t, even)] = codes[::2] | (codes[1::2] << 4)
        page[scale_at(D, t, np.arange(0, D, GROUP))] = scales


def append(pages, k_rows, v_rows, block_table, cu, plen):
    """The pages [num_blocks, Hkv, 17 D] after the suffix rows [T, Hkv, D] (64-bit values) are
    appended; tokens of blocks outside the cache are dropped."""
    pages = pages.copy()
    D = pages.shape[2] // 17
    for r in range(len(plen)):
        for i in range(int(cu[r + 1] - cu[r])):
            t = int(plen[r]) + i
            b = int(block_table[r][t // BS])
            if 0 <= b < len(pages):
                for g in range(pages.shape[1]):
                    store(pages[b, g], D, t % BS, k_rows[int(cu[r]) + i, g], v_rows[int(cu[r]) + i, g])
    return pages


def logical_rows(pages, block_row, first: int, n: int):
    """(keys, values) [n, Hkv, D] of a request's tokens first .. first + n - 1; zeros for a block
    outside the cache."""
    D = pages.shape[2] // 17
    out = [np.zeros((n, pages.shape[1], D)) for _ in range(2)]
    for j in range(first // BS, -(-(first + n) // BS)):
        b = int(block_row[j])
        a, e = max(first, j * BS), min(first + n, j * BS + BS)
        if a < e and 0 <= b < len(pages):
            for o, (codes, scales) in zip(out, unpack(pages[b], D)):
                o[a - first:e - first] = values_of(codes, scales)[:, a - j * BS:e - j * BS].transpose(1, 0, 2)
    return out


def rotate(x, cos_sin, interleaved: bool):
    """Rows [T, heads, D] with the first 2 n columns rotated by cos_sin [T, n, 2], in 64 bits; pairs
    (j, j + n), or (2 j, 2 j + 1) interleaved."""
    x = np.array(x, dtype=np.float64)
    cos_sin = np.asarray(cos_sin, dtype=np.float64)
    n = cos_sin.shape[1]
    for j in range(n):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + n)
        c, s = cos_sin[:, None, j, 0], cos_sin[:, None, j, 1]
        x[:, :, a], x[:, :, b] = x[:, :, a] * c - x[:, :, b] * s, x[:, :, b] * c + x[:, :, a] * s
    return x


def exact_rotation(row, cos_sin, interleaved: bool):
    """One row [D] rotated by cos_sin [n, 2] in rational arithmetic: a list of D Fractions (finite inputs). Two
    products may lie further apart than the 53 bits of a double."""
    out = [Fraction(float(u)) for u in row]
    n = len(cos_sin)
    for j in range(n):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + n)
        (x, y), (c, s) = (out[a], out[b]), (Fraction(float(t)) for t in cos_sin[j])
        out[a], out[b] = x * c - y * s, y * c + x * s
    return out


def exact_codes(row):
    """(codes [D], scale bytes [D / 32]) of a row of Fractions, as `round_rows` has them of 64-bit values; the
    code of a negative value that rounds to zero, or of zero, is 0."""
    codes, scales = [], []
    for at in range(0, len(row), GROUP):
        group = row[at:at + GROUP]
        e = MIN_EXP
        while e < MAX_EXP and max(map(abs, group)) > 7 * Fraction(2) ** e:
            e += 1
        scales.append(e + 127)
        for u in group:
            a = abs(u) / Fraction(2) ** e
            c = min(range(8), key=lambda i: (abs(a - Fraction(VALUES[i])), i % 2))
            codes.append(c + 8 if u < 0 and c else c)
    return np.array(codes, np.uint8), np.array(scales, np.uint8)
