"""fp64 reference for the 8-bit layer path: e4m3 values, the norm that writes 8-bit
rows, the product with a scale per block of 128, and the append into an 8-bit cache.

TEST INFRASTRUCTURE ONLY (see the package docstring).

* e4m3 is the OCP format: sign, 4 exponent bits (bias 7), 3 mantissa bits; the
  pattern of all ones is NaN, so the largest value is 448 = 1.75 * 2^8 and there
  is no infinity; subnormals are multiples of 2^-9.
* Rounding is to nearest, ties to even.
* A cache block of 16 tokens holds, per KV head, codes and one power-of-two scale
  that its first rows set and later rows may only raise; rows already there are
  then rounded to the new scale.
"""
from __future__ import annotations

import math

import numpy as np

MAX = 448.0
GROUP = 128
MIN_EXP, MAX_EXP = -100, 120


def _as_f64(x) -> np.ndarray:
    if hasattr(x, "detach"):
        x = x.detach().to("cpu").double().numpy()
    return np.asarray(x, dtype=np.float64)


def decode(codes) -> np.ndarray:
    """Values of e4m3 codes (uint8)."""
    c = np.asarray(codes, dtype=np.uint8).astype(np.int64)
    sign = np.where(c & 0x80, -1.0, 1.0)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (8 + m) * np.exp2(e - 10.0), m * 2.0 ** -9)
    return np.where((c & 0x7F) == 0x7F, np.nan, sign * v)


def step(x) -> np.ndarray:
    """Distance of neighbouring e4m3 values at |x|."""
    a = np.abs(np.asarray(x, dtype=np.float64))
    with np.errstate(divide="ignore"):
        e = np.maximum(np.floor(np.log2(np.where(a > 0, a, 1e-300))), -6.0)
    return np.exp2(e - 3)


def round_value(x) -> np.ndarray:
    """The e4m3 value nearest to x (ties to the even code); infinite, NaN and too
    large ones are NaN."""
    x = np.asarray(x, dtype=np.float64)
    s = step(np.where(np.isfinite(x), x, 0.0))
    with np.errstate(invalid="ignore"):
        v = np.rint(x / s) * s
    return np.where(np.isfinite(x) & (np.abs(v) <= MAX), v, np.nan)


def add_rms_norm(x, residual, weight, eps: float):
    """h (the bf16 sum, given by the caller as `x` when residual is None), the
    normed rows y, and their scales per 128 columns. x and residual are bf16
    values; the sum is rounded to bf16 by the caller's choice of `x`."""
    h = _as_f64(x) if residual is None else _as_f64(x) + _as_f64(residual)
    y = h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps) * _as_f64(weight)[None, :]
    groups = [np.abs(y[:, a:a + GROUP]).max(axis=1) / MAX for a in range(0, y.shape[1], GROUP)]
    scales = np.stack(groups, axis=1)
    return y, np.where(scales > 0, scales, 1.0)


def linear(x8, x_scale, w8, w_scale, bias=None):
    """(y, sum of the magnitudes of its terms) of the block-scaled product; x8 and
    w8 are e4m3 values."""
    x, w, xs, ws = (_as_f64(t) for t in (x8, w8, x_scale, w_scale))
    k = np.arange(x.shape[1]) // GROUP
    xd = x * xs[:, k]
    wd = w * ws[np.arange(len(w)) // GROUP][:, k]
    y, mag = xd @ wd.T, np.abs(xd) @ np.abs(wd).T
    if bias is not None:
        y, mag = y + _as_f64(bias)[None, :], mag + np.abs(_as_f64(bias))[None, :]
    return y, mag


def linear_cut(x8, x_scale, w8, w_scale):
    """For every output the sum over groups of 8 consecutive columns of (a bound of) the
    group's largest scaled product, and the sum of their squares: what an arithmetic that
    cuts a group's products below its largest one can lose."""
    x, w, xs, ws = (_as_f64(t) for t in (x8, w8, x_scale, w_scale))
    pad = -x.shape[1] % 8
    gx = np.abs(np.pad(x, ((0, 0), (0, pad)))).reshape(len(x), -1, 8).max(axis=2)
    gw = np.abs(np.pad(w, ((0, 0), (0, pad)))).reshape(len(w), -1, 8).max(axis=2)
    b = np.arange(gx.shape[1]) // (GROUP // 8)
    gx, gw = gx * xs[:, b], gw * ws[np.arange(len(w)) // GROUP][:, b]
    return gx @ gw.T, (gx * gx) @ (gw * gw).T


def scale_for(amax: float) -> float:
    """Smallest 2^e with amax <= 448 * 2^e, e in [-100, 120]."""
    e = MIN_EXP
    while e < MAX_EXP and amax > MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append(values, scales, rows, block_table, cu, plen, block_size: int = 16):
    """The cache (values of the codes [nb, Hkv, bs, D] and scales [nb, Hkv]) after
    the suffix rows [T, Hkv, D] are appended; blocks outside it are dropped."""
    values, scales, rows = values.copy(), scales.copy(), _as_f64(rows)
    for r in range(len(plen)):
        p, end = int(plen[r]), int(plen[r]) + int(cu[r + 1] - cu[r])
        while p < end:
            stop = min(end, (p // block_size + 1) * block_size)
            b, a = int(block_table[r][p // block_size]), p % block_size
            new = rows[int(cu[r]) + p - int(plen[r]):int(cu[r]) + stop - int(plen[r])]
            if 0 <= b < len(values):
                for g in range(values.shape[1]):
                    x = new[:, g]
                    fin = np.abs(x[np.isfinite(x)])
                    s = scale_for(float(fin.max()) if fin.size else 0.0)
                    if a > 0:
                        s = max(s, float(scales[b, g]))
                        if s > scales[b, g]:
                            values[b, g, :a] = round_value(values[b, g, :a] * (scales[b, g] / s))
                    values[b, g, a:a + stop - p] = round_value(x / s)
                    scales[b, g] = s
            p = stop
    return values, scales


def logical_rows(values, scales, block_row, length: int, block_size: int = 16) -> np.ndarray:
    """A request's first `length` keys (or values) [length, Hkv, D]: code times scale
    through its block-table row; zeros for a block outside the cache."""
    out = np.zeros((length, values.shape[1], values.shape[3]))
    for j in range(math.ceil(length / block_size)):
        b, n = int(block_row[j]), min(block_size, length - j * block_size)
        if 0 <= b < len(values):
            out[j * block_size:j * block_size + n] = (values[b, :, :n] * scales[b][:, None, None]).transpose(1, 0, 2)
    return out
