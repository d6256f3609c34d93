"""fp64 restatement of the batch-serving operators: rotary positions, e4m3 / bf16 pages, ragged paged attention.

Plain numpy, no code shared with the CUDA path; loops where a loop is the definition.
"""
import math

import numpy as np

MIN_EXP, MAX_EXP = -110, 119      # range of a row's scale exponent
NAN_CODE = 0x7F


def e4m3_values() -> np.ndarray:
    """Value of every 8-bit code: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN, no infinities."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = (1 + m / 8) * 2.0 ** (e - 7) if e else (m / 8) * 2.0 ** -6
        out[c] = math.nan if (c & 0x7F) == 0x7F else (-v if c & 0x80 else v)
    return out


def quantise_row(x):
    """(codes uint8 [d], scale byte) of one row by the definition, every code found by search."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    most = np.abs(x[fine]).max() if fine.any() else 0.0
    e = MIN_EXP
    while e < MAX_EXP and most > 448.0 * 2.0 ** e:
        e += 1
    table = e4m3_values()[:127]                     # non-negative finite codes, ascending
    y = np.minimum(np.abs(x) * 2.0 ** -e, 448.0)
    y[~fine] = 0.0
    hi = np.searchsorted(table, y).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    low, high = y - table[lo], table[hi] - y
    code = np.where((low < high) | ((low == high) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(fine, code, NAN_CODE).astype(np.uint8), e + 127


def rope_frequencies(rotary, base, scaling="none", factor=1.0, ctx=0.0, low=1.0, high=32.0):
    out = []
    for j in range(rotary // 2):
        b = base * factor ** (rotary / (rotary - 2)) if scaling == "ntk" else base
        theta = b ** (-2.0 * j / rotary)
        if scaling == "linear":
            theta /= factor
        if scaling == "parts":
            turns = ctx * theta / (2 * math.pi)
            g = min(max((turns - low) / (high - low), 0.0), 1.0)
            theta = (1 - g) * theta / factor + g * theta
        out.append(theta)
    return np.array(out)


def rope(x, positions, theta, layout, gain=1.0, backward=False):
    """x [T, H, d] fp64."""
    y = np.array(x, dtype=np.float64)
    half = len(theta)
    for t, p in enumerate(positions):
        for j in range(half):
            a, b = (j, j + half) if layout == "half" else (2 * j, 2 * j + 1)
            ang = -float(p) * theta[j] if backward else float(p) * theta[j]
            c, s = math.cos(ang) * gain, math.sin(ang) * gain
            y[t, :, a], y[t, :, b] = x[t, :, a] * c - x[t, :, b] * s, x[t, :, b] * c + x[t, :, a] * s
    return y


def attend(q, k, v, scale):
    """q [Hq, d], k and v [n, Hkv, d] -> (out [Hq, d], lse [Hq], weight of |v| [Hq, d], largest sum |q k| scale)."""
    hq, d = q.shape
    n, hkv, _ = k.shape
    if n == 0:
        return np.zeros((hq, d)), np.full(hq, -np.inf), np.zeros((hq, d)), 0.0
    out, lse, size, most = np.empty((hq, d)), np.empty(hq), np.empty((hq, d)), 0.0
    for h in range(hq):
        g = h // (hq // hkv)
        s = k[:, g] @ q[h] * scale
        most = max(most, float((np.abs(k[:, g]) @ np.abs(q[h])).max() * scale))
        p = np.exp(s - s.max())
        out[h], size[h] = p @ v[:, g] / p.sum(), p @ np.abs(v[:, g]) / p.sum()
        lse[h] = s.max() + math.log(p.sum())
    return out, lse, size, most
