"""Oracle of rotary positions and of 8-bit pages: plain numpy in fp64 and Python
integers. Test infrastructure, like the rest of this package."""
from __future__ import annotations

import math

import numpy as np

PAGE = 64
NOT_FINITE = 32767
EXP_MIN, EXP_MAX = -96, 119


def phase_of(f):
    """Radians a position as a 64-bit fraction of a turn."""
    return round(math.fmod(f / (2 * math.pi), 1.0) * 2.0 ** 64) % 2 ** 64


def angle(phase, p):
    """2 pi of the fraction of a turn at position p, the product taken in integers."""
    u = (int(phase) * int(p)) % 2 ** 64
    return 2 * math.pi * ((u - 2 ** 64 if u >= 2 ** 63 else u) / 2.0 ** 64)


def pairs(n, layout):
    return [(i, i + n) if layout == "half" else (2 * i, 2 * i + 1) for i in range(n)]


def rotate(row, phases, pos, layout, factor=1.0, transpose=False):
    """One row [..., D] turned; pos: one position, or one for each pair."""
    y = np.array(row, dtype=np.float64)
    n = len(phases)
    for i, (a, b) in enumerate(pairs(n, layout)):
        t = angle(phases[i], pos[i] if np.ndim(pos) else pos)
        c, s = factor * math.cos(t), factor * math.sin(t) * (-1 if transpose else 1)
        u, v = np.array(row[..., a], dtype=np.float64), np.array(row[..., b], dtype=np.float64)
        y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    return y


def values():
    """The 127 finite non-negative e4m3 values, by code: four exponent bits of bias 7, three
    mantissa bits, subnormals, no infinities."""
    return np.array([(m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def power(amax):
    """The smallest e with amax <= 448 2^e, within its limits."""
    if not math.isfinite(amax):
        return NOT_FINITE
    e = EXP_MIN
    while e < EXP_MAX and amax > 448 * 2.0 ** e:
        e += 1
    return e


def encode(x, e):
    """Codes of x 2^-e: the nearest value, the even code of two equally near, the largest beyond it."""
    t = values()
    a = np.minimum(np.abs(np.asarray(x, dtype=np.float64)) * 2.0 ** -e, 448.0)
    hi = np.clip(np.searchsorted(t, a), 1, 126)
    lo = hi - 1
    up = (t[hi] - a < a - t[lo]) | ((t[hi] - a == a - t[lo]) & (hi % 2 == 0))
    return np.where(up, hi, lo).astype(np.uint8) | (np.signbit(x).astype(np.uint8) << 7)


def decode(codes, e):
    """Values of codes with a power (broadcast)."""
    t = np.append(values(), np.nan)
    c = np.asarray(codes)
    e = np.asarray(e, dtype=np.float64)
    v = np.where(c & 0x80, -1.0, 1.0) * t[c & 0x7f]
    return np.where(e == NOT_FINITE, np.nan, v * 2.0 ** np.where(e == NOT_FINITE, 0, e))


def quantize_page(x):
    """A page [64, Hkv, D]: codes and the power of each head."""
    es = [power(np.abs(x[:, g]).max()) for g in range(x.shape[1])]
    codes = np.stack([encode(x[:, g], 0 if e == NOT_FINITE else e) for g, e in enumerate(es)], 1)
    return codes, np.array(es, dtype=np.int16)
