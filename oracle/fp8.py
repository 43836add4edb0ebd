"""Plain CPU oracle for activations in 8 bits: e4m3 values with a power-of-two
scale for each block of 128 features, the norm in front of a layer, and the
products with such activations.

TEST INFRASTRUCTURE.  Only ``tests/`` may import this module; the GPU library
shares no code with it.  Everything is float64; the e4m3 numbers come from
their definition (sign, 4 exponent bits with bias 7, 3 mantissa bits, code
0x7f a NaN), and rounding is a search among them.
"""

from __future__ import annotations

import math

import numpy as np

BLOCK = 128


def _table() -> np.ndarray:
    """The value of every e4m3 code."""
    out = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        v = math.ldexp(f, -9) if e == 0 else math.ldexp(8 + f, e - 10)
        out[c] = math.nan if c & 127 == 127 else (-v if c & 128 else v)
    return out


E4M3 = _table()
_POSITIVE = E4M3[:127]          # ascending, 0 .. 448


def round_e4m3(v: np.ndarray) -> np.ndarray:
    """v rounded to the nearest e4m3 number, of two equally near the one with an
    even code; beyond 448 and for infinities and NaN a NaN (a block's scale
    leaves no finite value there)."""
    v = np.asarray(v, dtype=np.float64)
    a = np.abs(v)
    out = np.full(v.shape, np.nan)
    ok = a <= 448.0
    up = np.searchsorted(_POSITIVE, a[ok])
    lo, hi = np.maximum(up - 1, 0), up
    dlo, dhi = a[ok] - _POSITIVE[lo], _POSITIVE[hi] - a[ok]
    code = np.where((dlo < dhi) | ((dlo == dhi) & (lo % 2 == 0)), lo, hi)
    out[ok] = np.copysign(_POSITIVE[code], v[ok])
    return out


def scale_exponents(x: np.ndarray, block_rows: int = 1) -> np.ndarray:
    """e of each block's scale 2^e: the least e >= -127 with the block's largest
    finite magnitude <= 448 2^e, 0 for a block without one above 0.  (Values
    from 2^128 on count as infinite: float32 has none.)"""
    x = np.asarray(x, dtype=np.float64)
    T, m = x.shape
    B, G = -(-T // block_rows), -(-m // BLOCK)
    out = np.zeros((B, G), dtype=np.int64)
    for b in range(B):
        for g in range(G):
            a = np.abs(x[b * block_rows:(b + 1) * block_rows, g * BLOCK:(g + 1) * BLOCK])
            a = a[a < 2.0 ** 128]
            a = a.max() if a.size else 0.0
            if a > 0:
                f, e = math.frexp(a)               # a = f 2^e; 448 = 0.875 2^9
                out[b, g] = max(e - 9 + (1 if f > 0.875 else 0), -127)
    return out


def quantize(x: np.ndarray, block_rows: int = 1):
    """(values, exponents) of x [T, m]."""
    x = np.asarray(x, dtype=np.float64)
    e = scale_exponents(x, block_rows)
    wide = expand(e, *x.shape, block_rows)
    return round_e4m3(np.where(np.abs(x) < 2.0 ** 128, np.ldexp(x, -wide), np.nan)), e


def expand(s: np.ndarray, rows: int, m: int, block_rows: int = 1) -> np.ndarray:
    """A block scale for every element."""
    return np.repeat(np.repeat(s, block_rows, 0)[:rows], BLOCK, 1)[:, :m]


def dequantize(v: np.ndarray, e: np.ndarray, block_rows: int = 1) -> np.ndarray:
    return np.ldexp(v, expand(e, *v.shape, block_rows))


def rmsnorm(x, residual, gain, eps):
    """(y, h): h = x + residual summed in float32, y = (h gain) / root in float64
    (h gain is exact there)."""
    h = np.asarray(x, dtype=np.float32)
    if residual is not None:
        h = (h + np.asarray(residual, dtype=np.float32)).astype(np.float32)
    d = h.astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        hg = d if gain is None else d * np.asarray(gain, dtype=np.float64)
        return hg / np.sqrt(np.mean(d * d, axis=1, keepdims=True) + eps), h
