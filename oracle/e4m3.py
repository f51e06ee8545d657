"""8-bit keys and values -- oracle (test infrastructure only).

A block is one token's numbers of one kv-head.  Its scale is the smallest power of
two 2^e with max |x| <= 448 * 2^e, at least 2^-117; a number is stored as x / 2^e
rounded to the nearest e4m3 number, ties to the even one, and read as that times 2^e.
Where a key or value of a token and kv-head is not finite, all of them read as NaN.

The e4m3 numbers are built here from the format (1 sign, 4 exponent bits with bias 7,
3 mantissa bits, the all-ones pattern NaN, no infinities) and rounding is a search
among them.
"""
from __future__ import annotations

import numpy as np


def _positive_numbers() -> np.ndarray:
    """The 127 numbers of codes 0 .. 126, ascending."""
    out = []
    for code in range(127):
        e, m = code >> 3, code & 7
        out.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(out)


NUMBERS = _positive_numbers()


def nearest(y: np.ndarray) -> np.ndarray:
    """y (|y| <= 448) rounded to the nearest e4m3 number, ties to the even code."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(NUMBERS, a), 1, 126)   # NUMBERS[hi - 1] < a <= NUMBERS[hi]
    lo = hi - 1
    up, down = NUMBERS[hi] - a, a - NUMBERS[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0))
    return np.copysign(NUMBERS[np.where(take_hi, hi, lo)], y)


def exponent(top: np.ndarray) -> np.ndarray:
    """The scale's exponent for blocks with largest magnitude `top` (finite)."""
    e = np.full(np.shape(top), -117)
    for cand in range(-117, 122):
        e = np.where(top > 448.0 * 2.0 ** cand, cand + 1, e)
    return e


def stored(x: np.ndarray) -> np.ndarray:
    """What blocks along the last axis read as after being stored (finite x)."""
    f = 2.0 ** exponent(np.abs(x).max(axis=-1, keepdims=True)).astype(np.float64)
    return nearest(x / f) * f


def store_kv(k: np.ndarray, v: np.ndarray):
    """(k, v) [..., D] as a cache in 8 bits reads them."""
    ok = np.isfinite(k).all(-1, keepdims=True) & np.isfinite(v).all(-1, keepdims=True)
    return (np.where(ok, stored(np.where(ok, k, 0.0)), np.nan), np.where(ok, stored(np.where(ok, v, 0.0)), np.nan))
