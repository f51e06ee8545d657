"""Microscaled numbers and the operators of a decoder layer over them -- oracle (test
infrastructure only).

32 neighbours of a row share the scale 2^e, e the smallest integer with max |x| <= top 2^e
and at least -117; a number is stored as x / 2^e rounded to the nearest number of the
format, ties to the even one.  A block with a number that is not finite reads as NaN.
"""
from __future__ import annotations

import numpy as np

from . import e4m3

#: The formats' numbers of codes 0, 1, 2, ..., ascending, without the sign.
NUMBERS = {"e4m3": e4m3.NUMBERS, "e2m1": np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])}


def nearest_code(y: np.ndarray, fmt: str) -> np.ndarray:
    """Codes of y within the format's range: nearest number, ties to the even code; the
    sign bit above the magnitude's."""
    n = NUMBERS[fmt]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(n, a), 1, len(n) - 1)
    lo = hi - 1
    up, down = n[hi] - a, a - n[lo]
    mag = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return mag + np.where(np.signbit(y), 128 if fmt == "e4m3" else 8, 0)


def exponent(top: np.ndarray, fmt: str) -> np.ndarray:
    """The scale's exponent for blocks with largest magnitude `top` (finite)."""
    most = NUMBERS[fmt][-1]
    m, p = np.frexp(top / most)          # top / most = m 2^p, m in [0.5, 1): 2^p, or 2^(p-1) where m is 0.5
    e = np.where(top > most * np.exp2(p - 1.0), p, p - 1)
    return np.maximum(np.where(top > 0, e, -117), -117).astype(np.int64)


def quantise(x: np.ndarray, fmt: str):
    """(codes, scale bytes) of float64 rows; codes one a number."""
    R, C = x.shape
    b = x.reshape(R, C // 32, 32)
    ok = np.isfinite(b).all(-1, keepdims=True)
    b = np.where(ok, b, 0.0)
    e = exponent(np.abs(b).max(-1, keepdims=True), fmt)
    codes = nearest_code(b * np.exp2(-e.astype(np.float64)), fmt)
    return codes.reshape(R, C), np.where(ok, e + 127, 255)[..., 0]


def numbers(codes: np.ndarray, scales: np.ndarray, fmt: str) -> np.ndarray:
    """float64 numbers of codes (one a number) and scale bytes."""
    half = 128 if fmt == "e4m3" else 8
    n = np.append(NUMBERS[fmt], np.nan) if fmt == "e4m3" else NUMBERS[fmt]
    x = n[codes % half] * np.where(codes >= half, -1.0, 1.0)
    f = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return x * np.repeat(f, 32, axis=1)


def pack_e2m1(codes: np.ndarray) -> np.ndarray:
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def unpack_e2m1(b: np.ndarray) -> np.ndarray:
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[0], -1).astype(np.int64)


def norm(h: np.ndarray, gain: np.ndarray, eps: float) -> np.ndarray:
    return h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * gain


def gated(x: np.ndarray, g: np.ndarray) -> np.ndarray:
    with np.errstate(over="ignore", invalid="ignore"):
        return x * (g / (1.0 + np.exp(-g)))


def turned(x: np.ndarray, positions: np.ndarray, axes, freqs, adjacent: bool) -> np.ndarray:
    """Heads [rows, H, D] turned: pair j by positions[axes[j]] * freqs[j]."""
    y = np.array(x, dtype=np.float64)
    n = len(freqs)
    for j in range(n):
        a, b = (2 * j, 2 * j + 1) if adjacent else (j, j + n)
        t = positions[axes[j]].astype(np.float64)[:, None] * freqs[j]
        y[..., a], y[..., b] = x[..., a] * np.cos(t) - x[..., b] * np.sin(t), x[..., b] * np.cos(t) + x[..., a] * np.sin(t)
    return y
