"""CPU oracle of the 8-bit cache's rows (test infrastructure only), from the rule in include/hardkv.h.

Every step that the rule rounds to fp32 is formed in float64 and rounded once: products of two fp32
numbers are exact there, and a quotient's second rounding moves nothing (53 >= 2 * 24 + 2).
"""
from __future__ import annotations

import math

import numpy as np

LEAST = 2.0 ** -100
MOST = {"i8": 127.0, "e4m3": 448.0}


def _f32(x):
    return np.float64(np.float32(x))


def e4m3_code(x: float) -> int:
    """Bits of the nearest 8-bit float (4 exponent bits, bias 7, 3 mantissa bits; ties to even)."""
    sign = 0x80 if math.copysign(1.0, x) < 0 else 0
    a = min(abs(x), 448.0)
    if a == 0.0:
        return sign
    e = max(math.frexp(a)[1] - 1, -6)
    n = round(a / 2.0 ** (e - 3))                  # (Python rounds ties to even)
    if n == 16:
        e, n = e + 1, 8
    return sign | (n if n < 8 else (e + 7) << 3 | (n - 8))


def e4m3_value(b: int) -> float:
    exp, man = b >> 3 & 15, b & 7
    if exp == 15 and man == 7:
        return math.nan
    a = man * 2.0 ** -9 if exp == 0 else (8 + man) * 2.0 ** (exp - 10)
    return -a if b & 0x80 else a


def quantise(row, fmt: str):
    """(codes as bytes, scale) of one row of finite or other numbers."""
    x = np.asarray(row, np.float64)
    if not np.isfinite(x).all():
        return np.zeros(len(x), np.uint8), math.nan
    a = max(float(np.abs(x).max()), LEAST)
    up = _f32(MOST[fmt] / a)
    y = [float(_f32(v * up)) for v in x]
    if fmt == "i8":
        codes = np.array([round(v) for v in y], np.int64).astype(np.int8).view(np.uint8)
    else:
        codes = np.array([e4m3_code(v) for v in y], np.uint8)
    return codes, float(_f32(a / MOST[fmt]))


def values(codes, fmt: str):
    """What codes (bytes, any shape) stand for, without their scale."""
    c = np.asarray(codes, np.uint8)
    if fmt == "i8":
        return c.view(np.int8).astype(np.float64)
    return np.array([e4m3_value(b) for b in range(256)])[c]
