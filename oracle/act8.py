"""Activation checkpoints in 8 bits (oracle): e4m3 codes with one power-of-two
scale per 32 consecutive rows of a column, in float64 from the definitions.

e4m3 has a 3-bit mantissa, exponents -6..8, subnormal step 2^-9, largest value
448 and no infinity.  A group's exponent e is the smallest with its largest
finite magnitude <= 448 * 2^e, kept within [EMIN, EMAX] of the half format.
"""
from __future__ import annotations

import numpy as np

GROUP = 32
EMIN = {"f16": -15, "bf16": -117}
EMAX = {"f16": 8, "bf16": 120}


def exponents(x, fmt: str) -> np.ndarray:
    """Scale exponents [ceil(M / 32), K] of the matrix x [M, K]."""
    with np.errstate(invalid="ignore"):      # signalling NaN inputs stay NaN
        x = np.asarray(x, np.float64)
    M, K = x.shape
    a = np.zeros((-(-M // GROUP) * GROUP, K))
    a[:M] = np.where(np.isfinite(x), np.abs(x), 0.0)
    a = a.reshape(-1, GROUP, K).max(axis=1)
    f, p = np.frexp(np.where(a > 0, a, 2.0 ** -300))   # a = f * 2^p, 0.5 <= f < 1
    # 448 = 0.875 * 2^9
    e = np.where(f <= 0.875, p - 9, p - 8)
    return np.clip(e, EMIN[fmt], EMAX[fmt]).astype(np.int64)


def e4m3(y) -> np.ndarray:
    """y rounded to the nearest e4m3 value, ties to even (|y| <= 448; NaN stays)."""
    y = np.asarray(y, np.float64)
    _, E = np.frexp(y)
    q = np.ldexp(1.0, np.maximum(E - 1, -6) - 3)
    return np.rint(y / q) * q


def pack(x, fmt: str):
    """Codes (as e4m3 values, NaN for non-finite x) and exponents of x."""
    e = exponents(x, fmt)
    rows = np.repeat(e, GROUP, axis=0)[:np.shape(x)[0]]
    with np.errstate(invalid="ignore"):
        x = np.asarray(x, np.float64)
        c = e4m3(np.ldexp(np.where(np.isfinite(x), x, np.nan), -rows))
    top = (rows == EMAX[fmt]) & (np.abs(c) > 240.0)
    return np.where(top, np.copysign(240.0, c), c), e


def code_bytes(c) -> np.ndarray:
    """The e4m3 bytes of code values (NaN: 0x7F)."""
    c = np.asarray(c, np.float64)
    nan = np.isnan(c)
    a = np.abs(np.where(nan, 0.0, c))
    f, E = np.frexp(a)
    normal = a >= 2.0 ** -6
    b = np.where(normal, ((E - 1 + 7) << 3) + np.where(normal, (2.0 * f - 1.0) * 8.0, 0.0), a * 2.0 ** 9)
    b = b.astype(np.int64) | np.where(np.signbit(c), 0x80, 0)
    return np.where(nan, 0x7F, b).astype(np.uint8)


def byte_values(b) -> np.ndarray:
    """The value of every e4m3 byte."""
    b = np.asarray(b).astype(np.int64)
    m, E, s = b & 7, (b >> 3) & 15, np.where(b & 0x80, -1.0, 1.0)
    v = np.where(E > 0, np.ldexp(1.0 + m / 8.0, E - 7), m * 2.0 ** -9)
    return s * np.where((b & 0x7F) == 0x7F, np.nan, v)


def values(c, e) -> np.ndarray:
    """The matrix a checkpoint stands for."""
    return np.ldexp(np.asarray(c, np.float64), np.repeat(e, GROUP, axis=0)[:np.shape(c)[0]])
