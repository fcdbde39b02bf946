"""CPU fp64 oracle of the append's norms and rotation and of rows held in 8 bits
(test infrastructure only).

A head row x becomes n = x / sqrt(mean(x^2) + eps) * w, then pair i of its first
rotary dims (a, b) becomes (a cos - b sin, a sin + b cos). A row in 8 bits is a
scale 2^e, e the least integer in -100 .. 120 with max |x| <= 448 * 2^e, and per
value the e4m3 number (sign, four exponent bits of bias 7, three mantissa bits,
no infinities) nearest to x / 2^e, ties to the even code."""

from __future__ import annotations

import numpy as np

MIN_EXP, MAX_EXP = -100, 120
NAN_CODE = 0x7F


def _e4m3_values() -> np.ndarray:
    code = np.arange(128)
    exp, mant = code >> 3, code & 7
    v = np.where(exp > 0, (1 + mant / 8) * 2.0 ** (exp - 7.0), mant * 2.0 ** -9)
    v[NAN_CODE] = np.nan
    return v


E4M3 = np.concatenate([_e4m3_values(), -_e4m3_values()])   # the value of every code


def rotate(x, positions, table, adjacent: bool):
    """x [n][heads][D] float64; positions [n][pairs]: each pair's row of the table [rows][2 pairs]."""
    half = table.shape[1] // 2
    y = x.copy()
    pair = np.arange(half)
    c = table[positions, pair][:, None].astype(np.float64)
    s = table[positions, half + pair][:, None].astype(np.float64)
    a, b = (2 * pair, 2 * pair + 1) if adjacent else (pair, pair + half)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def norm(x, weight, eps):
    """x [..., D] float64, each row over its own root mean square, times the weights."""
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight


def row_exponents(x):
    """The scale exponent of each row [..., D] (over its finite values)."""
    amax = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    m, e = np.frexp(amax)                        # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    e = np.where(amax == 0, MIN_EXP, np.where(m <= 0.875, e - 9, e - 8))
    return np.clip(e, MIN_EXP, MAX_EXP)


def encode(x):
    """e4m3 codes (uint8) and scale bytes (uint8) of rows [..., D]."""
    e = row_exponents(x)
    z = x / 2.0 ** e[..., None].astype(np.float64)
    mag = np.abs(np.where(np.isfinite(z), z, 0.0))
    # spacing 2^(b - 3) in [2^b, 2^(b + 1)), 2^-9 below 2^-6; the number of steps is rounded
    # half to even, and from the 8th on counts through the binades as the code does
    b = np.where(mag > 0, np.maximum(np.frexp(mag)[1] - 1, -6), -6)
    code = np.rint(np.ldexp(mag, 3 - b)).astype(np.int64) + 8 * (b + 6)
    code = np.where(np.signbit(z), code + 128, code)
    code = np.where(np.isfinite(x), code, NAN_CODE)
    return code.astype(np.uint8), (e + 127).astype(np.uint8)


def decode_rows(codes, scale_bytes):
    """The float64 values of codes [..., D] with scale bytes [...]."""
    return E4M3[codes] * 2.0 ** (scale_bytes.astype(np.float64) - 127.0)[..., None]
