"""Root-mean-square norm, e4m3 rounding and the epilogue of a product, in fp64 (extensions: Section 3.2 fixes neither
normalisation nor feed-forward)."""
from __future__ import annotations

import math

import numpy as np


def _e4m3_table():
    """Values of the bit patterns 0 .. 0x7e (sign, 4 exponent bits with bias 7, 3 mantissa bits; 0x7f is NaN)."""
    out = []
    for b in range(0x7f):
        e, m = b >> 3, b & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


E4M3 = _e4m3_table()


def to_e4m3(a):
    """Bit patterns (uint8) of the nearest e4m3 values, ties to the even pattern, magnitudes beyond 448 to 448."""
    a = np.asarray(a, dtype=np.float64)
    mag = np.minimum(np.abs(a), E4M3[-1])
    hi = np.clip(np.searchsorted(E4M3, mag), 0, len(E4M3) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3[hi] - mag, mag - E4M3[lo]
    pick = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return (pick | np.where(np.signbit(a), 0x80, 0)).astype(np.uint8)


def from_e4m3(bits):
    bits = np.asarray(bits, dtype=np.uint8)
    mag = np.append(E4M3, np.nan)[bits & 0x7f]
    return np.where(bits & 0x80, -mag, mag)


def rms_norm(s, gamma, eps):
    s = np.asarray(s, dtype=np.float64)
    return s / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps) * np.asarray(gamma, dtype=np.float64)


def row_scales(n):
    return np.maximum(np.abs(n).max(axis=1), 2.0 ** -100) / 448.0


def _logistic(z):
    return np.where(z >= 0, 1.0, np.exp(-np.abs(z))) / (1.0 + np.exp(-np.abs(z)))


def activation(v, act):
    v = np.asarray(v, dtype=np.float64)
    if act == "relu":
        return np.maximum(v, 0.0)
    if act == "gelu":
        return v * 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-v / math.sqrt(2.0))
    if act == "gelu_tanh":
        # (1 + tanh z) / 2 = 1 / (1 + e^-2z), which keeps its digits where tanh z is next to -1
        return v * _logistic(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))
    if act == "silu":
        return v * _logistic(v)
    return v
