"""Plain float64 NumPy oracle of the 8-bit path (test infrastructure only, as the rest of this package): values kept as
e4m3 codes with one power of two for each group of 128, the product of two such operands, the weight gradient from a
checkpoint, and the norms with their backward pass. It shares no code with the HIP path or with ``perf/operators.py``.

Definitions
-----------
* e4m3 (OCP 8-bit floating point, E4M3): sign, 4 exponent bits with bias 7, 3 mantissa bits; 0x7F and 0xFF are NaN, there
  is no infinity, the largest value is 448, subnormals are multiples of 2^-9.
* A group's exponent e is the smallest integer >= -126 with (largest finite magnitude) / 2^e <= 448; its codes are
  value / 2^e rounded to nearest, ties to even; NaN and infinities become NaN.
* Layer norm and RMS norm as in ``norm``; the backward is their derivative (checked against differences in the tests).
"""
from __future__ import annotations

import numpy as np


def code_values() -> np.ndarray:
    """The 256 values of the codes (NaN for 0x7F, 0xFF)."""
    out = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, c >> 3 & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = np.nan if e == 15 and m == 7 else -v if s else v
    return out


VALUES = code_values()


def encode(v: np.ndarray) -> np.ndarray:
    """Codes of float64 values of magnitude <= 448 (or NaN, infinite): nearest, ties to the even code."""
    mag = VALUES[:127]                                # 0 .. 448, ascending
    a = np.abs(v)
    bad = ~np.isfinite(v)
    a = np.where(bad, 0.0, a)
    hi = np.clip(np.searchsorted(mag, a, side="left"), 1, 126)
    lo = hi - 1
    dl, dh = a - mag[lo], mag[hi] - a
    c = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    c = np.where(bad, 0x7F, c)
    return (c | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def group_exponent(amax: np.ndarray) -> np.ndarray:
    """Smallest integer e >= -126 with amax / 2^e <= 448."""
    amax = np.asarray(amax, dtype=np.float64)
    e = np.full(amax.shape, -126)
    pos = amax > 0
    g = np.ceil(np.log2(amax[pos] / 448.0)).astype(int)
    g += amax[pos] > 448.0 * 2.0 ** g                   # log2's rounding, either way
    g -= amax[pos] <= 448.0 * 2.0 ** (g - 1)
    e[pos] = np.maximum(g, -126)
    return e


def _magnitudes(x):
    return np.where(np.isfinite(x), np.abs(x), 0.0)


def quant_rows(x: np.ndarray):
    """float64 [M, K] -> codes uint8 [M, K up to 128], exponent bytes uint8 [M, K/128 up to 4]."""
    m, k = x.shape
    g = -(-k // 128)
    xp = np.zeros((m, g * 128))
    xp[:, :k] = x
    xg = xp.reshape(m, g, 128)
    e = group_exponent(_magnitudes(xg).max(axis=2)) if m else np.zeros((0, g), int)
    codes = encode(xg / 2.0 ** e[:, :, None]).reshape(m, g * 128)
    exps = np.zeros((m, -(-g // 4) * 4), dtype=np.uint8)
    exps[:, :g] = e + 127
    return codes, exps


def values_rows(codes, exps, k):
    m, kp = codes.shape
    e = exps[:, : kp // 128].astype(int) - 127
    return (VALUES[codes].reshape(m, kp // 128, 128) * 2.0 ** e[:, :, None]).reshape(m, kp)[:, :k]


def quant_weight(w: np.ndarray):
    """float64 [N, K] -> row-major codes uint8 [N, K] and exponents int [N/128 up, K/128 up], one for each 128 x 128 block."""
    n, k = w.shape
    codes = np.empty((n, k), np.uint8)
    e = np.empty((-(-n // 128), -(-k // 128)), int)
    for i in range(e.shape[0]):
        for j in range(e.shape[1]):
            b = w[128 * i:128 * i + 128, 128 * j:128 * j + 128]
            e[i, j] = group_exponent(_magnitudes(b).max())
            codes[128 * i:128 * i + 128, 128 * j:128 * j + 128] = encode(b / 2.0 ** e[i, j])
    return codes, e


def values_weight(codes, e):
    n, k = codes.shape
    return VALUES[codes] * 2.0 ** np.repeat(np.repeat(e, 128, 0)[:n], 128, 1)[:, :k]


def tiles(codes):
    """Row-major codes as the library's tiles, one code at a time from the layout's definition."""
    n, k = codes.shape
    out = np.zeros((-(-n // 16), -(-k // 128), 2, 4, 16, 16), np.uint8)
    r, c = np.meshgrid(np.arange(n), np.arange(k), indexing="ij")
    out[r // 16, c // 128, c % 32 // 16, c % 128 // 32, r % 16, c % 16] = codes
    return out


def exponent_rows(e):
    """Block exponents as the library's bytes, rows padded with zeros to words."""
    out = np.zeros((e.shape[0], -(-e.shape[1] // 4) * 4), np.uint8)
    out[:, : e.shape[1]] = e + 127
    return out


def norm(x, gamma, beta, eps, rms):
    """(y, mean, rstd) of the rows of float64 x; mean zero for the RMS norm."""
    mean = np.zeros(x.shape[0]) if rms else x.mean(axis=1)
    d = x - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).mean(axis=1) + eps)
    y = d * rstd[:, None]
    y = y if gamma is None else y * gamma
    return (y if beta is None else y + beta), mean, rstd


def norm_bwd(dy, x, gamma, mean, rstd, rms):
    """(dx, dgamma, dbeta) at the given statistics."""
    xh = (x - mean[:, None]) * rstd[:, None]
    t = dy if gamma is None else dy * gamma
    dx = t - xh * (t * xh).mean(axis=1, keepdims=True)
    if not rms:
        dx = dx - t.mean(axis=1, keepdims=True)
    return dx * rstd[:, None], (dy * xh).sum(axis=0), dy.sum(axis=0)
