"""E4M3 with a power-of-two scale for every block of 128, and the expert FFN on it, in float64 numpy from the definitions."""
from __future__ import annotations

import numpy as np

BLOCK = 128


def stride(C):
    return (C // BLOCK + 3) // 4 * 4


def scale_bytes(top):
    """E8M0 of the smallest power of two, from 2^-126, that leaves at most 448; 255 where top is not finite."""
    top = np.asarray(top, dtype=np.float64)
    with np.errstate(all="ignore"):
        frac, exp = np.frexp(top / 448)          # top / 448 = frac 2^exp with frac in [0.5, 1)
        k = np.where(frac == 0.5, exp - 1, exp)
    b = np.where(top > 0, np.maximum(k, -126) + 127, 1)
    return np.where(np.isfinite(top), b, 255).astype(np.uint8)


def scale_value(b):
    return np.where(b == 255, np.nan, np.exp2(b.astype(np.float64) - 127))


def to_e4m3(y):
    """Nearest of E4M3's values (at most 448 in magnitude on entry), ties to even."""
    with np.errstate(all="ignore"):
        step = np.exp2(np.floor(np.log2(np.maximum(abs(y), 2.0 ** -6))) - 3)
    return np.rint(y / step) * step


def _all_values():
    """Every code's value: sign, four bits of exponent (bias 7), three of fraction; 0x7f and 0xff are NaN."""
    c = np.arange(256)
    exp, frac = (c >> 3) & 15, c & 7
    v = np.where(exp == 0, frac * 2.0 ** -9, (8 + frac) * np.exp2(exp - 10.0))
    return np.where((c & 127) == 127, np.nan, np.where(c & 128, -v, v))


VALUES = _all_values()


def codes_of(y):
    """Codes of values that E4M3 has; NaN as 0x7f."""
    order = np.argsort(VALUES[:127])
    mag = np.searchsorted(VALUES[:127][order], np.nan_to_num(abs(y)))
    c = order[mag] | np.where(np.signbit(y), 128, 0)
    return np.where(np.isnan(y), 0x7f, c).astype(np.uint8)


def quantize_rows(x):
    """Codes [R, C] and scales [R, C / 128] of x, as bytes."""
    R, C = x.shape
    v = np.asarray(x, dtype=np.float64).reshape(R, -1, BLOCK)
    b = scale_bytes(abs(v).max(2)) if v.size else np.zeros(v.shape[:2], dtype=np.uint8)
    return codes_of(to_e4m3(v / scale_value(b)[:, :, None])).reshape(R, C), b


def quantize_square(w):
    """Codes [N, K] and scales [N / 128, K / 128] of w."""
    N, K = w.shape
    v = np.asarray(w, dtype=np.float64).reshape(N // BLOCK, BLOCK, K // BLOCK, BLOCK)
    b = scale_bytes(abs(v).max((1, 3)))
    return codes_of(to_e4m3(v / scale_value(b)[:, None, :, None])).reshape(N, K), b


def rows_value(codes, b):
    C = codes.shape[1]
    return VALUES[codes] * np.repeat(scale_value(b[:, :C // BLOCK]), BLOCK, axis=1)


def square_value(codes, b):
    K = codes.shape[1]
    return VALUES[codes] * np.repeat(np.repeat(scale_value(b[:, :K // BLOCK]), BLOCK, axis=0), BLOCK, axis=1)


def quantized_range(v, err):
    """Smallest and largest value that quantising rows gives for values within err of v."""
    R, C = v.shape
    v, err = v.reshape(R, -1, BLOCK), err.reshape(R, -1, BLOCK)
    lo, hi = (abs(v) - err).max(2), (abs(v) + err).max(2)
    got = []
    for top in (lo, hi):
        s = scale_value(scale_bytes(np.maximum(top, 0)))[:, :, None]
        got += [np.clip(to_e4m3(np.clip((v + e) / s, -448, 448)), -448, 448) * s for e in (-err, err)]
    return np.minimum.reduce(got).reshape(R, C), np.maximum.reduce(got).reshape(R, C)


def sigmoid(g):
    return np.where(g >= 0, 1 / (1 + np.exp(-abs(g))), np.exp(-abs(g)) / (1 + np.exp(-abs(g))))
