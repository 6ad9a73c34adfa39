"""float64 oracle of the 8-bit paged cache and of the head norms, written from their definitions (numpy).

A row x is held as e4m3 codes c and a byte e, x_i ~ c_i * 2^(e - 127): e is the smallest in [1, 254] with
max |x_i| <= 448 * 2^(e - 127), the codes are the nearest (ties to even).
"""
from __future__ import annotations

import numpy as np


def _table():
    """The number that each of the 256 codes stands for: sign, 4 bits of exponent (bias 7), 3 of fraction; all ones: NaN."""
    t = np.empty(256)
    for c in range(256):
        sign, e, f = -1.0 if c & 128 else 1.0, c >> 3 & 15, c & 7
        t[c] = np.nan if c & 127 == 127 else sign * (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
    return t


CODES = _table()


def power(e):
    """What scale bytes stand for."""
    e = np.asarray(e)
    return np.where(e == 255, np.nan, np.exp2(e.astype(np.float64) - 127))


def values(codes, scales):
    """What codes [.., dim] and scale bytes [..] stand for."""
    return CODES[codes] * power(scales)[..., None]


def scale_byte(x):
    """Scale bytes of rows x [.., dim]."""
    most = np.abs(x).max(-1)
    out = np.full(most.shape, 255, np.int64)
    for i in np.ndindex(most.shape):
        if np.isfinite(most[i]):
            e = 1
            while e < 254 and most[i] > 448 * 2.0 ** (e - 127):
                e += 1
            out[i] = e
    return out


def nearest(x):
    """The e4m3 number nearest to x (|x| <= 448), ties to an even code."""
    a = np.abs(x)
    step = np.exp2(np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.sign(x) * np.round(a / step) * step                      # (np.round: halves to even)


def hold(x):
    """(what rows x [.., dim] are held as, their scale bytes)."""
    e = scale_byte(x)
    s = power(e)[..., None]
    return np.where(np.isnan(s), np.nan, nearest(np.where(np.isnan(s), 0, x) / np.where(np.isnan(s), 1, s)) * s), e


def norm(x, weight, eps):
    """x [.., heads, dim]; weight [dim] or [heads, dim], or None."""
    if weight is None:
        return x
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
