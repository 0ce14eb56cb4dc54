"""The 4-bit pool in float64: its format, its quantisation and what its bytes stand for.

Written from the definition (include/louiskv.h): blocks of 32 channels, the scale
2^E with the smallest E in [-125, 125] for which max|x| <= 7 * 2^E (125 if there is
none), every element the nearest level times the scale, ties to the even level index.
"""
from __future__ import annotations

import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32
MIN_EXP, MAX_EXP = -125, 125


def block_exponent(top: float) -> int:
    """The smallest E in [-125, 125] with top <= 7 * 2^E, or 125."""
    e = MIN_EXP
    if top > 0.0:
        e = max(e, math.frexp(top)[1] - 4)
        while top > 7.0 * 2.0 ** e:
            e += 1
    return min(e, MAX_EXP)


def quantise(rows: np.ndarray):
    """(levels [n][128] as 4-bit codes, scale bytes [n][4]) of float64 rows [n][128]."""
    n = rows.shape[0]
    codes = np.zeros((n, 128), dtype=np.uint8)
    scales = np.zeros((n, 4), dtype=np.uint8)
    for i in range(n):
        for b in range(4):
            x = rows[i, BLOCK * b:BLOCK * (b + 1)]
            if not np.all(np.isfinite(x)):
                scales[i, b] = 255
                continue
            e = block_exponent(float(np.abs(x).max()))
            scales[i, b] = e + 127
            gap = np.abs(np.abs(x)[:, None] / 2.0 ** e - LEVELS)     # a power of two: exact
            best = gap.min(axis=1, keepdims=True)
            near = gap == best
            first = near.argmax(axis=1)
            tied = near.sum(axis=1) == 2                             # two levels equally near: the even one
            idx = np.where(tied & (first % 2 == 1), first + 1, first)
            codes[i, BLOCK * b:BLOCK * (b + 1)] = idx + 8 * np.signbit(x)
    return codes, scales


def pack_bytes(k_codes, k_scales, v_codes, v_scales):
    """Pool bytes of rows: (codes [n][128], scales [n][8])."""
    def nib(c):
        return c[:, 0::2] | (c[:, 1::2] << 4)
    return np.concatenate([nib(k_codes), nib(v_codes)], axis=1), np.concatenate([k_scales, v_scales], axis=1)


def values(codes: np.ndarray, scales: np.ndarray):
    """(keys [n][128], values [n][128]) in float64 that pool bytes [n][128], [n][8] stand for."""
    n = codes.shape[0]
    nib = np.empty((n, 256), dtype=np.int64)
    nib[:, 0::2] = codes & 15
    nib[:, 1::2] = codes >> 4
    x = np.where(nib >= 8, -1.0, 1.0) * LEVELS[nib & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    x = (x.reshape(n, 8, BLOCK) * s[:, :, None]).reshape(n, 256)
    return x[:, :128], x[:, 128:]
