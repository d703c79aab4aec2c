"""Weights with a scale per group in numpy float64 (TEST INFRASTRUCTURE ONLY).

The uniform quantiser of the paper (Eq. 2, midpoints upwards) at 4 bits on the range
[-a, a] of each group of consecutive weights of a row, a their largest magnitude.
"""
import numpy as np


def quantize(w, group):
    """(signed codes c = q - 8, q in 0..15, scales [groups, N] = a / 15) of [N, K]."""
    w = np.asarray(w, np.float64)
    N, K = w.shape
    groups = -(-K // group)
    codes = np.empty((N, K), np.int64)
    scales = np.empty((groups, N))
    for g in range(groups):
        part = w[:, g * group:(g + 1) * group]
        a = np.abs(part).max(1, keepdims=True)
        safe = np.where(a > 0, a, 1.0)
        # q = floor((w + a) 15 / (2 a) + 1/2) as one quotient of numbers of 28 bits or so: a
        # quotient that is no whole number is further from one than its rounding
        q = np.floor((15.0 * part + 16.0 * safe) / (2.0 * safe))
        # (the border at w = 0, where small negative weights vanish beside a)
        q = np.where((part < 0) & (q == 8), 7, q)
        q = np.where(a > 0, np.clip(q, 0, 15), 8)
        codes[:, g * group:(g + 1) * group] = q.astype(np.int64) - 8
        scales[g] = a[:, 0] / 15.0
    return codes, scales


def per_weight(scales, K, group):
    """scales [groups, N] -> [N, K]."""
    return np.repeat(np.asarray(scales, np.float64).T, group, axis=1)[:, :K]


def values(codes, scales, group, w_offset=0.5):
    """What codes stand for: scale (2 c + 1), or scale c."""
    c = np.asarray(codes, np.float64)
    v = 2.0 * c + 1.0 if w_offset == 0.5 else c
    return v * per_weight(scales, c.shape[1], group)


def linear(x, codes, scales, group, bias=None, row_scale=None, w_offset=0.5):
    """(Y, sum_k |terms|) of Y = row_scale X w^T + bias."""
    x = np.asarray(x, np.float64)
    if row_scale is not None:
        x = x * np.asarray(row_scale, np.float64)[:, None]
    w = values(codes, scales, group, w_offset)
    y = x @ w.T
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return y, np.abs(x) @ np.abs(w).T
