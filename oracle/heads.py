"""Norms of heads with the position rotation in numpy float64 (TEST INFRASTRUCTURE ONLY).

    n = x rstd w,  rstd = 1/sqrt(mean x^2 + eps)   of heads [tokens, heads, D]
    pairs (n1, n2) of the first R elements turned by positions[axis[i]] f[i]
"""
import numpy as np


def angles(pos, freq, axis=None):
    """[tokens, R/2] in float64; pos [axes, tokens]."""
    pos, freq = np.atleast_2d(np.asarray(pos)).astype(np.float64), np.asarray(freq, np.float64)
    axis = np.zeros(len(freq), int) if axis is None else np.asarray(axis, int)
    return pos[axis].T * freq


def turn(v, a, interleaved=False):
    """Heads turned by the angles a (as a rotation matrix applied pair by pair)."""
    v, out = np.asarray(v, np.float64), np.array(v, np.float64)
    R = 2 * a.shape[1]
    for i in range(R // 2):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        c, s = np.cos(a[:, i])[:, None], np.sin(a[:, i])[:, None]
        out[..., p] = c * v[..., p] - s * v[..., q]
        out[..., q] = s * v[..., p] + c * v[..., q]
    return out


def partner(v, a, interleaved=False):
    """|element| + |its partner| (the magnitude of a turned pair's terms)."""
    v = np.abs(np.asarray(v, np.float64))
    out, R = v.copy(), 2 * a.shape[1]
    for i in range(R // 2):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        out[..., p] = out[..., q] = v[..., p] + v[..., q]
    return out


def normed(x, w, eps):
    """(n, rstd); rstd 0 for a head of zeros with eps = 0."""
    x = np.asarray(x, np.float64)
    mean = (x * x).mean(-1, keepdims=True) + eps
    with np.errstate(divide="ignore"):
        r = np.where(mean == 0, 0.0, 1.0 / np.sqrt(mean))
    return x * r * (1.0 if w is None else np.asarray(w, np.float64)), r


def forward(x, w, a, eps, interleaved=False, norm=True):
    return turn(normed(x, w, eps)[0] if norm else x, a, interleaved)


def backward(gy, x, w, a, eps, interleaved=False, norm=True):
    """(grad_x, grad_w, magnitudes of the terms of each)."""
    g, G = turn(gy, -a, interleaved), partner(gy, a, interleaved)
    if not norm:
        return g, None, G, None
    w = np.ones(g.shape[-1]) if w is None else np.asarray(w, np.float64)
    n, r = normed(x, None, eps)
    gx = r * (g * w - n * (g * w * n).mean(-1, keepdims=True))
    mag = r * (G * np.abs(w) + np.abs(n) * (G * np.abs(w * n)).mean(-1, keepdims=True))
    return gx, (g * n).sum((0, 1)), mag, (G * np.abs(n)).sum((0, 1))
