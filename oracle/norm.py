"""Root-mean-square norm with an 8-bit output in numpy float64 (TEST INFRASTRUCTURE ONLY).

    h = x + residual,  rstd = 1/sqrt(mean h^2 + eps),  y = h rstd w
    scale = max |y| / 127 over a row,  q = floor(y / scale + 1/2)

and the gradients of y with the codes' steps passed straight through.
"""
import numpy as np


def forward(x, w, eps, residual=None):
    """(h, y, rstd) of rows [M, K] in float64."""
    h = np.asarray(x, np.float64)
    if residual is not None:
        h = h + np.asarray(residual, np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h, h * rstd[:, None] * np.asarray(w, np.float64), rstd


def eight_bits(y):
    """(q before its floor, scale): the value y / scale, whose floor(. + 1/2) is the code."""
    scale = np.abs(y).max(1) / 127.0
    return y / np.where(scale > 0, scale, 1.0)[:, None], scale


def backward(grad_y, h, w, rstd, grad_h=None):
    """(grad_x, grad_w, magnitude of the terms of grad_x, of grad_w)."""
    gy, h, w = (np.asarray(a, np.float64) for a in (grad_y, h, w))
    rstd = np.asarray(rstd, np.float64)[:, None]
    g, n = gy * w, h * rstd
    gx = rstd * (g - n * (g * n).mean(1, keepdims=True))
    mag = rstd * (np.abs(g) + np.abs(n) * np.abs(g * n).mean(1, keepdims=True))
    if grad_h is not None:
        gx = gx + np.asarray(grad_h, np.float64)
        mag = mag + np.abs(np.asarray(grad_h, np.float64))
    return gx, (gy * n).sum(0), mag, np.abs(gy * n).sum(0)


def exact_codes(h, w):
    """floor(127 h w / a + 1/2), a = max |h w| of a row, of binary32 values h [M, K] and w [K]: decided
    exactly, by 254 h w >= (2 q - 1) a.  (A product of two binary32 numbers fits float64; with a number of
    eight bits more it fits the 64 bits of a long double.)  Rows of zeros: codes 0."""
    hw = np.asarray(h, np.float64) * np.asarray(w, np.float64)
    a = np.abs(hw).max(1, keepdims=True)
    safe = np.where(a > 0, a, 1.0)
    q = np.floor(127.0 * (hw / safe) + 0.5)
    wide = np.longdouble
    assert np.finfo(wide).nmant >= 63
    x, a = wide(254) * hw.astype(wide), safe.astype(wide)
    q -= x < (2 * q - 1).astype(wide) * a
    q += x >= (2 * q + 1).astype(wide) * a
    return q.astype(np.int64)
