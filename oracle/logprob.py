"""Log probabilities, entropy and alternatives of rows of logits in numpy float64 (TEST INFRASTRUCTURE ONLY)."""
import numpy as np


def forward(x, targets, scale=1.0):
    """dict of lse, logp, entropy, and of what tolerances are made of: log s, the spread z_t - m, the first
    and second moments of m - z.  Rows of nothing but -infinity as the interface has them."""
    z = np.asarray(x, np.float64) * scale
    m = z.max(1, keepdims=True)
    none = np.isneginf(m[:, 0])
    with np.errstate(invalid="ignore", divide="ignore"):
        d = np.where(none[:, None], -np.inf, z - m)
        e = np.exp(d)
        s = e.sum(1)
        lse = np.where(none, -np.inf, m[:, 0] + np.log(s))
        p = np.where(none[:, None], 0.0, e / s[:, None])
        lp = np.where(none[:, None], -np.inf, d - np.log(s)[:, None])
        entropy = -np.where(p > 0, p * lp, 0.0).sum(1)
        dd = np.where(p > 0, -d, 0.0)
    rows = np.arange(len(z))
    t = np.asarray(targets)
    safe = np.clip(t, 0, z.shape[1] - 1)
    logp = np.where(t < 0, 0.0, np.where(t >= z.shape[1], np.nan, lp[rows, safe]))
    return dict(lse=lse, logp=logp, entropy=entropy, lp=lp, p=p, log_s=np.where(none, 0.0, np.log(np.maximum(s, 1.0))),
                first=(p * dd).sum(1), second=(p * dd * dd).sum(1))


def largest(x, k):
    """Indices of the k largest of each row, equal ones by index, NaN last."""
    v = np.where(np.isnan(x), -np.inf, x).astype(np.float64)
    return np.stack([np.lexsort((np.arange(len(r)), np.isnan(o), -r))[:k] for r, o in zip(v, x)])


def backward(x, targets, lse, g, entropy, ge, scale=1.0):
    """(grad, magnitude of the terms, |log p|)."""
    z = np.asarray(x, np.float64) * scale
    g, ge, h = (np.zeros(len(z)) if v is None else np.asarray(v, np.float64) for v in (g, ge, entropy))
    t = np.asarray(targets) if targets is not None else np.full(len(z), -1)
    g = np.where(t < 0, 0.0, g)
    lse = np.asarray(lse, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        l = z - lse[:, None]
        p = np.exp(l)
        plh = np.where(p > 0, p * (l + h[:, None]), 0.0)
    one = (np.arange(z.shape[1]) == t[:, None]).astype(np.float64)
    grad = scale * (g[:, None] * (one - p) - ge[:, None] * plh)
    mag = scale * (np.abs(g)[:, None] * p + np.abs(ge)[:, None] * (np.abs(plh) + p))
    zero = ((g == 0) & (ge == 0)) | np.isneginf(lse)
    grad[zero] = 0
    mag[zero] = 0
    return grad, mag, scale * np.abs(g)[:, None] * one, np.where(p > 0, np.abs(l), 0.0)
