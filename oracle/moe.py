"""A layer of experts on 4-bit weights in numpy float64 (TEST INFRASTRUCTURE ONLY).

    y_t = residual_t + sum_s weights_ts W_out[e] (act(W_gate[e] x_t) * (W_up[e] x_t)),  e = ids_ts
"""
import numpy as np

from . import groups


def route(logits, k, renormalise=True):
    z = np.asarray(logits, np.float64)
    ids = np.argsort(-np.where(np.isnan(z), -np.inf, z), axis=1, kind="stable")[:, :k]
    m = z.max(1, keepdims=True)
    e = np.where(np.isneginf(m), 0.0, np.exp(z - np.where(np.isneginf(m), 0.0, m)))
    chosen = np.take_along_axis(e, ids, 1)
    total = (chosen if renormalise else e).sum(1, keepdims=True)
    return ids, np.where(total > 0, chosen / np.where(total > 0, total, 1.0), 0.0)


def act(g, kind):
    if kind == "silu":
        return g / (1.0 + np.exp(-g))
    return 0.5 * g * (1.0 + np.tanh(np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)))


def layer(x, ids, weights, c_in, s_in, c_out, s_out, E, I, group, kind="silu", w_offset=0.5, residual=None,
          eps_in=0.0, eps_out=0.0, eps_mid=0.0, digits=0.0):
    """(y, bound): the bound takes sums of the first products to be off by eps_in of their terms' magnitudes, mid
    by eps_mid of itself, sums of the second by eps_out, and x and mid by `digits` of the largest element of a row.  c_in: codes [E 2 I, H], c_out [E H, I]."""
    x = np.asarray(x, np.float64)
    T, H = x.shape
    y = np.zeros((T, H)) if residual is None else np.array(residual, np.float64)
    bound = np.zeros((T, H))
    for e in range(E):
        hit = np.argwhere(ids == e)
        if not len(hit):
            continue
        rows = slice(e * 2 * I, (e + 1) * 2 * I)
        w1 = groups.values(c_in[rows], s_in[:, rows], group, w_offset)
        rows = slice(e * H, (e + 1) * H)
        w2 = groups.values(c_out[rows], s_out[:, rows], group, w_offset)
        for t, s in hit:
            both, mag = w1 @ x[t], np.abs(w1) @ (np.abs(x[t]) * eps_in + digits * np.abs(x[t]).max())
            g, u = both[:I], both[I:]
            mid = act(g, kind) * u
            off = 1.13 * mag[:I] * (np.abs(u) + mag[I:]) + np.abs(act(g, kind)) * mag[I:] + eps_mid * np.abs(mid)
            off = off + digits * np.abs(mid).max()
            y[t] += weights[t, s] * (w2 @ mid)
            bound[t] += abs(weights[t, s]) * (np.abs(w2) @ off * (1 + eps_out) + eps_out * (np.abs(w2) @ np.abs(mid)))
    return y, bound
