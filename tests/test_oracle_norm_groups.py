"""Oracle pins of the norm, of its gradients and of group-wise weights: closed forms and
central differences."""
from fractions import Fraction

import numpy as np

from oracle import groups, norm


def test_norm_closed_forms():
    x = np.array([[3.0, 4.0], [0.0, 0.0], [-2.0, 2.0]])
    h, y, rstd = norm.forward(x, np.array([1.0, 2.0]), 0.5, residual=np.array([[0.0, 0.0]] * 3))
    assert np.allclose(rstd, [1 / np.sqrt(13.0), np.sqrt(2.0), 1 / np.sqrt(4.5)])
    assert np.allclose(y[0], [3 / np.sqrt(13.0), 8 / np.sqrt(13.0)])
    v, scale = norm.eight_bits(np.array([[127.0, -63.5, 0.4], [0.0, 0.0, 0.0]]))
    assert np.allclose(scale, [1.0, 0.0]) and np.array_equal(np.floor(v + 0.5)[0], [127, -63, 0])


def test_norm_gradients_are_those_of_differences():
    rng = np.random.default_rng(5)
    x, gy, gh = rng.normal(size=(3, 3, 7))
    w = rng.normal(size=7)
    eps, d = 1e-2, 1e-6

    def loss(x, w):
        h, y, _ = norm.forward(x, w, eps)
        return (gy * y).sum() + (gh * h).sum()

    h, _, rstd = norm.forward(x, w, eps)
    gx, gw, _, _ = norm.backward(gy, h, w, rstd, gh)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = d
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * d) - gx[i]) < 1e-7
    for k in range(7):
        e = np.zeros_like(w)
        e[k] = d
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * d) - gw[k]) < 1e-7


def test_group_codes_are_exact():
    rng = np.random.default_rng(6)
    # small integers: every border is met
    w = rng.integers(-30, 31, (8, 100)).astype(np.float32)
    w[0, 64:] = 0.0
    w[1, 5] = -1e-30
    codes, scales = groups.quantize(w, 64)
    for n in range(8):
        for k in range(100):
            part = w[n, k // 64 * 64:(k // 64 + 1) * 64]
            a = Fraction(float(np.abs(part).max()))
            assert scales[k // 64, n] == float(a) / 15.0
            if a == 0:
                assert codes[n, k] == 0
                continue
            q = (15 * Fraction(float(w[n, k])) + 16 * a) / (2 * a)
            assert codes[n, k] == min(q.numerator // q.denominator, 15) - 8


def test_group_values_and_product():
    codes = np.array([[-8, 7, 0, -1, 3]])
    scales = np.array([[2.0], [0.5]])
    assert np.array_equal(groups.values(codes, scales, 3), [[-30.0, 30.0, 2.0, -0.5, 3.5]])
    assert np.array_equal(groups.values(codes, scales, 3, 0.0), [[-16.0, 14.0, 0.0, -0.5, 1.5]])
    y, mag = groups.linear(np.array([[1, 1, 1, 2, 0]]), codes, scales, 3, bias=np.array([10.0]),
                           row_scale=np.array([0.5]))
    assert y[0, 0] == 0.5 * (2.0 - 1.0) + 10.0 and mag[0, 0] == 0.5 * 63.0
