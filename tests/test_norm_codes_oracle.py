"""Oracle pin of the norm's 8-bit codes: against whole fractions, at borders and beside them."""
from fractions import Fraction

import numpy as np

from oracle import norm


def test_codes_are_exact():
    rng = np.random.default_rng(11)
    h = rng.normal(size=(6, 60)).astype(np.float32)
    w = (1 + 0.1 * rng.normal(size=60)).astype(np.float32)
    # rows of whole and half numbers below 127 times an odd number: borders in many places
    h[:4] = rng.integers(-380, 381, (4, 60)) * 0.5
    h[:4, 0] = 127 * 3, -127 * 5, 127 * 7, 127
    w[:] = np.where(rng.random(60) < 0.7, 1.0, w)
    w[0] = 1.0
    h[5] = 0
    q = norm.exact_codes(h, w)
    met = 0
    for m in range(6):
        hw = [Fraction(float(a)) * Fraction(float(b)) for a, b in zip(h[m], w)]
        a = max(map(abs, hw)) or Fraction(1)
        for k in range(60):
            v = 127 * hw[k] / a + Fraction(1, 2)
            met += v.denominator == 1
            assert q[m, k] == v.numerator // v.denominator
    assert met >= 10
