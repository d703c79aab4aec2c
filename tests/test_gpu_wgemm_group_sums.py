"""GPU: what is exact and what is rounded in a product with 8-bit rows and long groups.

Sums of a piece of up to 128 codes (128, 64 or 32, which no group's end cuts) are exact in int32, and in binary32; each enters the
total times its group's scale with one rounding.  Sixteen additions more join the totals of warps and blocks, and row
scale and bias take two: (ceil(K / piece) + 18) 2^-24 of the magnitudes added."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import groups as G
from gpu_util import T, N

U = 2.0 ** -24


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


@pytest.mark.parametrize("form", [0, 1, 2])
@pytest.mark.parametrize("size", [(2, 40, 1 << 16, 1 << 16), (5, 33, 70016, 1 << 15), (1, 64, 65552, 4096), (20, 130, 16384, 1 << 20),
                                  (64, 128, 8192, 8192), (3, 20, 4112, 96), (9, 50, 2064, 64)])
def test_long_groups(dsq, size, form):
    M, n, k, group = size
    rng = np.random.default_rng(k + M)
    codes = rng.integers(-8, 8, (n, k)).astype(np.int8)
    scales = rng.uniform(0.5, 1.5, (-(-k // group), n)).astype(np.float32)
    x = rng.integers(-128, 128, (M, k)).astype(np.int8)
    rs = rng.uniform(0.01, 0.02, M).astype(np.float32)
    bias = rng.normal(size=n).astype(np.float32)
    whole = min(group, k)
    piece = 128 if group >= k or group % 128 == 0 else 64 if group % 64 == 0 else 32
    dsq.dsq_set_wgemm_group_form(form)
    try:
        for off in (0.5, 0.0):
            Y = dsq.dsq_wgemm_group(T(x), dsq.dsq_pack_codes(T(codes), 4), M, n, k, 4, group, T(scales), bias=T(bias), row_scale=T(rs),
                                    w_offset=off)
            ref, mag = G.linear(x, codes, scales, whole, bias, rs, off)
            # (magnitudes of whole pieces, which is what the totals add)
            w = G.values(codes, scales, whole, off)
            xs = x * rs[:, None].astype(np.float64)
            mag = sum(np.abs(xs[:, i:i + piece] @ w[:, i:i + piece].T) for i in range(0, k, piece))
            tol = 1.01 * ((-(-k // piece) + 18) * U * mag + 2 * U * np.abs(bias))
            assert np.all(np.abs(N(Y).astype(np.float64) - ref) <= tol + U * np.abs(ref))
    finally:
        dsq.dsq_set_wgemm_group_form(0)


def test_pieces_of_128_are_exact(dsq):
    """Scales that are powers of two, one piece of 128 with the largest products, the others 0: exact."""
    k, n = 2048, 64
    for M in (1, 7, 40):
        for c, v in ((7, 127), (-8, -128), (-8, 127), (7, -128)):
            codes = np.zeros((n, k), np.int8)
            x = np.zeros((M, k), np.int8)
            codes[:, 640:768] = c
            x[:, 640:768] = v
            x[:, 650] = 1
            Y = dsq.dsq_wgemm_group(T(x), dsq.dsq_pack_codes(T(codes), 4), M, n, k, 4, k, T(np.ones((1, n), np.float32)),
                                    row_scale=T(np.ones(M, np.float32)), w_offset=0.0)
            assert (N(Y) == 127 * c * v + c).all()
