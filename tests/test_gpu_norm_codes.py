"""GPU: the norm's 8-bit codes are those of the exact quotient 127 h w / a, h the sum in binary32:
they are equal, at borders between two codes too."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import norm
from gpu_util import T, N

TYPES = [torch.float32, torch.bfloat16, torch.float16]
# every number of threads a row, rows that shift, rows beyond the registers
LENGTHS = [5, 64, 72, 250, 264, 511, 777, 1024, 1777, 2048, 4096, 4100, 8192, 8193, 9000, 12296]


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


def check(dsq, x, r, w, h):
    """h: the sums in binary32."""
    _, y, codes, scale, _ = dsq.dsq_rmsnorm_fwd(x, w, 1e-5, residual=r, quantised=True, want_codes=True)
    want = norm.exact_codes(h, N(w))
    assert np.array_equal(N(codes).astype(np.int64), want)
    # the fake-quantised output is the same codes': one product, one rounding to the type
    s = N(scale).astype(np.float64)[:, None]
    f = torch.finfo(x.dtype)
    ref = s * want
    assert np.all(np.abs(N(y.double()) - ref) <= (2.0 ** -24 + f.eps / 2) * (1 + f.eps) * np.abs(ref)
                  + f.smallest_normal * f.eps)


def sum32(x, r):
    return N(x.float()) if r is None else N(x.float()) + N(r.float())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("K", LENGTHS)
def test_borders(dsq, K, t):
    """Rows of multiples of 1/2 whose largest is 127 times an odd number: every half code is met, and
    127 / a is no number of binary32 (but where the odd number is 1)."""
    rng = np.random.default_rng(K)
    M = 11
    odd = rng.choice([1, 3, 5, 7, 9, 11, 13], M)
    # h = odd (j + 1/2), as the sum of two parts that each type holds
    j = rng.integers(-127, 127, (M, K))
    h = odd[:, None] * (j + 0.5)
    part = np.round(h / 16) * 16
    at = rng.integers(0, K, M)
    h[np.arange(M), at] = 127 * odd * rng.choice([-1, 1], M)
    part[np.arange(M), at] = np.round(h[np.arange(M), at] / 16) * 16
    x, r = (torch.from_numpy(a).to(t).cuda() for a in (part, h - part))
    assert np.array_equal(sum32(x, r), h)
    check(dsq, x, r, torch.ones(K, device="cuda"), h)
    # weights that are powers of two, and negative
    w = np.ldexp(1.0, rng.integers(-2, 3, K)) * rng.choice([-1, 1], K)
    check(dsq, x, r, T(w.astype(np.float32)), sum32(x, r))


@pytest.mark.parametrize("e", [-110, -100, -61, -59, -20, 40, 100])
def test_borders_of_small_and_large_rows(dsq, e):
    rng = np.random.default_rng(200 + e)
    M, K = 9, 1500
    odd = rng.choice([3, 5, 7, 9, 11, 13], M)
    h = odd[:, None] * (rng.integers(-127, 127, (M, K)) + 0.5)
    h[:, 7] = 127 * odd
    x = torch.from_numpy(np.ldexp(h, e - 3)).float().cuda()
    check(dsq, x, None, torch.ones(K, device="cuda"), sum32(x, None))
    # the weight takes a part of the power of two, and products of 48 bits
    w = np.ldexp(1 + rng.integers(0, 2 ** 20, K) * 2.0 ** -20, -3).astype(np.float32)
    check(dsq, x, None, T(w), sum32(x, None))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("K", [72, 264, 1024, 1777, 4096, 9000])
def test_many_rows(dsq, K, t):
    """Three million elements a case: some thirty are within binary32's rounding of a border."""
    M = 3_000_000 // K
    g = torch.Generator(device="cuda").manual_seed(K)
    x, r = (torch.randn(M, K, device="cuda", generator=g) * s for s in (1.0, 2.0))
    x[:, ::61] *= 12
    w = 1 + 0.1 * torch.randn(K, device="cuda", generator=g)
    x, r = x.to(t), r.to(t)
    check(dsq, x, r, w, sum32(x, r))


def test_largest_products_that_round_alike(dsq):
    """Several products share the largest rounded magnitude: the exact largest one is the row's."""
    rng = np.random.default_rng(77)
    M, K = 400, 640
    x = rng.normal(size=(M, K)).astype(np.float32) * 0.2
    w = (1 + 0.2 * rng.normal(size=K)).astype(np.float32)
    # products that are 3 as nearly as binary32 allows
    near = np.argsort(rng.random((M, K)), 1)[:, :K // 2]
    for m in range(M):
        x[m, near[m]] = (3.0 / w[near[m]].astype(np.float64)).astype(np.float32) * rng.choice([-1, 1], K // 2)
    check(dsq, T(x), None, T(w), x)
    # elements beside every border of such rows
    for m in range(M):
        k = near[m, ::3]
        x[m, k] = (3.0 * (2 * rng.integers(-127, 127, len(k)) + 1) / 254 / w[k].astype(np.float64)).astype(np.float32)
    check(dsq, T(x), None, T(w), x)
