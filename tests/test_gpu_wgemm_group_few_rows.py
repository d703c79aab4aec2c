"""GPU: one or two rows of 16 bits with group-wise 4-bit weights, whatever the spread of a row's elements.

An element's product with a code is exact.  What is rounded is the addition of sums of up to 128 codes (of a piece:
128, 64 or 32 codes that no group's end cuts) in binary32.  A warp's total of one of the four digits takes
ceil(K / 2048) 256 / piece of them, eight warps' totals 8 more, the digits 4, and the digits' magnitudes add up to at
most three times the element's (1 0 0 and -128 where the element is 128).  Elements that need a second or third turn
of digits add as many additions again, of sums 2^-30 as large."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import groups as G
from gpu_util import T, N

U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


def check(Y, x, codes, scales, group, off):
    k = x.shape[1]
    ref, mag = G.linear(x, codes, scales, group, None, None, off)
    piece = 128 if group % 128 == 0 else 64 if group % 64 == 0 else 32
    adds = -(-k // 2048) * (256 // piece) + 12
    f = torch.finfo(Y.dtype)
    tol = 1.01 * adds * 3 * U * mag + f.eps / 2 * np.abs(ref) + f.smallest_normal * f.eps
    assert np.all(np.abs(N(Y.double()) - ref) <= tol)


def weights(dsq, rng, n, k, group, powers=False):
    codes = rng.integers(-8, 8, (n, k)).astype(np.int8)
    scales = rng.uniform(0.5, 1.5, (-(-k // group), n)) * 0.01
    if powers:
        scales = np.ldexp(1.0, rng.integers(-3, 3, scales.shape))
    return codes, scales.astype(np.float32)


SIZES = [(1, 40, 264, 32), (2, 33, 1032, 64), (1, 70, 4104, 128), (2, 64, 2056, 96), (1, 17, 200, 1 << 20), (2, 130, 8192, 128)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("e", [0, 4, 8, 10, 12, 14, 15])
@pytest.mark.parametrize("size", SIZES)
def test_outliers(dsq, size, e, t):
    """One element of each 256 2^e above the rest, with weights of any size and with weights of 0."""
    M, n, k, group = size
    rng = np.random.default_rng(7 * k + e)
    codes, scales = weights(dsq, rng, n, k, min(group, k))
    x = rng.normal(size=(M, k))
    at = np.arange(0, k, 256) + rng.integers(0, 256, -(-k // 256))
    at = at[at < k]
    x[:, at] = np.ldexp(rng.choice([-1.5, 1.25], (M, len(at))), e)
    x = torch.from_numpy(x).to(t)
    none = codes.copy()
    none[:, at] = 0
    for c, off in ((codes, 0.5), (codes, 0.0), (none, 0.0), (none, 0.5)):
        Y = dsq.dsq_wgemm_group(x.cuda(), dsq.dsq_pack_codes(T(c), 4), M, n, k, 4, group, T(scales), w_offset=off)
        check(Y, x.double().numpy(), c, scales, min(group, k), off)


@pytest.mark.parametrize("e", [16, 20, 22, 30, 31, 60, 100, 127])
@pytest.mark.parametrize("size", SIZES)
def test_outliers_beyond_fp16(dsq, size, e):
    """The outlier's own weight is 0: what is left is exact sums of small integers, in any order."""
    M, n, k, group = size
    rng = np.random.default_rng(11 * k + e)
    codes, scales = weights(dsq, rng, n, k, min(group, k), powers=True)
    x = rng.integers(-9, 10, (M, k)).astype(np.float64)
    at = rng.integers(0, k, (M, 3))
    for m in range(M):
        x[m, at[m]] = np.ldexp(rng.choice([-1.0, 1.25], 3), e)
        codes[:, at[m]] = 0
    x = torch.from_numpy(x).to(torch.bfloat16)
    Y = dsq.dsq_wgemm_group(x.cuda(), dsq.dsq_pack_codes(T(codes), 4), M, n, k, 4, group, T(scales), w_offset=0.0)
    assert np.array_equal(N(Y), G.linear(x.double().numpy(), codes, scales, min(group, k), w_offset=0.0)[0])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_digit(dsq, group, t):
    """Integers that fill all digits of a chunk's grid, one nonzero code a column: each product by itself, exact."""
    n = k = 520
    rng = np.random.default_rng(group)
    bits = 8 if t == torch.bfloat16 else 11
    codes = np.zeros((n, k), np.int8)
    codes[np.arange(n), rng.permutation(k)] = rng.choice([-8, -3, -1, 1, 2, 7], n)
    scales = np.ldexp(1.0, rng.integers(-4, 5, (-(-k // group), n))).astype(np.float32)
    for spread in (12, 20, 24):
        # numbers of 8 (11) bits, shifted
        low = -24 if t == torch.float16 else -40
        x = rng.integers(-2 ** bits + 1, 2 ** bits, (2, k)) * np.ldexp(1.0, low + rng.integers(0, spread + 1, (2, k)))
        x = torch.from_numpy(x).to(t)
        Y = dsq.dsq_wgemm_group(x.cuda(), dsq.dsq_pack_codes(T(codes), 4), 2, n, k, 4, group, T(scales), w_offset=0.0)
        assert np.array_equal(N(Y), G.linear(x.double().numpy(), codes, scales, group, w_offset=0.0)[0])


def test_smallest_and_largest_elements(dsq):
    """All of bf16's range beside one another, and chunks of its smallest numbers alone."""
    n, k, group = 64, 1024, 128
    rng = np.random.default_rng(5)
    codes = np.zeros((n, k), np.int8)
    codes[np.arange(n), rng.permutation(k)[:n]] = rng.integers(1, 8, n)
    for lo, hi, sc in ((-133, -126, 120), (-133, -100, 110), (-133, 119, 0), (100, 119, -60)):
        x = rng.integers(-255, 256, (2, k)) * np.ldexp(1.0, rng.integers(lo, hi + 1, (2, k)))
        x = torch.from_numpy(x).to(torch.bfloat16)
        scales = np.full((k // group, n), np.ldexp(1.0, sc), np.float32)
        Y = dsq.dsq_wgemm_group(x.cuda(), dsq.dsq_pack_codes(T(codes), 4), 2, n, k, 4, group, T(scales), w_offset=0.0)
        ref = G.linear(x.double().numpy(), codes, scales, group, w_offset=0.0)[0]
        assert np.isfinite(ref).all() and np.array_equal(N(Y), ref.astype(np.float32))


@pytest.mark.parametrize("e", [30, 40, 46, 50, 90, 126])
@pytest.mark.parametrize("low", [-20, -60, -75, -100, -133])
def test_elements_beside_one_that_is_out_of_their_range(dsq, low, e):
    """One large element with a weight of 0 and all others so small that their quotient by its grid is none of
    binary32's."""
    n, k, group = 48, 520, 32
    rng = np.random.default_rng(e - low)
    codes, scales = weights(dsq, rng, n, k, group)
    codes[:, [3, 300]] = 0
    x = rng.integers(-15, 16, (1, k)) * np.ldexp(1.0, low)
    x[:, [3, 300]] = 2.0 ** e
    scales[:] = np.ldexp(1.0, -low - 20)
    x = torch.from_numpy(x).to(torch.bfloat16)
    Y = dsq.dsq_wgemm_group(x.cuda(), dsq.dsq_pack_codes(T(codes), 4), 1, n, k, 4, group, T(scales), w_offset=0.0)
    assert np.array_equal(N(Y), G.linear(x.double().numpy(), codes, scales, group, w_offset=0.0)[0])


@pytest.mark.parametrize("t", TYPES)
def test_a_bad_row_beside_one_with_outliers(dsq, t):
    n, k, group = 100, 1000, 64
    rng = np.random.default_rng(9)
    codes, scales = weights(dsq, rng, n, k, group)
    codes[:, 5] = 0
    x = torch.from_numpy(rng.normal(size=(2, k))).to(t)
    x[1, 5] = 2.0 ** 15
    packed = dsq.dsq_pack_codes(T(codes), 4)
    alone = dsq.dsq_wgemm_group(x[1:].cuda(), packed, 1, n, k, 4, group, T(scales), w_offset=0.0)
    check(alone, x[1:].double().numpy(), codes, scales, group, 0.0)
    for bad in (float("inf"), -float("inf"), float("nan")):
        x[0, 700] = bad
        Y = dsq.dsq_wgemm_group(x.cuda(), packed, 2, n, k, 4, group, T(scales), w_offset=0.0)
        assert torch.equal(Y[1], alone[0]) and not torch.isfinite(Y[0]).any()


def test_one_row_and_three_rows_agree(dsq):
    """The same row by itself and among others: the kernels differ by the roundings of their additions alone."""
    n, k, group = 300, 4096, 128
    rng = np.random.default_rng(21)
    codes, scales = weights(dsq, rng, n, k, group)
    x = rng.normal(size=(3, k))
    x[:, ::256] = 3000.0
    codes[:, ::256] = 0
    x = torch.from_numpy(x).bfloat16()
    packed = dsq.dsq_pack_codes(T(codes), 4)
    few = dsq.dsq_wgemm_group(x[:1].cuda(), packed, 1, n, k, 4, group, T(scales), w_offset=0.0)
    three = dsq.dsq_wgemm_group(x.cuda(), packed, 3, n, k, 4, group, T(scales), w_offset=0.0)
    mag = G.linear(x.double().numpy(), codes, scales, group, w_offset=0.0)[1][0]
    # (one row: above; three: 128 additions of a group in the tensor core, each off by 2^-23 of what is there, and 32 groups)
    assert np.all(np.abs(N(few[0].double()) - N(three[0].double())) <= ((32 + 12) * 3 + 128 * 2 + 32) * U * mag)
