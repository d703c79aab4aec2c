"""GPU: weights in groups of 4-bit codes against exact arithmetic: codes are equal, scales and
values off by their own rounding."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import groups as G
from gpu_util import T, N

TYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


def unpacked(dsq, codes, n, k):
    return N(dsq.dsq_unpack(codes, n, k, 4, True)).astype(np.int64)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("size", [(1, 1, 32), (3, 31, 32), (5, 33, 32), (7, 64, 64), (130, 200, 128),
                                  (9, 1777, 256), (33, 1800, 256), (17, 320, 96), (4, 2000, 512),
                                  (3, 100, 1 << 40), (2, 70000, 70016), (600, 1024, 128)])
def test_codes_scales_values(dsq, size, t):
    n, k, group = size
    rng = np.random.default_rng(n * 7919 + k)
    # half of the rows small integers: ratios on the borders between codes
    w = rng.normal(size=(n, k)) * 0.02
    w[::2] = rng.integers(-45, 46, w[::2].shape)
    w = torch.from_numpy(w).to(t)
    w[-1, -min(k, 40):] = 0.0
    codes, scales = dsq.dsq_quantize_groups(w.cuda(), 4, group)
    C, S = G.quantize(w.double().numpy(), min(group, k))
    assert codes.shape == (n, dsq.dsq_row_pitch(k, 4)) and scales.shape == S.shape
    assert np.array_equal(unpacked(dsq, codes, n, k), C)
    # spare codes are zero
    width = 2 * codes.shape[1]
    assert not unpacked(dsq, codes, n, width)[:, k:].any()
    assert np.all(np.abs(N(scales) - S) <= U * S)
    for off in (0.5, 0.0):
        for to in TYPES:
            v = dsq.dsq_dequantize_groups(codes, scales, n, k, 4, group, off, to)
            V = G.values(C, N(scales).astype(np.float64), min(group, k), off)
            f = torch.finfo(to)
            # one product in binary32, one rounding to the type
            assert v.dtype == to and np.all(np.abs(N(v.double()) - V) <= (U + f.eps / 2) * (1 + U) * np.abs(V)
                                            + f.smallest_normal * f.eps)


def test_extreme_ranges(dsq):
    """Magnitudes at both ends of binary32, subnormal ones too, and rows with NaN and infinities."""
    rng = np.random.default_rng(3)
    w = rng.normal(size=(12, 64))
    for i, e in enumerate((-149, -140, -127, -126, -100, -60, 60, 100, 125)):
        w[i] = np.ldexp(w[i] / np.abs(w[i]).max() * 1.9, e)
    w = w.astype(np.float32)
    w[9, 3], w[10, 40], w[11, 0] = np.inf, np.nan, -np.inf
    codes, scales = dsq.dsq_quantize_groups(T(w), 4, 32)
    C, S = G.quantize(w[:9], 32)
    assert np.array_equal(unpacked(dsq, codes, 12, 64)[:9], C)
    s = N(scales)
    assert np.all(np.abs(s[:, :9] - S) <= U * S + 2.0 ** -150)
    bad = np.isnan(s[:, 9:])
    assert np.array_equal(bad, [[True, False, True], [False, True, False]])
    v = N(dsq.dsq_dequantize_groups(codes, scales, 12, 64, 4, 32, out_dtype=torch.float32))
    assert np.isnan(v[9, :32]).all() and np.isfinite(v[9, 32:]).all() and np.isnan(v[10, 32:]).all()


def test_more_than_2_to_the_31_weights(dsq):
    """Offsets that pass 32 bits: the last rows of a long matrix are those of a short one."""
    n, k = 33000, 66000
    free, _ = torch.cuda.mem_get_info()
    if free < 16 << 30:
        pytest.skip("needs 16 GB")
    w = torch.zeros(n, k, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(3, k, device="cuda").bfloat16()
    w[-3:] = tail
    codes, scales = dsq.dsq_quantize_groups(w, 4, 128)
    c, s = dsq.dsq_quantize_groups(tail, 4, 128)
    assert torch.equal(codes[-3:], c) and torch.equal(scales[:, -3:], s)
    del w
    v = dsq.dsq_dequantize_groups(codes, scales, n, k, 4, 128)
    assert torch.equal(v[-3:], dsq.dsq_dequantize_groups(c, s, 3, k, 4, 128))
    assert not v[:-3].any()


@pytest.mark.parametrize("t", TYPES)
def test_weights_far_below_the_largest(dsq, t):
    """Below zero, by however little beside the group's largest, is code -1; zero and above is 0."""
    f = torch.finfo(t)
    least = f.smallest_normal * f.eps
    small = torch.tensor([-least, least, -f.smallest_normal, f.smallest_normal, -0.0, 0.0, -3 * least, 5 * least],
                         dtype=torch.float64)
    for top in (f.max, 1.0, 2.0 ** -13):
        w = torch.zeros(2, 64, dtype=torch.float64)
        w[:, 8:16] = small
        w[:, 40:48] = small
        w[:, 0] = torch.tensor([top, -top], dtype=torch.float64)
        w[:, 63] = -top
        w = w.to(t)
        C, S = G.quantize(w.double().numpy(), 32)
        codes, scales = dsq.dsq_quantize_groups(w.cuda(), 4, 32)
        assert np.array_equal(unpacked(dsq, codes, 2, 64), C)
        if top >= 1.0:        # (fp16's smallest normal number is half of 2^-13)
            assert (C[:, 8:16] == [-1, 0, -1, 0, 0, 0, -1, 0]).all()
