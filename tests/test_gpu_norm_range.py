"""GPU: rows whose squares leave binary32's range, rows of zeros with eps = 0, and their neighbours.

Tolerances as in the norm's other tests, in units u = 2^-24 (a power of two more is exact): rstd 34 u, y 38 u and half a
step of its type, the scale 38 u.  Where rstd is subnormal it is off by half of 2^-149 too."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import norm
from gpu_util import T, N

U = 2.0 ** -24
LENGTHS = [3, 64, 100, 250, 256, 511, 640, 1024, 1777, 2048, 4096, 8184, 8193, 12296]


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


def rounding(t, ref):
    f = torch.finfo(t)
    return f.eps / 2 * np.abs(ref) + f.smallest_normal * f.eps


def check(dsq, x, w, eps, rows, oracle_rows=None):
    t = x.dtype
    xd = N(x.double())
    H, Y, R = norm.forward(xd, N(w), eps)
    _, y, _, _, rstd = dsq.dsq_rmsnorm_fwd(x, w, eps, want_rstd=True)
    _, y8, codes, scale, rstd8 = dsq.dsq_rmsnorm_fwd(x, w, eps, quantised=True, want_codes=True, want_rstd=True)
    r, y, y8, s = (N(a.double()) for a in (rstd, y, y8, scale))
    assert torch.equal(rstd, rstd8)
    for m in rows:
        off = 34 * U + 2.0 ** -150 / R[m]
        assert abs(r[m] - R[m]) <= off * R[m]
        assert np.all(np.abs(y[m] - Y[m]) <= (off + 4 * U) * np.abs(Y[m]) + rounding(t, Y[m]) * (1 + 40 * U))
        S = np.abs(Y[m]).max() / 127
        assert abs(s[m] - S) <= (off + 4 * U) * S
        assert np.array_equal(N(codes)[m].astype(np.int64), norm.exact_codes(xd[m:m + 1], N(w))[0])
        v = s[m] * N(codes)[m]
        assert np.all(np.abs(y8[m] - v) <= U * np.abs(v) + rounding(t, v) * (1 + 2 * U))
    return r, y, y8, s, N(codes)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", LENGTHS)
def test_large_rows(dsq, K, t):
    rng = np.random.default_rng(K)
    x = rng.normal(size=(13, K))
    x[2] *= 1e19
    x[3] *= 1e20
    x[4] *= 1e30
    x[7] *= 3e37
    x[9, 0] = 1e25                    # one element
    x[12] = 2.0 ** 126 * rng.choice([-1, 1], K)
    x = torch.from_numpy(x).to(t).cuda()
    w = T((1 + 0.1 * rng.normal(size=K)).astype(np.float32) * 0.5)
    check(dsq, x, w, 1e-5, range(13))
    check(dsq, x, w, 0.0, range(13))
    # the large rows alone do not change their neighbours
    few = [0, 1, 5, 6, 8, 10, 11]
    z = x.clone()
    for m in set(range(13)) - set(few):
        z[m] = 1.0
    a, b = (dsq.dsq_rmsnorm_fwd(v, w, 1e-5, quantised=True, want_codes=True, want_rstd=True)[1:] for v in (x, z))
    for i in range(4):
        assert torch.equal(a[i][few], b[i][few])


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", LENGTHS)
def test_small_rows_and_no_eps(dsq, K, t):
    rng = np.random.default_rng(K + 1)
    x = rng.normal(size=(11, K))
    for m, e in ((1, -40), (2, -60), (3, -75), (5, -90), (6, -110)):
        x[m] = np.ldexp(x[m], e)
    x[8] = 0
    x = torch.from_numpy(x).to(t).cuda()
    w = T((1 + 0.1 * rng.normal(size=K)).astype(np.float32))
    r, y, y8, s, codes = check(dsq, x, w, 0.0, [m for m in range(11) if m != 8])
    assert r[8] == 0 and s[8] == 0 and not y[8].any() and not y8[8].any() and not codes[8].any()
    check(dsq, x, w, 1e-30, [m for m in range(11) if m != 8])
    # backward: what reaches a row of zeros is the residual stream's gradient
    gy, gh = (torch.randn(11, K, device="cuda").to(t) for _ in range(2))
    _, _, _, _, rstd = dsq.dsq_rmsnorm_fwd(x, w, 0.0, want_rstd=True)
    gx, gw = dsq.dsq_rmsnorm_bwd(gy, x, w, rstd, grad_h=gh)
    assert torch.equal(gx[8], gh[8]) and torch.isfinite(gw).all()


def test_rstd_beyond_binary32(dsq):
    """Subnormal rows with eps = 0: rstd is the largest number, what is computed with it finite."""
    x = torch.full((3, 512), 2.0 ** -140, device="cuda")
    x[1] = 1.0
    _, y, _, _, rstd = dsq.dsq_rmsnorm_fwd(x, torch.ones(512, device="cuda"), 0.0, want_rstd=True)
    top = torch.finfo(torch.float32).max
    assert rstd[0] == top and rstd[2] == top and rstd[1] == 1 and torch.equal(y[1], x[1])
    assert torch.equal(y[0], x[0] * top)


@pytest.mark.parametrize("eps", [1e20, 3e38])
def test_large_eps(dsq, eps):
    x = torch.randn(5, 700, device="cuda")
    x[2] *= 1e19
    check(dsq, x, torch.ones(700, device="cuda"), float(np.float32(eps)), range(5))
