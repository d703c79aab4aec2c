"""GPU: the root-mean-square norm with residual and 8-bit output, and its gradients, against
the float64 oracle.

Tolerances, in units u = 2^-24 of binary32 (relative error of one rounding):
  sum of squares   at most 48 additions a thread and 10 of the tree, all terms positive: 60 u;
                   rstd half of that and 3 roundings more: 33 u
  y                two products more: 36 u; then half a step of its type
  scale            rstd, product, division's constant: 36 u
  codes            127 h w / a: product, quotient, fused sum: 4 u of at most 127, and 0.5 + that
                   of a step from the value; h w of a rounded h: 1 u more
  grad_x           the sum over k (60 u of sum |g n|), six roundings of each term: 70 u of the terms'
                   magnitudes
  grad_w           M terms, 3 roundings each, added in any order: (M + 3) u of their magnitudes
"""
import ctypes as C

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import norm
from gpu_util import T, N

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# one element, less than a vector, one and two vectors a row, odd lengths in all forms of the
# kernels, their borders (256, 512, 1024, 2048, 4096, 8192), rows beyond the registers
SHAPES = [(1, 1), (3, 5), (9, 8), (17, 13), (5, 250), (33, 256), (7, 264), (19, 511), (2, 1000),
          (300, 1024), (11, 1032), (5, 1777), (6, 2048), (3, 2056), (2, 4096), (600, 4096), (4, 4100),
          (3, 8184), (2, 8192), (3, 8193), (2, 12296), (9, 10007), (1, 49152), (2500, 72), (1201, 129)]


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


def case(M, K, t, seed=0, spread=1.0):
    rng = np.random.default_rng(1000 * M + K + seed)
    x = torch.from_numpy(rng.normal(size=(M, K)) * spread).to(t)
    r = torch.from_numpy(rng.normal(size=(M, K)) * 2).to(t)
    w = torch.from_numpy(1 + 0.2 * rng.normal(size=K)).float()
    return x, r, w


def rounding(t, ref):
    """Half a step of type t at |ref| (its smallest subnormal below its normal numbers)."""
    f = torch.finfo(t)
    return f.eps / 2 * np.abs(ref) + f.smallest_normal * f.eps


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(dsq, shape, t):
    M, K = shape
    x, r, w = case(M, K, t)
    for res in (None, r):
        h, y, codes, scale, rstd = dsq.dsq_rmsnorm_fwd(
            x.cuda(), w.cuda(), 1e-5, residual=None if res is None else res.cuda(), want_rstd=True)
        H, Y, R = norm.forward(x.double().numpy(), w.numpy(), 1e-5,
                               None if res is None else res.double().numpy())
        assert codes is None and scale is None and (h is None) == (res is None)
        # (eps itself is rounded to binary32)
        assert np.all(np.abs(N(rstd) - R) <= 34 * U * R)
        assert y.dtype == t and y.shape == x.shape
        # (the sum of x and residual is one rounding more)
        assert np.all(np.abs(N(y.double()) - Y) <= 38 * U * np.abs(Y) + rounding(t, Y) * (1 + 40 * U))
        if res is not None:
            assert np.all(np.abs(N(h.double()) - H) <= U * np.abs(H) + rounding(t, H) * (1 + 2 * U))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_eight_bits(dsq, shape, t):
    M, K = shape
    x, r, w = case(M, K, t, seed=1)
    h, y, codes, scale, _ = dsq.dsq_rmsnorm_fwd(x.cuda(), w.cuda(), 1e-5, residual=r.cuda(),
                                                quantised=True, want_codes=True)
    _, Y, _ = norm.forward(x.double().numpy(), w.numpy(), 1e-5, r.double().numpy())
    V, S = norm.eight_bits(Y)
    s, q = N(scale).astype(np.float64), N(codes).astype(np.float64)
    assert np.all(np.abs(s - S) <= 38 * U * S)
    assert np.all(np.abs(q - V) <= 0.5 + 8 * U * 127) and np.abs(q).max(1).min() == 127
    assert np.all(np.abs(N(y.double()) - s[:, None] * q) <= U * np.abs(s[:, None] * q)
                  + rounding(t, s[:, None] * q) * (1 + 2 * U))
    # codes alone, values alone: the same
    for want_y, want_codes in ((False, True), (True, False)):
        h2, y2, c2, s2, _ = dsq.dsq_rmsnorm_fwd(x.cuda(), w.cuda(), 1e-5, residual=r.cuda(),
                                                quantised=True, want_y=want_y, want_codes=want_codes)
        assert torch.equal(h, h2) and torch.equal(scale, s2)
        assert (torch.equal(y, y2) if want_y else y2 is None)
        assert (torch.equal(codes, c2) if want_codes else c2 is None)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(dsq, shape, t):
    M, K = shape
    h, gy, w = case(M, K, t, seed=2)
    gh = case(M, K, t, seed=3)[0]
    _, _, R = norm.forward(h.double().numpy(), w.numpy(), 1e-5)
    rstd = torch.from_numpy(R).float()
    for add in (None, gh):
        gx, gw = dsq.dsq_rmsnorm_bwd(gy.cuda(), h.cuda(), w.cuda(), rstd.cuda(),
                                     grad_h=None if add is None else add.cuda())
        GX, GW, mx, mw = norm.backward(gy.double().numpy(), h.double().numpy(), w.numpy(),
                                       rstd.numpy(), None if add is None else add.double().numpy())
        assert gx.dtype == t
        assert np.all(np.abs(N(gx.double()) - GX) <= 71 * U * mx + rounding(t, GX))
        assert gw.dtype == torch.float32 and np.all(np.abs(N(gw) - GW) <= (M + 3) * U * mw)
        only, none = dsq.dsq_rmsnorm_bwd(gy.cuda(), h.cuda(), w.cuda(), rstd.cuda(),
                                         grad_h=None if add is None else add.cuda(),
                                         want_weight=False)
        assert none is None and torch.equal(only, gx)
        again = dsq.dsq_rmsnorm_bwd(gy.cuda(), h.cuda(), w.cuda(), rstd.cuda(),
                                    grad_h=None if add is None else add.cuda())
        assert torch.equal(again[0], gx) and torch.equal(again[1], gw)


@pytest.mark.parametrize("shape", [(64, 1024), (37, 1777), (4, 8193)])
@pytest.mark.parametrize("t", TYPES)
def test_in_place_and_leading_dimensions(dsq, shape, t):
    M, K = shape
    x, r, w = case(M, K, t, seed=4)
    ref = dsq.dsq_rmsnorm_fwd(x.cuda(), w.cuda(), 1e-6, residual=r.cuda(), quantised=True,
                              want_codes=True, want_rstd=True)
    for which in ("x", "residual"):
        xs, rs = x.cuda().view(1, M, K), r.cuda().view(1, M, K)
        out = xs if which == "x" else rs
        got = dsq.dsq_rmsnorm_fwd(xs, w.cuda(), 1e-6, residual=rs, quantised=True, want_codes=True,
                                  want_rstd=True, out_h=out)
        assert got[0] is out and got[3].shape == (1, M)
        for a, b in zip(ref, got):
            assert torch.equal(a.view(-1), b.view(-1))
    # the gradient into the buffer of one of its inputs (raw entry point)
    gy, gh = (case(M, K, t, seed=s)[0].cuda() for s in (5, 6))
    gx, gw = dsq.dsq_rmsnorm_bwd(gy, ref[0], w.cuda(), ref[4], grad_h=gh)
    ws = torch.empty(dsq.dsq_rmsnorm_bwd_workspace_bytes(M, K), dtype=torch.uint8, device="cuda")
    wc = w.cuda()
    for which in (0, 1):
        g = [gy.clone(), gh.clone()]
        out = torch.empty(K, device="cuda")
        p = [C.c_void_p(a.data_ptr()) for a in (g[0], g[1], ref[0], wc, ref[4], g[which], out, ws)]
        st = dsq.lib.dsq_rmsnorm_bwd(*p[:5], M, K, {torch.float32: 0, torch.bfloat16: 1,
                                                    torch.float16: 2}[t], p[5], p[6], p[7],
                                     ws.numel(), C.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert st == 0 and torch.equal(g[which], gx) and torch.equal(out, gw)


@pytest.mark.parametrize("K", [64, 1777, 4096, 9000])
def test_rows_that_are_zero_infinite_or_nan(dsq, K):
    x = torch.randn(6, K, device="cuda", dtype=torch.bfloat16)
    x[1] = 0
    x[2, K // 2] = float("inf")
    x[3, K - 1] = float("nan")
    x[4] = x[0]
    w = torch.ones(K, device="cuda")
    _, y, codes, scale, rstd = dsq.dsq_rmsnorm_fwd(x, w, 1e-5, quantised=True, want_codes=True,
                                                   want_rstd=True)
    assert scale[1] == 0 and not codes[1].any() and not y[1].any()
    for m in (2, 3):
        assert torch.isnan(scale[m]) and not codes[m].any() and torch.isnan(y[m]).all()
    # a bad row leaves the others alone (a row's sum may be taken in another order where rows shift)
    assert torch.equal(codes[4], codes[0]) and torch.isfinite(y[5]).all()
    assert torch.allclose(scale[4], scale[0], rtol=1e-6, atol=0)
    _, y, _, _, _ = dsq.dsq_rmsnorm_fwd(x, w, 1e-5)
    ref = x.float() * torch.rsqrt(x.float().square().mean(1, keepdim=True) + 1e-5)
    assert torch.equal(torch.isnan(y), torch.isnan(ref)) and not y[1].any()


def test_nothing_outside_the_rows_is_written(dsq):
    M, K = 5, 333
    pad = torch.full((M * K + 64,), 7.0, device="cuda", dtype=torch.bfloat16)
    res = torch.randn(M * K, device="cuda").bfloat16()
    pad[:M * K] = res
    x = torch.randn(M, K, device="cuda").bfloat16()
    w = torch.ones(K, device="cuda")
    h, _, _, _, _ = dsq.dsq_rmsnorm_fwd(x, w, 1e-5, residual=pad[:M * K].view(M, K),
                                        out_h=pad[:M * K].view(M, K))
    assert (pad[M * K:] == 7.0).all()
    assert torch.equal(pad[:M * K].view(M, K), (x.float() + res.view(M, K).float()).bfloat16())


@pytest.mark.parametrize("K", [4096, 49152])
def test_more_than_2_to_the_31_elements(dsq, K):
    M = 2 ** 31 // K + 40
    base = torch.randn(64, K, device="cuda").bfloat16()
    x = torch.empty(M, K, device="cuda", dtype=torch.bfloat16)
    x[:] = 1.0
    x[-64:] = base
    w = 1 + 0.1 * torch.randn(K, device="cuda")
    alone = dsq.dsq_rmsnorm_fwd(base, w, 1e-5, quantised=True, want_codes=True, want_rstd=True)
    _, y, codes, scale, rstd = dsq.dsq_rmsnorm_fwd(x, w, 1e-5, quantised=True, want_codes=True, want_rstd=True)
    for a, b in zip((y, codes, scale, rstd), alone[1:]):
        assert torch.equal(a[-64:], b)
    del y, codes
    gx, _ = dsq.dsq_rmsnorm_bwd(x, x, w, rstd, want_weight=False)
    want, _ = dsq.dsq_rmsnorm_bwd(base, base, w, alone[4], want_weight=False)
    assert torch.equal(gx[-64:], want)


def test_captured_backward_passes_beside_one_another(dsq):
    """Two captured steps with a workspace each, replayed at once on two streams, with new inputs."""
    M, K = 700, 2048
    w = 1 + 0.1 * torch.randn(K, device="cuda")
    def inputs(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        return [torch.randn(M, K, device="cuda", generator=g).bfloat16() for _ in range(3)]

    def step(x, r, gy, ws):
        h, y, _, _, rstd = dsq.dsq_rmsnorm_fwd(x, w, 1e-5, residual=r, want_rstd=True)
        return (y,) + tuple(dsq.dsq_rmsnorm_bwd(gy, h, w, rstd, grad_h=gy, ws=ws))

    size = dsq.dsq_rmsnorm_bwd_workspace_bytes(M, K)
    held = []
    for i in range(2):
        a, ws = inputs(50 + i), torch.empty(size, dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(*a, ws)
        held.append((g, a, ws, out, torch.cuda.Stream()))
    for seed in range(4):
        new = [inputs(2 * seed + i) for i in range(2)]
        ref = [step(*a, None) for a in new]
        for (g, a, _, _, _), n in zip(held, new):
            for t, v in zip(a, n):
                t.copy_(v)
        torch.cuda.synchronize()
        for _ in range(3):
            for g, _, _, _, s in held:
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for (_, _, _, out, _), r in zip(held, ref):
            assert all(torch.equal(a, b) for a, b in zip(out, r))
