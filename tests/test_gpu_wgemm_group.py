"""GPU: products of few rows with group-wise 4-bit weights against float64.

Tolerances: products are exact; a group's sum in the tensor core's binary32 and the sum over
groups take at most K additions, each off by 2^-23 of the terms added so far (the core may cut
instead of rounding): K 2^-23 sum |x v s|, 2^-22 of that for scale, bias and row scale, half a step
of the type.  In int8 a group's sum is exact: (groups + 5) 2^-24 of the groups' magnitudes."""
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


def weights(dsq, n, k, group, seed=0):
    rng = np.random.default_rng(seed + 31 * n + k)
    codes = rng.integers(-8, 8, (n, k)).astype(np.int8)
    scales = (rng.uniform(0.5, 1.5, (-(-k // group), n)) * 0.01).astype(np.float32)
    bias = rng.normal(size=n).astype(np.float32)
    return codes, scales, bias, dsq.dsq_pack_codes(T(codes), 4)


def check(Y, x, codes, scales, group, bias, off, row_scale=None):
    k = x.shape[1]
    ref, mag = G.linear(x, codes, scales, group, bias, row_scale, off)
    f = torch.finfo(Y.dtype)
    exact = row_scale is not None
    tol = ((scales.shape[0] + 5) * U if exact else (k + 2) * 2 * U) * mag + 4 * U * np.abs(ref)
    tol = tol + f.eps / 2 * np.abs(ref) + f.smallest_normal * f.eps
    assert np.all(np.abs(N(Y.double()) - ref) <= tol)
    if Y.dtype == torch.float32 and not exact and k > 512:
        # errors of single additions do not add up: far inside the bound on average
        assert np.mean(np.abs(N(Y.double()) - ref)) <= 0.05 * np.mean(tol)


SIZES = [(1, 1, 8, 32), (1, 33, 64, 32), (2, 40, 96, 96), (5, 17, 136, 64), (8, 100, 200, 128),
         (9, 31, 1032, 128), (16, 65, 520, 32), (17, 70, 264, 64), (31, 33, 2056, 256), (32, 8, 128, 64),
         (33, 96, 776, 32), (64, 130, 1288, 128), (65, 45, 392, 96), (130, 24, 640, 128), (1, 3000, 4104, 160),
         (3, 4750, 640, 64), (4, 1201, 1288, 1 << 40), (7, 64, 8200, 8224)]


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", SIZES)
def test_floating_rows(dsq, size, t):
    M, n, k, group = size
    codes, scales, bias, packed = weights(dsq, n, k, min(group, k))
    rng = np.random.default_rng(M)
    x = torch.from_numpy(rng.normal(size=(M, k))).to(t)
    for off, b, out in ((0.5, bias, torch.float32), (0.0, None, torch.float32), (0.5, None, t),
                        (0.0, bias, torch.float16)):
        Y = dsq.dsq_wgemm_group(x.cuda(), packed, M, n, k, 4, group, T(scales),
                                bias=None if b is None else T(b), w_offset=off, out_dtype=out)
        assert Y.dtype == out and Y.shape == (M, n)
        check(Y, x.double().numpy(), codes, scales, min(group, k), b, off)


@pytest.mark.parametrize("size", [s for s in SIZES if s[2] % 16 == 0] + [(6, 50, 48, 32), (40, 33, 1040, 64)])
def test_eight_bit_rows(dsq, size):
    M, n, k, group = size
    codes, scales, bias, packed = weights(dsq, n, k, min(group, k), 1)
    rng = np.random.default_rng(M)
    x = rng.integers(-128, 128, (M, k)).astype(np.int8)
    rs = rng.uniform(0.01, 0.02, M).astype(np.float32)
    for off, b, out in ((0.5, bias, torch.float32), (0.0, None, torch.float32), (0.5, bias, torch.bfloat16)):
        Y = dsq.dsq_wgemm_group(T(x), packed, M, n, k, 4, group, T(scales), row_scale=T(rs),
                                bias=None if b is None else T(b), w_offset=off, out_dtype=out)
        check(Y, x, codes, scales, min(group, k), b, off, rs)


@pytest.mark.parametrize("M", [1, 8, 16, 24, 64, 70])
def test_whole_numbers_are_exact(dsq, M):
    """Small integers and scales that are powers of two: every sum is exact, any order."""
    n, k, group = 200, 1000, 64
    codes, _, _, packed = weights(dsq, n, k, group)
    rng = np.random.default_rng(M)
    scales = np.ldexp(1.0, rng.integers(-3, 3, (16, n))).astype(np.float32)
    x = rng.integers(-4, 5, (M, k)).astype(np.float32)
    for t in (torch.bfloat16, torch.float16):
        Y = dsq.dsq_wgemm_group(T(x).to(t), packed, M, n, k, 4, group, T(scales))
        assert np.array_equal(N(Y), G.linear(x, codes, scales, group)[0])


def test_extreme_codes_and_largest_magnitudes(dsq):
    """Codes and 8-bit activations all at their ends: the largest group sums."""
    n, k = 40, 1 << 16
    for c, xv in ((7, 127), (-8, -128), (-8, 127)):
        codes = np.full((n, k), c, np.int8)
        packed = dsq.dsq_pack_codes(T(codes), 4)
        x = np.full((2, k), xv, np.int8)
        ones = np.ones((1, n), np.float32)
        Y = dsq.dsq_wgemm_group(T(x), packed, 2, n, k, 4, k, T(ones), row_scale=T(np.ones(2, np.float32)))
        want = float(k * xv * (2 * c + 1))
        assert np.all(np.abs(N(Y) - want) <= 6 * U * abs(want))


def test_nan_and_infinity_stay_in_their_rows_and_columns(dsq):
    M, n, k, group = 20, 70, 264, 64
    codes, scales, _, packed = weights(dsq, n, k, group)
    x = torch.randn(M, k, device="cuda").bfloat16()
    x[3, k - 1] = float("inf")
    x[17, 0] = float("nan")
    scales[2, 5] = np.nan
    scales[4, 69] = np.inf
    Y = N(dsq.dsq_wgemm_group(x, packed, M, n, k, 4, group, T(scales)))
    bad = ~np.isfinite(Y)
    want = np.zeros((M, n), bool)
    want[[3, 17]] = True
    want[:, [5, 69]] = True
    assert np.array_equal(bad, want)


def test_out_and_rows_behind_it(dsq):
    M, n, k = 9, 77, 200
    codes, scales, _, packed = weights(dsq, n, k, 32)
    x = torch.randn(M + 3, k, device="cuda").bfloat16()
    x[M:] = float("nan")
    out = torch.full((M + 3, n), 5.0, device="cuda")
    assert dsq.dsq_wgemm_group(x, packed, M, n, k, 4, 32, T(scales), out=out) is out
    assert (out[M:] == 5.0).all()
    check(out[:M].clone(), N(x[:M].double()), codes, scales, 32, None, 0.5)


@pytest.mark.parametrize("M", [1, 16, 64])
def test_a_call_gives_the_same_bits_again(dsq, M):
    n, k = 500, 2048
    codes, scales, bias, packed = weights(dsq, n, k, 128)
    x = torch.randn(M, k, device="cuda").bfloat16()
    Y = dsq.dsq_wgemm_group(x, packed, M, n, k, 4, 128, T(scales), bias=T(bias))
    for _ in range(5):
        assert torch.equal(Y, dsq.dsq_wgemm_group(x, packed, M, n, k, 4, 128, T(scales), bias=T(bias)))


def test_binding_refuses_small_buffers(dsq):
    codes, scales, bias, packed = weights(dsq, 10, 64, 32)
    x = torch.randn(2, 64, device="cuda").bfloat16()
    s = T(scales)
    bad = [dict(M=3), dict(N=11), dict(K=128), dict(group=16), dict(bias=torch.zeros(9, device="cuda")),
           dict(out=torch.empty(19, device="cuda"))]
    for b in bad:
        a = dict(M=2, N=10, K=64, group=32, bias=None, out=None)
        a.update(b)
        with pytest.raises((ValueError, dsq.DsqError)):
            dsq.dsq_wgemm_group(x, packed, a["M"], a["N"], a["K"], 4, a["group"], s, bias=a["bias"], out=a["out"])
    with pytest.raises(TypeError):
        dsq.dsq_wgemm_group(x.float(), packed, 2, 10, 64, 4, 32, s)
    with pytest.raises(TypeError):
        dsq.dsq_wgemm_group(x, packed, 2, 10, 64, 4, 32, s, out_dtype=torch.int32)
    with pytest.raises(dsq.DsqError):
        dsq.dsq_wgemm_group(x.to(torch.int8), packed, 2, 10, 64, 4, 32, s)


def test_layer_front_as_it_serves(dsq):
    """norm -> 8-bit codes -> product, then the next norm on the stream, eager, on another stream and
    as a replayed graph: the same numbers, and those of the definition."""
    M, K, n = 5, 512, 384
    rng = np.random.default_rng(8)
    x, r = (torch.from_numpy(rng.normal(size=(M, K))).bfloat16().cuda() for _ in range(2))
    w1 = T((1 + 0.1 * rng.normal(size=K)).astype(np.float32))
    w2 = T((1 + 0.1 * rng.normal(size=n)).astype(np.float32))
    W = torch.from_numpy(rng.normal(size=(n, K)) * 0.05).bfloat16().cuda()
    codes, scales = dsq.dsq_quantize_groups(W, 4, 64)
    codes2, scales2 = dsq.dsq_quantize_groups(W.t().contiguous(), 4, 128)

    def front(x, r):
        h, _, q, s, _ = dsq.dsq_rmsnorm_fwd(x, w1, 1e-5, residual=r, want_y=False, want_codes=True)
        y = dsq.dsq_wgemm_group(q, codes, M, n, K, 4, 64, scales, row_scale=s, out_dtype=torch.bfloat16)
        _, z, _, _, _ = dsq.dsq_rmsnorm_fwd(y, w2, 1e-5)
        return h, y, dsq.dsq_wgemm_group(z, codes2, M, K, n, 4, 128, scales2, out_dtype=torch.bfloat16)

    ref = front(x, r)
    xd, rd = x.double().cpu().numpy(), r.double().cpu().numpy()
    from oracle import norm
    _, Yn, _ = norm.forward(xd, N(w1), 1e-5, rd)
    V, S = norm.eight_bits(Yn)
    c1, s1 = G.quantize(N(W.double()), 64)
    y, mag = G.linear(np.floor(V + 0.5), c1, s1, 64, row_scale=S)
    # a code may fall on the other side of a border: one step of one activation
    step = np.max(S) * np.abs(G.values(c1, s1, 64)).max()
    assert np.all(np.abs(N(ref[1].double()) - y) <= 2.0 ** -8 * np.abs(y) + 1e-5 * mag + 2 * step)
    _, Z, _ = norm.forward(N(ref[1].double()), N(w2), 1e-5)
    c2, s2 = G.quantize(N(W.t().double()), 128)
    y2, mag2 = G.linear(Z, c2, s2, 128)
    assert np.all(np.abs(N(ref[2].double()) - y2) <= 2.0 ** -8 * np.abs(y2) + (2.0 ** -8 + 1e-5) * mag2)

    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = front(x, r)
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))

    xs, rs = torch.zeros_like(x), torch.zeros_like(r)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = front(xs, rs)
    for _ in range(3):
        xs.copy_(x)
        rs.copy_(r)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, held))
        xs.zero_()
        g.replay()


@pytest.fixture(params=[1, 2, 3])
def form(request, dsq):
    dsq.dsq_set_wgemm_group_form(request.param)
    yield request.param
    dsq.dsq_set_wgemm_group_form(0)


# both kernels at every size: columns and rows of a tile and one beyond, chunks of K and their
# remainders, each number of blocks along K
FORM_SIZES = [(1, 1, 16, 32), (1, 127, 128, 128), (3, 129, 256, 64), (8, 128, 384, 128), (9, 300, 2064, 32),
              (16, 257, 4096, 128), (17, 130, 1040, 64), (32, 128, 2048, 128), (33, 200, 3200, 32),
              (64, 384, 1152, 256), (65, 129, 1296, 64), (150, 140, 528, 96), (2, 1000, 8192, 128),
              (1, 20000, 1536, 128), (40, 2500, 1040, 128)]


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16, torch.int8])
@pytest.mark.parametrize("size", FORM_SIZES)
def test_both_kernels(dsq, form, size, t):
    M, n, k, group = size
    codes, scales, bias, packed = weights(dsq, n, k, group, 2)
    rng = np.random.default_rng(M)
    rs = None
    if t == torch.int8:
        x = torch.from_numpy(rng.integers(-128, 128, (M, k)).astype(np.int8))
        rs = rng.uniform(0.01, 0.02, M).astype(np.float32)
    else:
        x = torch.from_numpy(rng.normal(size=(M, k))).to(t)
    for off in (0.5, 0.0):
        Y = dsq.dsq_wgemm_group(x.cuda(), packed, M, n, k, 4, group, T(scales), bias=T(bias),
                                row_scale=None if rs is None else T(rs), w_offset=off)
        check(Y, x.double().numpy(), codes, scales, group, bias, off, rs)
        again = dsq.dsq_wgemm_group(x.cuda(), packed, M, n, k, 4, group, T(scales), bias=T(bias),
                                    row_scale=None if rs is None else T(rs), w_offset=off)
        assert torch.equal(Y, again)


@pytest.mark.parametrize("t", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("size", [(8, 128, 4096), (20, 300, 1024), (64, 4750, 256)])
def test_bounded_wait_runs_out_and_the_next_call_is_clean(dsq, size, t):
    """A wait that nothing satisfies: the test hook makes the copying warp leave out one stage, so the
    warps that wait for it run into the limit (3 ms here).  The kernel must come back by itself, with
    NaN where a block had that stage (each has a first one; blocks of a cluster and blocks on their
    own), and the same call with the hook off must be right."""
    M, n, k = size
    codes, scales, bias, packed = weights(dsq, n, k, 128)
    rng = np.random.default_rng(k)
    x = rng.integers(-20, 21, (M, k))
    xt = torch.from_numpy(x).to(t).cuda()
    rs = torch.ones(M, device="cuda") if t == torch.int8 else None
    args = (xt, packed, M, n, k, 4, 128, T(scales))
    dsq.dsq_set_wgemm_group_form(2)
    try:
        for skip in (0, 1):
            dsq.dsq_set_wait_limit_ns(3_000_000)
            dsq.dsq_set_test_skip_b_round(skip)
            bad = dsq.dsq_wgemm_group(*args, row_scale=rs)
            torch.cuda.synchronize()       # the kernel came back
            dsq.dsq_set_test_skip_b_round(-1)
            dsq.dsq_set_wait_limit_ns(0)
            if skip == 0:
                assert bad.isnan().all()
            Y = dsq.dsq_wgemm_group(*args, row_scale=rs)
            check(Y, x.astype(np.float64), codes, scales, 128, None, 0.5, None if rs is None else N(rs))
    finally:
        dsq.dsq_set_test_skip_b_round(-1)
        dsq.dsq_set_wait_limit_ns(0)
        dsq.dsq_set_wgemm_group_form(0)


@pytest.mark.parametrize("M", [1, 8, 40])
def test_codes_of_more_than_2_to_the_31_bytes(dsq, form, M):
    n, k, group = 262144 + 40, 16384, 128
    if form == 3 and M > 2:
        pytest.skip("one or two rows")
    packed = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda")
    scales = torch.rand(k // group, n, device="cuda")
    x = torch.randn(M, k, device="cuda").bfloat16()
    Y = dsq.dsq_wgemm_group(x, packed, M, n, k, 4, group, scales)
    for part in (slice(0, 64), slice(262144 - 64, 262144 + 40)):
        codes = N(dsq.dsq_unpack(packed[part].contiguous(), part.stop - part.start, k, 4, True)).astype(np.int64)
        check(Y[:, part], N(x.double()), codes, N(scales[:, part]), group, None, 0.5)


def test_two_streams_and_two_graphs_at_once(dsq):
    """Calls that overlap on the GPU share nothing: kernels of each form beside one another."""
    sizes = [(1, 4096, 4096, torch.bfloat16), (8, 2048, 2048, torch.bfloat16), (64, 1024, 4096, torch.bfloat16),
             (16, 1500, 4096, torch.int8), (40, 4096, 1024, torch.float16)]
    calls = []
    for M, n, k, t in sizes:
        codes, scales, _, packed = weights(dsq, n, k, 128)
        x = torch.randint(-90, 91, (M, k), device="cuda").to(t)
        rs = torch.rand(M, device="cuda") if t == torch.int8 else None
        calls.append((x, packed, M, n, k, T(scales), rs))

    def run(c, out=None):
        return dsq.dsq_wgemm_group(c[0], c[1], c[2], c[3], c[4], 4, 128, c[5], row_scale=c[6], out=out)

    ref = [run(c) for c in calls]
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [[torch.empty_like(r) for r in ref] for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                for j in range(len(calls)):
                    run(calls[(j + i) % len(calls)], outs[i][(j + i) % len(calls)])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, ref))

    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for c, o in zip(calls, outs[i]):
                run(c, o)
        graphs.append(g)
        for o in outs[i]:
            o.zero_()
    torch.cuda.synchronize()
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs[:2] for a, b in zip(o, ref))
