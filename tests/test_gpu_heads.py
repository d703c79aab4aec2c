"""GPU: norms of heads with the position rotation, and their gradients, against the float64 oracle.

Tolerances, in units u = 2^-24 of binary32 (relative error of one rounding):
  rstd      sum of squares: 16 terms a lane and 5 steps of the tree, all positive: 21 u; half of
            that, the mean's three roundings, root and quotient: 16 u
  n         two products more: 18 u
  turn      an angle below pi / 4 rounded: half a unit, sine and cosine 2 units: 4 u absolute; two
            products: 2 u; of |n1| + |n2|: 18 + 6 = 24 u; then half a step of the type
  grad_x    g (6 u of |g1| + |g2|), its sum with n over a head (21 u + 6 u), rstd twice, five products:
            below 90 u of the terms' magnitudes
  grad_w    terms of 23 u, M of them added in any order: (M + 30) u of their magnitudes
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import heads
from gpu_util import N

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# tokens, q heads, k heads, head_dim, rot_dim, axes, interleaved: one of everything, heads in vectors
# and not, one unit a lane and several, parts rotated or nothing, many tokens a tile, many heads
SHAPES = [(1, 1, 1, 2, 2, 1, False), (1, 32, 8, 128, 128, 1, False), (3, 5, 1, 6, 4, 2, True),
          (37, 4, 2, 64, 64, 3, False), (129, 3, 3, 80, 48, 2, True), (77, 2, 1, 72, 72, 1, False),
          (500, 1, 1, 64, 64, 1, True), (19, 40, 8, 128, 64, 1, False), (9, 6, 2, 256, 256, 3, False),
          (5, 3, 1, 512, 128, 1, True), (4, 2, 1, 510, 510, 2, False), (2, 70, 7, 96, 0, 1, False),
          (1, 600, 2, 16, 16, 1, False), (2000, 7, 1, 40, 40, 2, True), (3, 9, 2, 130, 66, 1, False)]


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


def rounding(t, ref):
    f = torch.finfo(t)
    return f.eps / 2 * np.abs(ref) + f.smallest_normal * f.eps


def case(shape, t, seed=0):
    tokens, hq, hk, D, R, axes, _ = shape
    rng = np.random.default_rng(tokens * 1000 + D + seed)
    heads_all = torch.from_numpy(rng.normal(size=(tokens, hq + 2 * hk, D)) * 2).to(t)
    pos = torch.from_numpy(rng.integers(-3, 1 << 20, (axes, tokens)))
    freq = torch.from_numpy(500000.0 ** -(np.arange(R // 2) / max(R // 2, 1))).float()
    axis = torch.from_numpy(rng.integers(0, axes, R // 2)).to(torch.uint8) if axes > 1 else None
    w = [torch.from_numpy(1 + 0.2 * rng.normal(size=D)).float() for _ in range(2)]
    return heads_all, pos, freq, axis, w


def cuda(v):
    return None if v is None else v.cuda()


def check_forward(y, x, w, a, eps, inter, t, norm=True):
    X = x.double().numpy()
    ref = heads.forward(X, w, a, eps, inter, norm)
    n = heads.normed(X, w, eps)[0] if norm else X
    tol = 24 * U * heads.partner(n, a, inter)
    assert y.dtype == t and np.all(np.abs(N(y.double()) - ref) <= tol + rounding(t, ref) * (1 + 2.0 ** -7))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(dsq, shape, t):
    tokens, hq, hk, D, R, axes, inter = shape
    x, pos, freq, axis, w = case(shape, t)
    a = heads.angles(pos.numpy(), freq.numpy(), None if axis is None else axis.numpy())
    g = x.cuda()
    q, k = dsq.dsq_headnorm_fwd(g[:, :hq], g[:, hq:hq + hk], pos.cuda(), freq.cuda(), w[0].cuda(),
                                w[1].cuda(), 1e-6, axis=cuda(axis), interleaved=inter)
    assert q.is_contiguous() and k.is_contiguous()
    check_forward(q, x[:, :hq], w[0].numpy(), a, 1e-6, inter, t)
    check_forward(k, x[:, hq:hq + hk], w[1].numpy(), a, 1e-6, inter, t)
    # the rotation alone, q alone, no weight: one at a time
    q2, none = dsq.dsq_headnorm_fwd(g[:, :hq], None, pos.cuda(), freq.cuda(), eps=1e-6, norm=False,
                                    axis=cuda(axis), interleaved=inter)
    assert none is None
    check_forward(q2, x[:, :hq], None, a, 1e-6, inter, t, norm=False)
    q3, _ = dsq.dsq_headnorm_fwd(g[:, :hq], None, pos.cuda(), freq.cuda(), eps=1e-6, axis=cuda(axis),
                                 interleaved=inter)
    check_forward(q3, x[:, :hq], None, a, 1e-6, inter, t)
    # in place, beside values that stay
    dsq.dsq_headnorm_fwd(g[:, :hq], g[:, hq:hq + hk], pos.cuda(), freq.cuda(), w[0].cuda(), w[1].cuda(),
                         1e-6, axis=cuda(axis), interleaved=inter, out_q=g[:, :hq], out_k=g[:, hq:hq + hk])
    assert torch.equal(g[:, :hq], q) and torch.equal(g[:, hq:hq + hk], k)
    assert torch.equal(g[:, hq + hk:].cpu(), x[:, hq + hk:])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(dsq, shape, t):
    tokens, hq, hk, D, R, axes, inter = shape
    x, pos, freq, axis, w = case(shape, t, seed=1)
    gy = case(shape, t, seed=2)[0]
    a = heads.angles(pos.numpy(), freq.numpy(), None if axis is None else axis.numpy())
    X, G = x.cuda(), gy.cuda()
    parts = (slice(0, hq), slice(hq, hq + hk))
    args = (pos.cuda(), freq.cuda(), w[0].cuda(), w[1].cuda(), 1e-6)
    out = dsq.dsq_headnorm_bwd(*(G[:, p] for p in parts), *(X[:, p] for p in parts), *args,
                               axis=cuda(axis), interleaved=inter)
    for i, p in enumerate(parts):
        gx, gw, mx, mw = heads.backward(gy[:, p].double().numpy(), x[:, p].double().numpy(), w[i].numpy(),
                                        a, 1e-6, inter)
        assert out[i].dtype == t
        assert np.all(np.abs(N(out[i].double()) - gx) <= 90 * U * mx + rounding(t, gx) * (1 + 2.0 ** -7))
        M = tokens * (p.stop - p.start)
        assert np.all(np.abs(N(out[2 + i]) - gw) <= (M + 30) * U * mw)
    again = dsq.dsq_headnorm_bwd(*(G[:, p] for p in parts), *(X[:, p] for p in parts), *args,
                                 axis=cuda(axis), interleaved=inter)
    assert all(torch.equal(u, v) for u, v in zip(out, again))
    # without weights' gradients, without weights, the rotation alone
    gq, gk, none, _ = dsq.dsq_headnorm_bwd(*(G[:, p] for p in parts), *(X[:, p] for p in parts), *args,
                                           axis=cuda(axis), interleaved=inter, want_weight=False)
    assert none is None and torch.equal(gq, out[0]) and torch.equal(gk, out[1])
    gq, none, gw, _ = dsq.dsq_headnorm_bwd(G[:, parts[0]], None, None, None, *args[:2], norm=False,
                                           axis=cuda(axis), interleaved=inter)
    ref, _, mag, _ = heads.backward(gy[:, parts[0]].double().numpy(), None, None, a, 0, inter, norm=False)
    assert none is None and gw is None
    assert np.all(np.abs(N(gq.double()) - ref) <= 6 * U * mag + rounding(t, ref) * (1 + 2.0 ** -7))


def test_gradient_against_differences(dsq):
    """Of sum(y c), by steps of x and of the weight in the oracle's forward pass and in the kernel's gradient."""
    shape = (3, 2, 1, 12, 8, 2, False)
    x, pos, freq, axis, w = case(shape, torch.float32, seed=5)
    c = case(shape, torch.float32, seed=6)[0]
    a = heads.angles(pos.numpy(), freq.numpy(), axis.numpy())
    gq, _, gw, _ = dsq.dsq_headnorm_bwd(c[:, :2].cuda(), None, x[:, :2].cuda(), None, pos.cuda(), freq.cuda(),
                                        w[0].cuda(), None, 1e-6, axis=axis.cuda())
    X, W, Cq, h = x[:, :2].double().numpy(), w[0].double().numpy(), c[:, :2].double().numpy(), 1e-5
    f = lambda X, W: (heads.forward(X, W, a, 1e-6) * Cq).sum()
    for at in np.ndindex(X.shape):
        d = np.zeros_like(X)
        d[at] = h
        # (differences: h^2 of third derivatives and 1e-16 |f| / h, some 1e-8)
        assert abs((f(X + d, W) - f(X - d, W)) / (2 * h) - float(gq[at])) < 2e-5
    for i in range(len(W)):
        d = np.zeros_like(W)
        d[i] = h
        assert abs((f(X, W + d) - f(X, W - d)) / (2 * h) - float(gw[i])) < 2e-5


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 66])
def test_squares_outside_binary32(dsq, t, D):
    """Heads of 1e25 and of 1e-25 (their squares are infinite, or 0), zeros with eps = 0, beside ordinary ones."""
    rng = np.random.default_rng(D)
    x = torch.from_numpy(rng.normal(size=(40, 3, D)))
    x[3, 1] *= 1e25
    x[7, 2] *= 1e-25
    x[11, 0] = 0
    x = x.to(t)
    gy = torch.from_numpy(rng.normal(size=x.shape)).to(t)
    pos, freq, w = torch.arange(40), torch.rand(D // 2), torch.ones(D) + torch.arange(D) / D
    a = heads.angles(pos.numpy(), freq.numpy())
    y, _ = dsq.dsq_headnorm_fwd(x.cuda(), None, pos.cuda(), freq.cuda(), w.cuda(), eps=0.0)
    check_forward(y, x, w.numpy(), a, 0.0, False, t)
    assert not y[11, 0].any()
    # (grad_x of 1e25 would be infinite in the type where rstd is 1e25)
    gy[7, 2] *= 1e-12
    gx, _, gw, _ = dsq.dsq_headnorm_bwd(gy.cuda(), None, x.cuda(), None, pos.cuda(), freq.cuda(), w.cuda(), eps=0.0)
    ref, rw, mx, mw = heads.backward(gy.double().numpy(), x.double().numpy(), w.numpy(), a, 0.0)
    assert np.all(np.abs(N(gx.double()) - ref) <= 90 * U * mx + rounding(t, ref) * (1 + 2.0 ** -7))
    assert np.all(np.abs(N(gw) - rw) <= 150 * U * mw)


@pytest.mark.parametrize("D", [64, 30])
def test_not_a_number_stays_in_its_head(dsq, D):
    x = torch.randn(9, 4, D).bfloat16()
    pos, freq = torch.arange(9).cuda(), torch.rand(D // 2).cuda()
    run = lambda v: dsq.dsq_headnorm_fwd(v.cuda(), None, pos, freq)[0]
    good = run(x)
    bad = x.clone()
    bad[2, 1, 5], bad[4, 3, 7] = float("nan"), float("inf")
    got = run(bad)
    assert got[2, 1].isnan().all() and got[4, 3, [7, (7 + D // 2)]].isnan().all()
    other = got[4, 3].clone()
    other[[7, 7 + D // 2]] = 0
    assert not other.any()                        # finite over infinite
    got[2, 1], got[4, 3] = good[2, 1], good[4, 3]
    assert torch.equal(got, good)


def test_far_positions(dsq):
    """Angles of positions of 2^31 and of 2^40, and of negative ones, are right to binary32's last bits."""
    D = 64
    pos = torch.tensor([0, 1, (1 << 31) + 12345, -(1 << 31), (1 << 40) + 7, -1])
    freq = torch.from_numpy(10000.0 ** -(np.arange(32) / 32)).float()
    x = torch.ones(6, 1, D)
    y, _ = dsq.dsq_headnorm_fwd(x.cuda(), None, pos.cuda(), freq.cuda(), norm=False)
    a = heads.angles(pos.numpy(), freq.numpy())
    # (the product of position and frequency is rounded on both sides: 2^-53 of it, 6e-5 at 2^40)
    tol = 6 * U * 2 + np.abs(np.concatenate([a, a], 1))[:, None] * 2.0 ** -51
    assert np.all(np.abs(N(y.double()) - heads.turn(np.ones((6, 1, D)), a)) <= tol)


def test_angles_beyond_binary64_are_nan(dsq):
    """2^50 - 3 is an angle, 2^50 and the ends of the range are none; the elements that are not turned stay."""
    x = torch.randn(6, 2, 64, device="cuda")
    top = 2 ** 63 - 1
    pos = torch.tensor([2 ** 50 - 3, -(2 ** 50) + 3, 2 ** 50, -(2 ** 50), top, -top - 1])
    freq = torch.ones(16)
    freq[1] = 0.0
    y, _ = dsq.dsq_headnorm_fwd(x, None, pos.cuda(), freq.cuda(), norm=False)
    check_forward(y[:2], x[:2].cpu(), None, heads.angles(pos[:2].numpy(), freq.numpy()), 0.0, False, torch.float32, norm=False)
    turned = torch.ones(64, dtype=torch.bool)
    turned[32:] = False
    turned[[1, 17]] = False
    assert y[2:][..., turned].isnan().all() and torch.equal(y[2:][..., ~turned], x[2:][..., ~turned])


def test_axis_out_of_range_is_nan(dsq):
    x, freq = torch.ones(2, 3, 32), torch.ones(16)
    axis = torch.zeros(16, dtype=torch.uint8)
    axis[3] = 2
    y, _ = dsq.dsq_headnorm_fwd(x.cuda(), None, torch.zeros(2, 2, dtype=torch.long).cuda(), freq.cuda(),
                                axis=axis.cuda())
    assert y.isnan().sum() == 2 * 3 * 2 and y[..., [3, 19]].isnan().all()


@pytest.mark.parametrize("t", TYPES)
def test_layouts(dsq, t):
    """Heads before tokens, odd addresses, an expanded input and gradient: the values of dense ones."""
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.normal(size=(21, 4, 64))).to(t).cuda()
    g = torch.from_numpy(rng.normal(size=(21, 4, 64))).to(t).cuda()
    pos, freq, w = torch.arange(21).cuda(), torch.rand(32).cuda(), torch.rand(64).cuda()
    f = lambda v, **kw: dsq.dsq_headnorm_fwd(v, None, pos, freq, w, **kw)[0]
    b = lambda v, h: dsq.dsq_headnorm_bwd(v, None, h, None, pos, freq, w)
    ref, refg = f(x), b(g, x)
    turned = x.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.zeros_like(turned.transpose(0, 1)).transpose(0, 1)
    assert torch.equal(f(turned), ref) and f(turned, out_q=out) is out and torch.equal(out, ref)
    store = torch.zeros(21 * 4 * 64 + 1, dtype=t, device="cuda")
    odd = store[1:].view(21, 4, 64)
    odd.copy_(x)
    # (element by element the sums have another order: a rounding apart)
    assert torch.allclose(f(odd).double(), ref.double(), rtol=4 * torch.finfo(t).eps, atol=1e-6)
    wide = torch.zeros(21, 4, 67, dtype=t, device="cuda")
    wide[..., :64] = x
    assert torch.allclose(f(wide[..., :64]).double(), ref.double(), rtol=4 * torch.finfo(t).eps, atol=1e-6)
    one = x[:, :1].expand(21, 4, 64)
    assert torch.equal(f(one), f(one.contiguous()))
    ge = g[:1, :1].expand(21, 4, 64)
    for u, v in zip(b(ge, x), b(ge.contiguous(), x)):
        assert u is None and v is None or torch.equal(u, v)


def test_streams_graphs_and_workspaces(dsq):
    """Two captured backward passes with a workspace each, replayed on two streams with changed inputs."""
    sets = []
    for seed in range(2):
        x = torch.randn(300, 6, 128, device="cuda").bfloat16()
        g = torch.randn(300, 6, 128, device="cuda").bfloat16()
        sets.append((x, g, torch.empty(dsq.dsq_headnorm_bwd_workspace_bytes(128), dtype=torch.uint8, device="cuda")))
    pos, freq, w = torch.arange(300).cuda(), torch.rand(64).cuda(), torch.rand(128).cuda()
    call = lambda s: dsq.dsq_headnorm_bwd(s[1][:, :4], s[1][:, 4:], s[0][:, :4], s[0][:, 4:], pos, freq, w, w, ws=s[2])
    graphs = []
    for s in sets:
        call(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call(s)
        graphs.append((graph, out))
    for s in sets:
        s[0].copy_(torch.randn(300, 6, 128))
    want = [[v.clone() for v in call(s)] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for st, (graph, _) in zip(streams, graphs):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for (_, out), ref in zip(graphs, want):
        assert all(torch.equal(u, v) for u, v in zip(out, ref))
