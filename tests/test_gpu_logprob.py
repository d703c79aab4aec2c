"""GPU: log probabilities of tokens, entropy, alternatives and the logits' gradient against the float64 oracle.

Tolerances, in units u = 2^-24 of binary32:
  s        a thread adds V / 1024 terms in each of two sums and rescales; 30 steps of trees and joins: A = V / 1024 +
           40 additions of positive terms; a term: 2^x 4 u, its exponent four roundings of |m - z|, which weighted
           sum to 4 u first (oracle: first, second moments of m - z)
  logp     that of s, log 2 u of itself, the difference and product of z_t: 4 u of |z_t - m|
  lse      the same and two roundings of itself and of m
  entropy  t's terms are |m - z| times those of s
  grad     p: 2^x 4 u, exponent 3 u |log p|; a product, two fused sums; then half a step of the type
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import logprob
from gpu_util import N

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF = float("inf")


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


def logits(M, V, t, seed=0, spread=2.5):
    rng = np.random.default_rng(M * 7919 + V + seed)
    x = torch.from_numpy(rng.normal(size=(M, V)) * spread).to(t)
    return x, torch.from_numpy(rng.integers(0, V, M))


def check(dsq, x, targets, scale=1.0, top=0, device_x=None):
    """All outputs of a forward pass; returns them."""
    V = x.shape[1]
    g = x.cuda() if device_x is None else device_x
    logp, entropy, lse, ids, top_logp = dsq.dsq_logprob_fwd(g, targets.cuda(), scale=scale, top=top)
    X = x.double().numpy()
    r = logprob.forward(X, targets.numpy(), np.float32(scale))
    A = V / 1024 + 40
    s = A + 4 + 4 * r["first"]
    z = np.where(np.isfinite(X), X, 0.0) * scale
    m = np.abs(z.max(1))

    def near(got, want, tol):
        got = N(got).astype(np.float64)
        same = np.isinf(want) | np.isnan(want)
        assert np.array_equal(got[same], want[same], equal_nan=True)
        off = np.abs(np.where(same, 0.0, got) - np.where(same, 0.0, want))
        assert np.all(off <= tol * U + 1e-30), (off / U - tol).max()

    finite = lambda v: np.where(np.isfinite(v), np.abs(v), 0.0)
    near(logp, r["logp"], s + 8 * finite(r["log_s"]) + 8 * finite(r["logp"]) + 2)
    near(lse, r["lse"], s + 4 * finite(r["lse"]) + 4 * m + 4 * r["log_s"] + 2)
    near(entropy, r["entropy"], (s + 8) * (1 + r["first"]) + 8 * r["second"] + 8 * r["log_s"])
    if top:
        want = logprob.largest(X, top)
        assert ids.dtype == torch.int64 and np.array_equal(N(ids), want)
        lp = np.take_along_axis(r["lp"], want, 1)
        near(top_logp, lp, (s + 8 * r["log_s"] + 2)[:, None] + 8 * finite(lp))
    else:
        assert ids is None and top_logp is None
    return logp, entropy, lse, ids, top_logp


# one element, less than a vector, a block's one turn and one more, all cluster sizes, many rows of one block
SHAPES = [(1, 1), (3, 5), (2, 8), (5, 33), (4, 513), (300, 1000), (9, 4097), (2, 16384), (1, 50261), (3, 65537),
          (1, 128000), (80, 40000), (40, 20001), (333, 8191), (150, 33000)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(dsq, shape, t):
    M, V = shape
    x, targets = logits(M, V, t)
    for scale, top in ((1.0, min(V, 20)), (0.7, 0), (1.5, min(V, 1)), (1.0, min(V, 32))):
        check(dsq, x, targets, scale, top)


@pytest.mark.parametrize("t", TYPES)
def test_masks(dsq, t):
    """Rows that keep one element, fewer than the alternatives, a tenth; all masked; the lowest value as a mask."""
    V = 40001
    x, targets = logits(8, V, t, seed=1)
    low = torch.finfo(t).min
    for row, keep, mask in ((0, 1, -INF), (1, 5, -INF), (2, V // 10, -INF), (3, 0, -INF), (4, 5, low), (5, 0, low)):
        kept = torch.randperm(V, generator=torch.Generator().manual_seed(row))[:keep]
        gone = torch.ones(V, dtype=torch.bool)
        gone[kept] = False
        x[row, gone] = mask
        if keep:
            targets[row] = kept[0]
    targets[6], targets[7] = -100, V
    logp, entropy, lse, ids, _ = check(dsq, x, targets, 1.0, 20)
    assert logp[3] == -INF and entropy[3] == 0 and lse[3] == -INF
    assert N(ids[3]).tolist() == list(range(20)) and logp[6] == 0 and logp[7].isnan()
    check(dsq, x[:1], targets[:1], 1.0, 32)
    check(dsq, x[3:4], targets[3:4], 2.0, 32)
    # a target that is masked
    targets[1] = int((x[1] == -INF).nonzero()[0])
    assert check(dsq, x, targets, 1.0, 0)[0][1] == -INF


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M", [1, 40, 400])
def test_ties(dsq, t, M):
    """Rows of few different values, of one value, with zeros of both signs: the lowest index first."""
    rng = np.random.default_rng(M)
    for V in (100, 5003, 20480):
        for values in ([1.0], [0.0, -0.0], [2.0, 1.0, 1.0, 1.0], list(range(7))):
            x = torch.from_numpy(rng.choice(values, (M, V))).to(t)
            check(dsq, x, torch.zeros(M, dtype=torch.long), 1.0, 20)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [1, 200, 300])
def test_large_elements_with_the_same_threads(dsq, t, M):
    """More candidates than a block has room for: a block's stride of large elements, in sorted order."""
    V = 128000
    x = torch.full((M, V), -4.0)
    vec = 16 // t.itemsize
    # all elements of the vectors of the first few threads, whatever block a row is cut into
    v = torch.arange(V) // vec
    part = V // vec // 8
    for period in (512 if M < 296 else 256,):
        here = ((v - 0) % period < 70) | ((v % part) % period < 70)
        x[:, here] = (torch.arange(int(here.sum())) % 977).float() * 0.0625
    check(dsq, x.to(t), torch.zeros(M, dtype=torch.long), 1.0, 32)


def test_not_a_number_and_infinity_stay_in_their_row(dsq):
    x, targets = logits(30, 9001, torch.bfloat16, seed=2)
    good = [v.clone() for v in dsq.dsq_logprob_fwd(x.cuda(), targets.cuda(), top=8)]
    bad = x.clone()
    bad[3, 17], bad[5, 4000], bad[9] = float("nan"), INF, float("nan")
    got = dsq.dsq_logprob_fwd(bad.cuda(), targets.cuda(), top=8)
    for row in (3, 5, 9):
        for i in (0, 1, 2, 4):
            assert got[i][row].isnan().all()
    assert torch.equal(got[3][3], good[3][3]) or (good[3][3] == 17).any()
    assert got[3][5, 0] == 4000 and N(got[3][9]).tolist() == list(range(8))
    keep = [i for i in range(30) if i not in (3, 5, 9)]
    for a, b in zip(got, good):
        assert torch.equal(a[keep], b[keep])


def test_extreme_values(dsq):
    """fp32 logits up to its ends, and peaks whose probability is 1."""
    x, targets = logits(6, 3001, torch.float32, seed=3)
    x[0] *= 1e30
    x[1, 5], targets[1] = 200.0, 5
    x[2] += 1e6
    x[3] -= 1e6
    x[4] *= 1e-30
    check(dsq, x, targets, 1.0, 5)


@pytest.mark.parametrize("t", TYPES)
def test_layouts(dsq, t):
    """Rows further apart than they are long, and at odd addresses: the values of dense ones."""
    for V in (1000, 1003):
        wide = torch.zeros(37, V + 9, dtype=t)
        x, targets = logits(37, V, t, seed=4)
        wide[:, 3:3 + V] = x
        g = wide.cuda()
        out = check(dsq, x, targets, 1.0, 7, device_x=g[:, 3:3 + V])
        grad = dsq.dsq_logprob_bwd(g[:, 3:3 + V], targets.cuda(), out[2], torch.ones(37).cuda())
        dense = dsq.dsq_logprob_bwd(x.cuda(), targets.cuda(), out[2], torch.ones(37).cuda())
        assert torch.equal(grad, dense)
        into = torch.full((37, V + 5), 7.0, dtype=t, device="cuda")
        got = dsq.dsq_logprob_bwd(x.cuda(), targets.cuda(), out[2], torch.ones(37).cuda(), out=into[:, 1:1 + V])
        assert torch.equal(got, dense) and (into[:, 0] == 7).all() and (into[:, 1 + V:] == 7).all()
        dsq.dsq_logprob_bwd(g[:, 3:3 + V], targets.cuda(), out[2], torch.ones(37).cuda(), out=g[:, 3:3 + V])
        assert torch.equal(g[:, 3:3 + V], dense) and (g[:, :3] == 0).all() and (g[:, 3 + V:] == 0).all()


def rounding(t, ref):
    f = torch.finfo(t)
    return f.eps / 2 * np.abs(ref) + f.smallest_normal * f.eps


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(dsq, shape, t):
    M, V = shape
    x, targets = logits(M, V, t, seed=5)
    rng = np.random.default_rng(V)
    g = torch.from_numpy(rng.normal(size=M)).float()
    ge = torch.from_numpy(rng.normal(size=M)).float()
    if M > 2:
        targets[1], g[2], ge[2] = -1, 0, 0
    scale = 0.8
    r = logprob.forward(x.double().numpy(), targets.numpy(), np.float32(scale))
    lse, h = torch.from_numpy(r["lse"]).float(), torch.from_numpy(r["entropy"]).float()
    for a, b in ((g, None), (None, ge), (g, ge)):
        got = dsq.dsq_logprob_bwd(x.cuda(), targets.cuda(), lse.cuda(), None if a is None else a.cuda(),
                                  None if b is None else h.cuda(), None if b is None else b.cuda(), scale)
        ref, mag, at, l = logprob.backward(x.double().numpy(), targets.numpy(), lse.numpy(),
                                           None if a is None else a.numpy(), None if b is None else h.numpy(),
                                           None if b is None else b.numpy(), np.float32(scale))
        tol = (12 + 6 * l) * U * mag + 4 * U * at
        assert got.dtype == t
        assert np.all(np.abs(N(got.double()) - ref) <= tol + rounding(t, ref) * (1 + 2.0 ** -7) + 1e-37)


def test_backward_of_masked_and_other_rows(dsq):
    x, targets = logits(7, 5001, torch.float32, seed=6)
    x[0] = -INF
    x[1, 100:] = -INF
    targets[1] = 200                              # masked: no probability
    x[2, 5], x[3] = float("nan"), float("nan")
    targets[4], targets[5] = -100, 5001
    g = torch.ones(7)
    g[3] = 0
    logp, h, lse, _, _ = dsq.dsq_logprob_fwd(x.cuda(), targets.cuda())
    grad = dsq.dsq_logprob_bwd(x.cuda(), targets.cuda(), lse, g.cuda())
    assert not grad[0].any() and not grad[3].any() and not grad[4].any()
    assert grad[2].isnan().all() and grad[5].isnan().all() and grad[1, 200] == 1 and grad[6].isfinite().all()
    assert abs(float(grad[6].double().sum())) < 1e-5 and not grad[1, 101:200].any()
    both = dsq.dsq_logprob_bwd(x.cuda(), targets.cuda(), lse, g.cuda(), h, torch.ones(7).cuda())
    assert not both[0].any() and both[1].isfinite().all() and both[4].any()


def test_gradient_against_differences(dsq):
    """Of sum(a logp + b entropy), by steps of each logit in the oracle's forward pass."""
    x, targets = logits(3, 11, torch.float32, seed=7)
    a, b, scale, step = torch.tensor([0.5, -1.0, 2.0]), torch.tensor([1.0, 0.3, -0.7]), 1.3, 1e-5
    logp, h, lse, _, _ = dsq.dsq_logprob_fwd(x.cuda(), targets.cuda(), scale)
    grad = dsq.dsq_logprob_bwd(x.cuda(), targets.cuda(), lse, a.cuda(), h, b.cuda(), scale)

    def loss(X):
        r = logprob.forward(X, targets.numpy(), np.float32(scale))
        return (a.numpy() * r["logp"] + b.numpy() * r["entropy"]).sum()

    X = x.double().numpy()
    for at in np.ndindex(X.shape):
        d = np.zeros_like(X)
        d[at] = step
        # (differences: step^2 of third derivatives and 1e-16 / step, some 1e-10; gradients of a few units)
        assert abs((loss(X + d) - loss(X - d)) / (2 * step) - float(grad[at])) < 1e-5


def test_far_rows(dsq):
    """Offsets beyond 2^31 elements."""
    V = 1 << 22
    x = torch.zeros(520, V, dtype=torch.bfloat16, device="cuda")
    targets = torch.arange(520, device="cuda")
    x[519, 519], x[515, 77] = 30.0, 20.0
    logp, _, lse, ids, _ = dsq.dsq_logprob_fwd(x, targets, top=1)
    assert ids[519, 0] == 519 and ids[515, 0] == 77 and ids[518, 0] == 0
    assert abs(float(logp[519])) < 1e-6 and abs(float(lse[518]) - np.log(V)) < 1e-4
    g = torch.zeros(520, device="cuda")
    g[519] = g[518] = 1
    dsq.dsq_logprob_bwd(x, targets, lse, g, out=x)
    assert float(x[518, 518]) == 1 and abs(float(x[518, 0]) * V + 1) < 1e-2 and not x[:518].any()


def test_streams_and_graphs(dsq):
    """Captured once, replayed with other logits; the same bits every time."""
    x = logits(50, 30001, torch.bfloat16, seed=8)[0].cuda()
    targets = torch.arange(50, device="cuda")
    g = torch.ones(50, device="cuda")

    def call():
        logp, h, lse, ids, tl = dsq.dsq_logprob_fwd(x, targets, top=20)
        return logp, h, lse, ids, tl, dsq.dsq_logprob_bwd(x, targets, lse, g, h, g)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    x.copy_(logits(50, 30001, torch.bfloat16, seed=9)[0])
    want = call()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(5):
            graph.replay()
        again = call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(out, want, again))
