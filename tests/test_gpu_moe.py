"""GPU: the router's choice and the layer of experts on 4-bit weights, against the float64 oracle.

Tolerances, in units u = 2^-24 of binary32, of the magnitudes of the terms:
  first sums    products are exact; a tensor-core instruction adds 16 of them to its sums within 8 u of their
                magnitudes, eight of which make up to 128 codes: 64 u; K / 32 fused sums with scales, 8 warps' sums:
                eps_in = (64 + K / 32 + 12) u
  mid           activation and product 16 u: eps_mid = 20 u; on 16 bits half a step of fp16, 2^-11, more where y is bf16,
                else of two such numbers, 2^-22
  digits        x and mid are kept to half a step, 2^-31 of the power of two above the largest of 128 elements:
                2^-30 of the largest of a row at most (and on 16 bits half of 2^-24 below 2^14: less)
  second sums   the same of I codes, k slots' sums and weights, 8 warps of 8 blocks: eps_out = (64 + I / 32 +
                2 k + 20) u
  y             the residual's addition u, then half a step of the type
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import moe
from gpu_util import N

U = 2.0 ** -24
INF = float("inf")


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


class Layer:
    """Random codes, scales and tokens of one layer, on the host and the GPU."""

    def __init__(self, dsq, T, H, I, E, k, group, t=torch.bfloat16, seed=0):
        rng = np.random.default_rng(T * 131 + H + I + seed)
        self.E, self.I, self.group = E, I, group
        self.c_in = rng.integers(-8, 8, (E * 2 * I, H)).astype(np.int8)
        self.c_out = rng.integers(-8, 8, (E * H, I)).astype(np.int8)
        self.s_in = (rng.uniform(0.5, 1.5, (-(-H // group), E * 2 * I)) * 0.1 / np.sqrt(H)).astype(np.float32)
        self.s_out = (rng.uniform(0.5, 1.5, (-(-I // group), E * H)) * 0.1 / np.sqrt(I)).astype(np.float32)
        cuda = lambda a: torch.from_numpy(a).cuda()
        self.weights = [dsq.dsq_pack_codes(cuda(self.c_in), 4), cuda(self.s_in),
                        dsq.dsq_pack_codes(cuda(self.c_out), 4), cuda(self.s_out), E, I, 4, group]
        self.x = torch.from_numpy(rng.normal(size=(T, H)) * 1.5).to(t)
        self.residual = torch.from_numpy(rng.normal(size=(T, H))).to(t)
        self.ids = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
        self.w = rng.uniform(0, 1, (T, k)).astype(np.float32)

    def run(self, dsq, **kw):
        kw.setdefault("residual", self.residual.cuda())
        return dsq.dsq_moe_group(self.x.cuda(), torch.from_numpy(self.ids).cuda(), torch.from_numpy(self.w).cuda(),
                                 *self.weights, **kw)

    def check(self, y, kind="silu", w_offset=0.5, residual=True):
        H, I, k = self.x.shape[1], self.I, self.ids.shape[1]
        # (a pass takes 64 tokens: the first ones say more than the last few)
        few = min(len(self.x), 64)
        narrow = w_offset == 0.5 and (few <= 4 or 2 * few * k <= 3 * self.E) and len(self.x) <= 64
        eps_mid = 20 * U + (0 if narrow else 2.0 ** -11 if y.dtype == torch.bfloat16 else 2.0 ** -22)
        ref, bound = moe.layer(self.x.double().numpy(), self.ids, self.w, self.c_in, self.s_in, self.c_out, self.s_out,
                               self.E, I, self.group, kind, w_offset, self.residual.double().numpy() if residual else None,
                               eps_in=(76 + H / 32) * U, eps_out=(84 + I / 32 + 2 * k) * U, eps_mid=eps_mid, digits=2.0 ** -30)
        f = torch.finfo(y.dtype)
        tol = bound + U * np.abs(ref) + (f.eps / 2 * (np.abs(ref) + bound) + f.smallest_normal * f.eps)
        err = np.abs(N(y.double()) - ref)
        assert np.all(err <= tol), (err / tol).max()


# T, H, I, E, k, group
SHAPES = [(1, 8, 1, 1, 1, 32), (1, 64, 32, 4, 2, 32), (3, 200, 77, 5, 3, 32), (1, 2048, 256, 8, 8, 128),
          (8, 520, 130, 9, 2, 64), (9, 512, 128, 9, 2, 128), (16, 1000, 300, 4, 4, 96), (33, 264, 96, 3, 1, 32),
          (64, 256, 160, 2, 2, 64), (64, 640, 64, 40, 6, 128), (65, 128, 64, 7, 2, 4096), (140, 96, 33, 6, 3, 32),
          (2, 4104, 1030, 3, 2, 128), (5, 136, 2056, 4, 2, 256), (20, 64, 48, 300, 32, 32)]


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", SHAPES)
def test_layer(dsq, shape, t):
    a = Layer(dsq, *shape, t=t)
    y = a.run(dsq)
    assert y.dtype == t and y.shape == a.x.shape
    a.check(y)
    assert torch.equal(y, a.run(dsq))
    f = a.run(dsq, residual=None, out_dtype=torch.float32)
    a.check(f, residual=False)


@pytest.mark.parametrize("T", [1, 6, 24])
def test_forms(dsq, T):
    """Both activations, both grids, all output types, in place, a workspace of the caller's."""
    a = Layer(dsq, T, 264, 100, 6, 3, 32)
    for kind in ("silu", "gelu_tanh"):
        for off in (0.5, 0.0):
            a.check(a.run(dsq, activation=kind, w_offset=off), kind, off)
    for t in (torch.float32, torch.float16):
        a.check(a.run(dsq, residual=None, out_dtype=t), residual=False)
    ws = torch.full((dsq.dsq_moe_workspace_bytes(T, 264, 100, 3),), 255, dtype=torch.uint8, device="cuda")
    y = a.residual.cuda()
    assert a.run(dsq, residual=y, out=y, ws=ws) is y
    assert torch.equal(y, a.run(dsq))


@pytest.mark.parametrize("T", [4, 40])
def test_choices(dsq, T):
    """Ids that are none, tokens without any, an expert twice for a token, all tokens on one expert."""
    a = Layer(dsq, T, 128, 96, 5, 4, 32, seed=1)
    a.ids[0] = [-1, 7, 5, -2]
    a.ids[1] = [2, 2, 2, 2]
    a.ids[2] = [0, -1, 0, 3]
    a.check(a.run(dsq))
    a.ids[:] = 3
    a.check(a.run(dsq))
    a.ids[:] = -1
    assert torch.equal(a.run(dsq), a.residual.cuda())
    assert not a.run(dsq, residual=None).any()


@pytest.mark.parametrize("T", [3, 20])
def test_not_a_number_and_infinity_stay_with_their_token(dsq, T):
    a = Layer(dsq, T, 256, 64, 4, 2, 64, seed=2)
    good = a.run(dsq)
    a.x[1, 5] = float("nan")
    a.x[2, 7] = INF
    got = a.run(dsq)
    assert got[1].isnan().all() and not got[2].isfinite().any()
    got[1:3] = good[1:3]
    assert torch.equal(got, good)
    # weights: 0, negative, infinite
    a = Layer(dsq, T, 256, 64, 4, 2, 64, seed=2)
    a.w[0], a.w[1, 0] = 0.0, -2.0
    a.check(a.run(dsq))
    a.w[2] = INF
    got = a.run(dsq)
    assert not got[2].isfinite().any() and got[[0, 1]].isfinite().all()


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("off", [0.5, 0.0])
@pytest.mark.parametrize("T", [1, 7, 30])
def test_outliers(dsq, T, t, off):
    """Elements far above the rest of their row; on the grid with a 0, behind weights that make them vanish."""
    a = Layer(dsq, T, 512, 96, 3, 2, 64, t=t, seed=6)
    big = 6e4 if t == torch.float16 else 1e30
    a.x[:, 5::128] = big
    a.x[:, 77] = 2.0 ** -20
    if off == 0.0:
        a.c_in[:, 5::128] = 0
        a.weights[0] = dsq.dsq_pack_codes(torch.from_numpy(a.c_in).cuda(), 4)
        y = a.run(dsq, w_offset=off, residual=None, out_dtype=torch.float32)
        b = Layer.__new__(Layer)
        b.__dict__.update(a.__dict__)
        b.x = a.x.clone()
        b.x[:, 5::128] = 0
        b.check(y, w_offset=off, residual=False)       # what is left is as exact as ever
    elif t == torch.float16:
        a.s_in *= 1e-3
        a.weights[1] = torch.from_numpy(a.s_in).cuda()
        a.check(a.run(dsq, out_dtype=torch.float32, residual=None), residual=False)


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("off", [0.5, 0.0])
@pytest.mark.parametrize("T", [3, 30])
def test_powers_of_two(dsq, T, off, t):
    """Rows far from 1 (of fp16 and the smallest of bf16: with elements below the type's normal numbers), and one of zeros."""
    for e in (-126, -60, 100) if t == torch.bfloat16 else (-14, -8, 10):
        a = Layer(dsq, T, 328, 64, 3, 2, 64, t=t, seed=7)
        a.x = (a.x.double() * 2.0 ** e).to(t)
        a.x[2] = 0
        a.s_in = (a.s_in * 2.0 ** -e).astype(np.float32)
        a.weights[1] = torch.from_numpy(a.s_in).cuda()
        a.check(a.run(dsq, w_offset=off, residual=None, out_dtype=torch.float32), w_offset=off, residual=False)


@pytest.mark.parametrize("T", [3, 30])
def test_outliers_of_bf16(dsq, T):
    """One element of a row 2^40 above the others: those still count to 2^-30 of it."""
    a = Layer(dsq, T, 512, 96, 3, 2, 64, seed=8)
    a.x[:, 5] = 2.0 ** 40
    a.s_in *= np.float32(2.0 ** -36)
    a.weights[1] = torch.from_numpy(a.s_in).cuda()
    a.check(a.run(dsq, out_dtype=torch.float32, residual=None), residual=False)


def test_large_values(dsq):
    """mid beyond fp16's range, x and outputs of fp16."""
    a = Layer(dsq, 4, 128, 64, 3, 2, 32, t=torch.float16, seed=3)
    a.s_in *= 3000
    a.s_out /= 1e6
    a.weights[1], a.weights[3] = torch.from_numpy(a.s_in).cuda(), torch.from_numpy(a.s_out).cuda()
    a.check(a.run(dsq))


@pytest.mark.parametrize("T,off", [(1, 0.5), (8, 0.5), (8, 0.0), (40, 0.5)])
def test_ids_and_weights_written_right_ahead(dsq, T, off):
    """A step that writes the router's logits, codes and scales before each call: nothing of the step before is used."""
    a, b = (Layer(dsq, T, 256, 128, 6, 2, 64, seed=s) for s in (9, 10))
    g = torch.Generator().manual_seed(T)
    logits = [torch.randn(T, 6, generator=g).cuda() for _ in range(2)]
    x = [v.x.cuda() for v in (a, b)]
    expected = []
    for i, v in enumerate((a, b)):
        ids, w = dsq.dsq_moe_route(logits[i], 2)
        expected.append(dsq.dsq_moe_group(x[i], ids, w, *v.weights, w_offset=off))
        torch.cuda.synchronize()
    now = [v.clone() for v in a.weights[:4]]
    z, X = logits[0].clone(), x[0].clone()
    ws = torch.empty(dsq.dsq_moe_workspace_bytes(T, 256, 128, 2), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(x[0]) for _ in range(8)]

    def steps():
        for i in range(8):
            for to, of in zip(now, (a, b)[i % 2].weights):
                to.copy_(of)
            z.copy_(logits[i % 2])
            X.copy_(x[i % 2])
            ids, w = dsq.dsq_moe_route(z, 2)
            dsq.dsq_moe_group(X, ids, w, *now, *a.weights[4:], w_offset=off, out=out[i], ws=ws)

    steps()
    assert all(torch.equal(o, expected[i % 2]) for i, o in enumerate(out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps()
    for o in out:
        o.zero_()
    graph.replay()
    assert all(torch.equal(o, expected[i % 2]) for i, o in enumerate(out))


@pytest.mark.parametrize("E", [1, 5, 64, 65, 256, 300, 2000])
@pytest.mark.parametrize("renormalise", [True, False])
def test_route(dsq, E, renormalise):
    rng = np.random.default_rng(E)
    z = torch.from_numpy(rng.normal(size=(37, E)) * 3).float()
    z[1] = 0.0
    z[2] = torch.from_numpy(rng.integers(0, 2, E)).float() - 0.0
    z[3] = -INF
    z[4, : E - 1] = -INF
    z[5] = torch.where(torch.rand(E) < 0.5, 0.0, -0.0)
    z[6] = 1e38
    for k in sorted({1, min(E, 8), min(E, 32)}):
        ids, w = dsq.dsq_moe_route(z.cuda(), k, renormalise)
        want, ref = moe.route(z.numpy(), k, renormalise)
        assert ids.dtype == torch.int32 and np.array_equal(N(ids), want)
        # expf 2 u and its argument's rounding u |z - m|, sums of E terms, the quotient
        Z = z.double().numpy()
        far = np.where(np.isinf(Z), 0.0, Z.max(1, keepdims=True).clip(-1e39) - Z).clip(0, 100).max(1)
        tol = (8 + E / 32 + 2 * far) * U
        assert np.all(np.abs(N(w) - ref) <= tol[:, None] * ref + 1e-37)
        assert not w[3].any()


def test_route_of_not_a_number(dsq):
    z = torch.randn(3, 20)
    z[1, 4] = float("nan")
    ids, w = dsq.dsq_moe_route(z.cuda(), 19)
    assert (ids[1] != 4).all() and w[[0, 2]].isfinite().all()
    assert (dsq.dsq_moe_route(z.cuda(), 20)[0][1, 19] == 4) and dsq.dsq_moe_route(z.cuda(), 20)[1][1].isnan().all()


def test_a_decoder_step(dsq):
    """Norm, router, experts, norm, vocabulary and log probabilities one after the other, as a decoder runs them;
    captured into a graph and replayed with another token."""
    T, H, I, E, k, V = 3, 512, 128, 8, 2, 1000
    a = Layer(dsq, T, H, I, E, k, 64)
    gen = torch.Generator().manual_seed(0)
    rand = lambda *s: torch.randn(*s, generator=gen)
    w = (1 + 0.1 * rand(H)).cuda()
    router = dsq.dsq_quantize_groups((rand(E, H) / 20).cuda(), 4, 64)
    head = dsq.dsq_quantize_groups((rand(V, H) / 10).cuda(), 4, 64)
    qk = dsq.dsq_quantize_groups((rand(6 * 64, H) / 20).cuda(), 4, 64)
    x, res = a.x.cuda(), a.residual.cuda()
    pos, freq, targets = torch.arange(T).cuda(), torch.rand(32, generator=gen).cuda(), torch.tensor([1, 2, 3]).cuda()

    def step():
        h, y, _, _, _ = dsq.dsq_rmsnorm_fwd(x, w, 1e-5, residual=res)
        both = dsq.dsq_wgemm_group(y, qk[0], T, 6 * 64, H, 4, 64, qk[1], out_dtype=torch.bfloat16).view(T, 6, 64)
        q, kk = dsq.dsq_headnorm_fwd(both[:, :4], both[:, 4:], pos, freq)
        z = dsq.dsq_wgemm_group(y, router[0], T, E, H, 4, 64, router[1])
        ids, weights = dsq.dsq_moe_route(z, k)
        out = dsq.dsq_moe_group(y, ids, weights, *a.weights, residual=h)
        _, n, _, _, _ = dsq.dsq_rmsnorm_fwd(out, w, 1e-5)
        logits = dsq.dsq_wgemm_group(n, head[0], T, V, H, 4, 64, head[1])
        return (y, z, ids, weights, h, out, logits, q, kk) + dsq.dsq_logprob_fwd(logits, targets, top=5)

    def check(r):
        y, z, ids, weights, h, out, logits, q, kk, logp, entropy, lse, top_ids, top_logp = r
        want, wref = moe.route(N(z), k)
        assert np.array_equal(N(ids), want) and np.allclose(N(weights), wref, rtol=1e-6)
        b = Layer.__new__(Layer)
        b.__dict__.update(a.__dict__)
        b.x, b.residual, b.ids, b.w = y.cpu(), h.cpu(), N(ids), N(weights)
        b.check(out)
        lp = torch.log_softmax(logits.double(), 1)
        assert torch.allclose(logp.double(), lp[torch.arange(T), targets], rtol=0, atol=1e-5)
        assert torch.equal(top_ids, lp.topk(5).indices) and q.isfinite().all() and kk.isfinite().all()

    check(step())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    x.copy_(torch.randn(T, H))
    graph.replay()
    torch.cuda.synchronize()
    check(out)
    assert all(torch.equal(u, v) for u, v in zip(out, step()))


def test_two_graphs_and_streams(dsq):
    """Layers of other sizes with a workspace each, at the same time."""
    sets = [Layer(dsq, 5, 512, 200, 6, 2, 64, seed=4), Layer(dsq, 40, 256, 300, 10, 3, 32, seed=5)]
    calls, graphs = [], []
    for a in sets:
        args = [a.x.cuda(), torch.from_numpy(a.ids).cuda(), torch.from_numpy(a.w).cuda()]
        ws = torch.empty(dsq.dsq_moe_workspace_bytes(*a.x.shape, a.I, a.ids.shape[1]), dtype=torch.uint8, device="cuda")
        call = lambda a=a, args=args, ws=ws: dsq.dsq_moe_group(*args, *a.weights, ws=ws)
        want = call().clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = call()
        calls.append((want, y, call))              # (a graph does not hold its inputs)
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(30):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for want, y, _ in calls:
        assert torch.equal(want, y)
