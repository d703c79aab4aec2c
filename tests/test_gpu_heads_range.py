"""GPU: heads that are done again in binary64, in every form of the kernels: teams of a warp that share a token's heads, heads of k,
heads beyond the 32nd of a part, neighbours paired, in place; and gradients whose products leave binary32's range.
Tolerances as in test_gpu_heads.py."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import heads
from gpu_util import N
from test_gpu_heads import U, check_forward, rounding


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


def near(got, ref, tol, t):
    err = np.abs(N(got.double()) - ref)
    assert np.all(err <= tol + rounding(t, ref) * (1 + 2.0 ** -7)), (err / (tol + 1e-300)).max()


# tokens, heads of q and k, head_dim, rotated
SHAPES = [(5, 32, 8, 128, 128), (5, 32, 8, 64, 64), (3, 70, 7, 64, 64), (3, 70, 7, 128, 128), (4, 33, 9, 80, 48),
          (4, 40, 34, 66, 66), (2900, 70, 7, 64, 64)]


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
def test_heads_done_again(dsq, shape, t, inter):
    tokens, hq, hk, D, R = shape
    rng = np.random.default_rng(hq + D)
    x = rng.normal(size=(tokens, hq + hk, D))
    g = rng.normal(size=x.shape)
    # of q, its last, past the 32nd, of k, its last; and those of the last token
    for i, h in enumerate((1, 31, 32, hq - 1, hq, hq + hk - 1)):
        x[i % tokens, h] *= 1e25 if i % 2 else 1e-25
        g[i % tokens, h] *= 1.0 if i % 2 else 1e-12
        x[tokens - 1, h] *= 1e-25 if i % 2 else 1e25
        g[tokens - 1, h] *= 1e-12 if i % 2 else 1.0
    x[0, 3] = x[tokens // 2, hq + 2] = 0
    x, g = torch.from_numpy(x).to(t), torch.from_numpy(g).to(t)
    pos, freq = torch.arange(tokens) * 7, torch.rand(R // 2, generator=torch.Generator().manual_seed(R))
    w = [torch.from_numpy(1 + 0.2 * rng.normal(size=D)).float() for _ in range(2)]
    a = heads.angles(pos.numpy(), freq.numpy())
    parts = (slice(0, hq), slice(hq, hq + hk))
    X, G = x.cuda(), g.cuda()
    args = (pos.cuda(), freq.cuda(), w[0].cuda(), w[1].cuda(), 0.0)
    out = dsq.dsq_headnorm_fwd(X[:, parts[0]], X[:, parts[1]], *args, interleaved=inter)
    for i, p in enumerate(parts):
        check_forward(out[i], x[:, p], w[i].numpy(), a, 0.0, inter, t)
    back = dsq.dsq_headnorm_bwd(*(G[:, p] for p in parts), *(X[:, p] for p in parts), *args, interleaved=inter)
    for i, p in enumerate(parts):
        gx, gw, mx, mw = heads.backward(g[:, p].double().numpy(), x[:, p].double().numpy(), w[i].numpy(), a, 0.0, inter)
        near(back[i], gx, 90 * U * mx, t)
        near(back[2 + i], gw, (tokens * (p.stop - p.start) + 30) * U * mw, torch.float32)
    dsq.dsq_headnorm_fwd(X[:, parts[0]], X[:, parts[1]], *args, interleaved=inter, out_q=X[:, parts[0]], out_k=X[:, parts[1]])
    assert all(torch.equal(X[:, p], o) for p, o in zip(parts, out))


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,hq,hk", [(64, 32, 8), (128, 5, 3), (66, 3, 1), (96, 12, 12)])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_not_a_number_in_q_and_k(dsq, t, D, hq, hk, inter):
    """A NaN or an infinity of one head stays there, forwards and backwards, in place too."""
    gen = torch.Generator().manual_seed(D)
    x, g = (torch.randn(6, hq + hk, D, generator=gen).to(t) for _ in range(2))
    pos, freq, w = torch.arange(6).cuda(), torch.rand(D // 2, generator=gen).cuda(), torch.rand(D, generator=gen).cuda()
    q, k = slice(0, hq), slice(hq, hq + hk)

    def run(x, g):
        X, G = x.cuda(), g.cuda()
        y = dsq.dsq_headnorm_fwd(X[:, q], X[:, k], pos, freq, w, w, interleaved=inter)
        b = dsq.dsq_headnorm_bwd(G[:, q], G[:, k], X[:, q], X[:, k], pos, freq, w, w, interleaved=inter)
        dsq.dsq_headnorm_fwd(X[:, q], X[:, k], pos, freq, w, w, interleaved=inter, out_q=X[:, q], out_k=X[:, k])
        assert X.isnan().equal(torch.cat(y, 1).isnan()) and torch.equal(X.nan_to_num(), torch.cat(y, 1).nan_to_num())
        return torch.cat(y, 1), torch.cat(b[:2], 1)

    good = run(x, g)
    bad_x, bad_g = x.clone(), g.clone()
    bad_x[1, hq - 1, 5], bad_x[4, hq + hk - 1, 7], bad_x[2, 0, D - 1] = float("nan"), float("inf"), float("nan")
    bad_g[3, hq, 1], bad_g[5, 1, 2] = float("nan"), float("inf")
    got = run(bad_x, bad_g)
    mark = torch.zeros(6, hq + hk, dtype=torch.bool)
    for spot in ((1, hq - 1), (4, hq + hk - 1), (2, 0)):
        mark[spot] = True
    assert torch.equal(got[0].cpu()[~mark], good[0].cpu()[~mark])
    assert got[0].cpu()[mark].isnan().any(1).all()
    mark[3, hq] = mark[5, 1] = True
    assert torch.equal(got[1].cpu()[~mark], good[1].cpu()[~mark])
    assert not got[1].cpu()[mark].isfinite().all(1).any()


@pytest.mark.parametrize("D,hq,hk", [(64, 32, 8), (128, 3, 1), (66, 5, 2)])
@pytest.mark.parametrize("size,of_g,eps", [(1e15, 1e25, 1e-6), (1e17, 1e30, 0.0), (1e-13, 1e-28, 0.0), (1e-9, 1e-30, 0.0), (1e-3, 1e37, 1e-6)])
def test_gradients_whose_products_leave_binary32(dsq, D, hq, hk, size, of_g, eps):
    """grad_y times x is beyond binary32 or below its normal numbers where grad_x is not."""
    rng = np.random.default_rng(D)
    x, g = rng.normal(size=(9, hq + hk, D)), rng.normal(size=(9, hq + hk, D))
    x[4], g[4] = x[4] * size, g[4] * of_g                       # beside ordinary ones
    x[8, hq], g[8, hq] = x[8, hq] * size, g[8, hq] * of_g
    x, g = torch.from_numpy(x).float(), torch.from_numpy(g).float()
    pos, freq = torch.arange(9), torch.rand(D // 2, generator=torch.Generator().manual_seed(D))
    w = [torch.from_numpy(1 + 0.2 * rng.normal(size=D)).float() for _ in range(2)]
    a = heads.angles(pos.numpy(), freq.numpy())
    parts = (slice(0, hq), slice(hq, hq + hk))
    X, G = x.cuda(), g.cuda()
    back = dsq.dsq_headnorm_bwd(*(G[:, p] for p in parts), *(X[:, p] for p in parts), pos.cuda(), freq.cuda(), w[0].cuda(), w[1].cuda(), eps)
    for i, p in enumerate(parts):
        gx, gw, mx, mw = heads.backward(g[:, p].double().numpy(), x[:, p].double().numpy(), w[i].numpy(), a, np.float32(eps))
        fits = np.abs(gx) < 1e38
        err = np.abs(N(back[i].double()) - gx)
        assert np.all((err <= 90 * U * mx + rounding(torch.float32, gx) * (1 + 2.0 ** -7))[fits])
        near(back[2 + i], gw, (9 * (p.stop - p.start) + 30) * U * mw, torch.float32)
