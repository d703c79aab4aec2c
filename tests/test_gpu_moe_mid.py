"""GPU: what a layer of experts keeps of mid, seen where the residual takes most of the experts' sum away.

Rows of x have one element, a power of two, so that the first products' sums are one product each; mid then is as exact as
its activation and what it is kept to.  Tolerances, in units u = 2^-24 of binary32, of the magnitudes of the terms:
  first sums    one product with its scale: eps_in = 2 u
  mid           activation and product 16 u, then 22 bits on 16 bits, 2^-31 of the largest on digits: eps_mid = 20 u + 2^-22
  second sums   an instruction's sums 64 u, I / 32 groups, k slots and the residual, 8 warps of 8 blocks: eps_out =
                (84 + I / 32 + 2 k) u
  y             half a step of the type
(mid to 11 bits is off by up to 2^-11 = 8192 u, a token's eight or sixteen of them together by some 1000 u.)
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import moe
from gpu_util import N
from test_gpu_moe import Layer, U


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


# T, E, k: digits; 16 bits with up to 8 and up to 16 slots of an expert, and with several groups of one
@pytest.mark.parametrize("T,E,k", [(3, 2, 1), (8, 2, 1), (16, 2, 1), (64, 2, 1), (64, 8, 2), (70, 3, 2)])
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("off", [0.5, 0.0])
@pytest.mark.parametrize("group", [32, 128])
def test_what_a_residual_leaves(dsq, T, E, k, t, off, group):
    H, I = 256, 8
    a = Layer(dsq, T, H, I, E, k, group, t=t, seed=11)
    rng = np.random.default_rng(T + E)
    x = np.zeros((T, H))
    x[np.arange(T), rng.integers(0, H, T)] = 2.0 ** rng.integers(4, 7, T)
    a.x = torch.from_numpy(x).to(t)
    eps = dict(eps_in=2 * U, eps_mid=20 * U + 2.0 ** -22, eps_out=(84 + I / 32 + 2 * k) * U, digits=0.0)
    args = (x, a.ids, a.w, a.c_in, a.s_in, a.c_out, a.s_out, E, I, group, "silu", off)
    sums, _ = moe.layer(*args, **eps)
    for of in (torch.float32, t):
        a.residual = torch.from_numpy(-sums).to(torch.bfloat16).to(of)
        y = a.run(dsq, w_offset=off, residual=a.residual.cuda(), out_dtype=of)
        ref, bound = moe.layer(*args, residual=a.residual.double().numpy(), **eps)
        # (digits: half a step of 2^-30 of the largest of a chunk, beside eps_mid of each)
        bound = bound + 2.0 ** -30 * np.abs(sums).max(1, keepdims=True) * 16
        f = torch.finfo(of)
        tol = bound + f.eps / 2 * (np.abs(ref) + bound) + f.smallest_normal * f.eps
        err = np.abs(N(y.double()) - ref)
        assert np.all(err <= tol), (err / tol).max()


@pytest.mark.parametrize("T", [1, 7, 30])
def test_outliers_of_bf16_on_the_grid_without_a_zero(dsq, T):
    """Elements of 1e30, one in each 128 of a row, where no code makes them vanish."""
    a = Layer(dsq, T, 512, 96, 3, 2, 64, seed=6)
    a.x[:, 5::128] = 1e30
    a.x[:, 77] = 2.0 ** -20
    a.s_in *= np.float32(1e-30)
    a.weights[1] = torch.from_numpy(a.s_in).cuda()
    a.check(a.run(dsq, out_dtype=torch.float32, residual=None), residual=False)
    a.check(a.run(dsq))


def test_a_layer_of_1024_experts(dsq):
    """Two slots an expert and one with many: more groups than 16 bits of slots would need."""
    a = Layer(dsq, 64, 64, 32, 1024, 32, 32, seed=12)
    a.ids[:, 0] = 1023
    a.check(a.run(dsq))
    a.ids[:] = 1023
    a.check(a.run(dsq))
