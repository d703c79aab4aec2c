"""GPU: alternatives of rows whose elements are mostly equal: masks that leave few tokens, masks of several kinds, rows of one value.
What is left comes first, then the mask's lowest indices (tolerances: test_gpu_logprob.py)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import logprob
from gpu_util import N
from test_gpu_logprob import INF, TYPES, check, logits


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


def kept(row, n, mask, seed, near=None):
    """The row with all but n elements (next to one another, or anywhere) masked."""
    V = len(row)
    g = torch.Generator().manual_seed(seed)
    here = torch.randperm(V, generator=g)[:n] if near is None else torch.arange(near, near + n) % V
    out = torch.full_like(row, mask)
    out[here] = row[here]
    return out


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,V", [(1, 128000), (3, 40001), (300, 5003), (2, 600), (40, 20001)])
def test_few_are_left(dsq, t, M, V):
    x, targets = logits(M, V, t, seed=21)
    for mask in (-INF, float(torch.finfo(t).min), -1e4):
        for n in (0, 1, 3, 19, 20, 21, 100):
            y = torch.stack([kept(r, min(n, V), mask, i + n, near=None if i % 2 else 7 * i + V - 5) for i, r in enumerate(x)])
            check(dsq, y, targets, 1.0, 20)
    check(dsq, y, targets, 1.0, 32)


@pytest.mark.parametrize("t", TYPES)
def test_masks_of_several_kinds(dsq, t):
    """-infinity among the lowest value and the other way round; ids alone where a NaN makes the numbers NaN."""
    V, low = 50021, float(torch.finfo(t).min)
    x, targets = logits(12, V, t, seed=22)
    g = torch.Generator().manual_seed(5)
    some = lambda n: torch.randperm(V, generator=g)[:n]
    for i, n in enumerate((0, 3, 10, 30)):
        x[i] = kept(x[i], n, -INF, i)
        x[i, some(6)] = low
    for i, n in enumerate((0, 3, 10, 30), 4):
        x[i] = kept(x[i], n, low, i)
        x[i, : V // 2] = -INF
    x[8] = kept(x[8], 4, -INF, 8)
    x[8, V - 30000:V - 15000] = low
    x[9:] = -INF
    x[9, V - 3:] = low
    x[10, 40000:] = 1.0
    x[11, ::2] = low
    targets[:] = 0
    for top in (1, 8, 32):
        check(dsq, x, targets, 1.0, top)
        check(dsq, x[8:9], targets[:1], 1.0, top)
    y = x.clone()
    y[0, : V - 11] = float("nan")
    y[3, : V // 2] = float("nan")
    y[5] = float("nan")
    y[8, 100:] = float("nan")
    y[9, some(V - 9)] = float("nan")
    y[10] = float("nan")
    y[10, some(3)] = 2.0
    for rows in (slice(0, 12), slice(8, 9), slice(10, 11)):
        for top in (1, 20, 32):
            ids = dsq.dsq_logprob_fwd(y[rows].cuda(), targets[rows].cuda(), top=top)[3]
            assert np.array_equal(N(ids), logprob.largest(y[rows].double().numpy(), top))


@pytest.mark.parametrize("M", [1, 30, 330])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_one_value_and_few_others(dsq, t, M):
    rng = np.random.default_rng(M)
    V = 60007
    for many in (1.0, 0.0, -3.0):
        x = torch.full((M, V), many)
        x[:, torch.from_numpy(rng.permutation(V)[:9])] = 5.0
        x[:, torch.from_numpy(rng.permutation(V)[: V // 3])] = -7.0
        if many == 0.0:
            x[:, 1::2][x[:, 1::2] == 0] = -0.0
        check(dsq, x.to(t), torch.zeros(M, dtype=torch.long), 1.0, 20)
        # the equal ones far back, at odd addresses
        wide = torch.full((M, V + 7), -9.0, dtype=t)
        wide[:, 3 + V // 2:] = many
        g = wide.cuda()
        check(dsq, wide[:, 3:3 + V], torch.zeros(M, dtype=torch.long), 1.0, 32, device_x=g[:, 3:3 + V])
