"""GPU: log probabilities at the ends of the range of scales (tolerances: test_gpu_logprob.py)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_logprob import check, logits


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


@pytest.mark.parametrize("V", [5, 1003, 40000])
def test_largest_and_smallest_scales(dsq, V):
    x, targets = logits(5, V, torch.float32, seed=11)
    x[1] = 0.0
    for e in (127, 100, -100, -120):
        y = torch.from_numpy(np.ldexp(x.numpy().astype(np.float64), -min(e, 126))).float()
        check(dsq, y, targets, 2.0 ** e, min(V, 5))
    # what is not nearly equal is apart by more than binary32 has
    z = torch.zeros(3, V)
    z[:, 1], z[1, 2], z[2, 3] = 1.0, 1.0, -1.0
    t = torch.tensor([1, 2, 1])
    logp, entropy, lse, ids, top = dsq.dsq_logprob_fwd(z.cuda(), t.cuda(), scale=2.0 ** 127, top=2)
    two = float(torch.tensor(2.0).log())
    assert np.allclose(logp.cpu(), [0, -two, 0], atol=1e-6) and np.allclose(entropy.cpu(), [0, two, 0], atol=1e-6)
    assert (lse == 2.0 ** 127).all() and ids[:, 0].tolist() == [1, 1, 1]
