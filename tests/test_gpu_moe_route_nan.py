"""GPU: a NaN among masked logits of the router.  What is summed (the chosen logits, or all of a row) makes the weights NaN, also
beside nothing but -infinity; where it is not summed the masked logits' weights are 0."""
import pytest
import torch

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    return d


@pytest.mark.parametrize("E", [2, 20, 64, 200, 256, 300, 1000])
def test_masked_logits_and_a_nan(dsq, E):
    z = torch.full((5, E), -INF)
    z[1, E // 2] = NAN
    z[2, 0] = z[2, E - 1] = NAN
    z[3] = NAN
    z[4, E - 1], z[4, 0] = NAN, 1.0
    for k in sorted({1, min(E - 1, 30), min(E, 32)}):
        ids, w = dsq.dsq_moe_route(z.cuda(), k, True)
        ids, w = ids.cpu(), w.cpu()
        order = [[e for e in range(E) if not row[e].isnan()] + [e for e in range(E) if row[e].isnan()] for row in z]
        order[4] = [0] + [e for e in range(1, E - 1)] + [E - 1]
        assert ids.tolist() == [o[:k] for o in order]
        for t in range(5):
            if z[t, ids[t].long()].isnan().any():
                assert w[t].isnan().all()
            else:
                assert w[t].tolist() == [1.0 if t == 4 and s == 0 else 0.0 for s in range(k)]
        ids, w = dsq.dsq_moe_route(z.cuda(), k, False)
        assert not w[0].any() and w[1:].isnan().all()
