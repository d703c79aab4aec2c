"""GPU: recorded products with group scales follow the process-wide hooks, and what a copy that is left out does to the
outputs."""
import ctypes as C

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import groups as G
from gpu_util import T, N


@pytest.fixture(scope="module")
def dsq():
    import paper_1908_05033_b200 as d
    yield d
    d.dsq_set_wgemm_group_form(0)
    d.dsq_set_test_skip_b_round(-1)
    d.dsq_set_wait_limit_ns(0)


def case(dsq, M, n, k, group=128):
    rng = np.random.default_rng(M + n + k)
    codes = rng.integers(-8, 8, (n, k)).astype(np.int8)
    scales = np.ldexp(1.0, rng.integers(-3, 3, (-(-k // group), n))).astype(np.float32)
    x = rng.integers(-4, 5, (M, k)).astype(np.float32)          # (every sum is exact)
    return T(x).bfloat16(), dsq.dsq_pack_codes(T(codes), 4), T(scales), G.linear(x, codes, scales, group)[0]


def test_a_recorded_product_is_out_of_date_once_the_form_changes(dsq):
    M, n, k = 2, 200, 1024
    x, packed, scales, want = case(dsq, M, n, k)
    Y = torch.empty(M, n, device="cuda")
    lib = dsq.lib
    lib.dsq_plan_run.argtypes = [C.c_void_p, C.c_void_p]
    lib.dsq_plan_valid.argtypes = lib.dsq_plan_free.argtypes = [C.c_void_p]
    for form in (0, 1, 2, 3):
        dsq.dsq_set_wgemm_group_form(form)
        plan = C.c_void_p()
        assert lib.dsq_plan_begin() == 0
        dsq.dsq_wgemm_group(x, packed, M, n, k, 4, 128, scales, out=Y)
        assert lib.dsq_plan_end(C.byref(plan)) == 0
        assert lib.dsq_plan_valid(plan) == 1
        Y.zero_()
        assert lib.dsq_plan_run(plan, C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        assert np.array_equal(N(Y), want)
        dsq.dsq_set_wgemm_group_form((form + 1) % 4)
        assert lib.dsq_plan_valid(plan) == 0
        lib.dsq_plan_free(plan)


@pytest.mark.parametrize("skip", [0, 1])
@pytest.mark.parametrize("M,n,k,stages", [(8, 128, 4096, 2), (33, 128, 8192, 2), (64, 4750, 256, 1), (8, 300, 128, 1)])
def test_a_stage_that_is_left_out(dsq, M, n, k, stages, skip):
    """stages: what every block has at least of pairs of chunks (eight blocks at most share K); or exactly, where it is 1."""
    x, packed, scales, want = case(dsq, M, n, k)
    dsq.dsq_set_wgemm_group_form(2)
    dsq.dsq_set_wait_limit_ns(3_000_000)
    dsq.dsq_set_test_skip_b_round(skip)
    Y = dsq.dsq_wgemm_group(x, packed, M, n, k, 4, 128, scales)
    torch.cuda.synchronize()
    dsq.dsq_set_test_skip_b_round(-1)
    dsq.dsq_set_wait_limit_ns(0)
    if skip < stages:
        assert Y.isnan().all()
    else:
        assert np.array_equal(N(Y), want)
    Y = dsq.dsq_wgemm_group(x, packed, M, n, k, 4, 128, scales)
    dsq.dsq_set_wgemm_group_form(0)
    assert np.array_equal(N(Y), want)
