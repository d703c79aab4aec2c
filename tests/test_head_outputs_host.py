"""Refusal of q and k with one buffer for what is written (no GPU needed: the status comes before anything is launched)."""
import ctypes as C

from paper_1908_05033_b200 import binding as B
from test_head_operators_host import P, fwd, lib


def test_one_output_for_q_and_k():
    assert fwd(k=B.dsq_heads_t(2 * P, P, None, 2, 256, 64, 256, 64)) == -4
    assert fwd(k=B.dsq_heads_t(P, P, None, 2, 256, 64, 256, 64)) == -4


def test_one_gradient_for_q_and_k():
    r = B.dsq_rotary_t(P, P, None, 64, 64, 1, 0)
    h = [B.dsq_heads_grad_t(i * P, i * P, None, 4 * P, None, 4, *(256, 64) * 3) for i in (1, 2)]
    assert lib.dsq_headnorm_bwd(C.byref(h[0]), C.byref(h[1]), 3, C.byref(r), 1, 1e-6, 1, P, 1 << 30, None) == -4
