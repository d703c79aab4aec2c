"""Refusals of the log probabilities and of their gradient (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_1908_05033_b200 as dsq

lib = dsq.lib
P, ODD = C.c_void_p(0x1000), C.c_void_p(0x1001)      # never dereferenced


def fwd(x=P, ld=100, M=4, V=100, t=1, targets=P, scale=1.0, top=0, logp=P, h=P, lse=P, ids=None, tl=None):
    return lib.dsq_logprob_fwd(x, ld, M, V, t, targets, scale, top, logp, h, lse, ids, tl, None)


def bwd(x=P, ld=100, M=4, V=100, t=1, targets=P, scale=1.0, lse=P, h=P, g=P, gh=None, grad=P, gld=100):
    return lib.dsq_logprob_bwd(x, ld, M, V, t, targets, scale, lse, h, g, gh, grad, gld, None)


@pytest.mark.parametrize("call,args,status", [
    (fwd, dict(x=None), -1), (fwd, dict(targets=None), -1), (fwd, dict(logp=None, h=None, lse=None), -1),
    (fwd, dict(M=0), -4), (fwd, dict(V=0), -4), (fwd, dict(ld=99), -4), (fwd, dict(M=1 << 29), -5),
    (fwd, dict(V=(1 << 30) + 1, ld=1 << 31), -5), (fwd, dict(t=3), -8), (fwd, dict(scale=0.0), -6),
    (fwd, dict(scale=-1.0), -6), (fwd, dict(scale=float("nan")), -6), (fwd, dict(scale=float("inf")), -6),
    (fwd, dict(top=3), -4), (fwd, dict(ids=P), -4), (fwd, dict(top=-1, ids=P), -4), (fwd, dict(top=101, ids=P), -4),
    (fwd, dict(top=33, ids=P), -8), (fwd, dict(x=ODD), -2), (fwd, dict(t=0, x=C.c_void_p(0x1002)), -2),
    (fwd, dict(targets=C.c_void_p(0x1004)), -2), (fwd, dict(lse=ODD), -2),
    (bwd, dict(x=None), -1), (bwd, dict(lse=None), -1), (bwd, dict(grad=None), -1), (bwd, dict(g=None), -1),
    (bwd, dict(targets=None), -1), (bwd, dict(gh=P, h=None), -1), (bwd, dict(gld=99), -4), (bwd, dict(ld=99), -4),
    (bwd, dict(V=-1), -4), (bwd, dict(t=9), -8), (bwd, dict(scale=0.0), -6), (bwd, dict(grad=ODD), -2),
    (bwd, dict(g=C.c_void_p(0x1002)), -2), (bwd, dict(M=1 << 28, V=1 << 20, ld=1 << 20, gld=1 << 20), -5),
])
def test_status(call, args, status):
    assert call(**args) == status


def test_the_binding_refuses_other_tensors():
    x, t = torch.zeros(4, 64), torch.zeros(4, dtype=torch.long)
    with pytest.raises(TypeError):                # not on a GPU
        dsq.dsq_logprob_fwd(x, t)
    with pytest.raises(TypeError):
        dsq.dsq_logprob_bwd(x, t, torch.zeros(4), torch.zeros(4))
