"""Refusals of the norm, of group-wise weights and of their products: the status comes from
the host before anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_1908_05033_b200 as dsq
from paper_1908_05033_b200 import binding as B

lib = dsq.lib
P = C.c_void_p(0x1000)          # aligned, never dereferenced
ODD = C.c_void_p(0x1008)
NAN = float("nan")


def norm(x=P, r=None, w=P, M=4, K=64, t=1, eps=1e-5, h=None, y=P, q=None, s=None, rstd=None):
    return lib.dsq_rmsnorm_fwd(x, r, w, M, K, t, eps, h, y, q, s, rstd, None)


def grad(gy=P, gh=None, h=P, w=P, rstd=P, M=4, K=64, t=1, gx=P, gw=P, ws=P, nbytes=1 << 30):
    return lib.dsq_rmsnorm_bwd(gy, gh, h, w, rstd, M, K, t, gx, gw, ws, nbytes, None)


def quantize(w=P, N=4, K=64, t=1, bits=4, group=32, codes=P, nbytes=1 << 30, scales=P):
    return lib.dsq_quantize_groups(w, N, K, t, bits, group, codes, nbytes, scales, None)


def values(codes=P, scales=P, N=4, K=64, bits=4, group=32, off=0.5, t=1, out=P):
    return lib.dsq_dequantize_groups(codes, scales, N, K, bits, group, off, t, out, None)


def linear(X=P, xt=1, rs=None, W=P, s=P, b=None, M=1, N=4, K=64, bits=4, group=32, off=0.5, yt=0,
           Y=P):
    return lib.dsq_wgemm_group(X, xt, rs, W, s, b, M, N, K, bits, group, off, yt, Y, None)


@pytest.mark.parametrize("call,args,status", [
    (norm, dict(x=None), -1), (norm, dict(w=None), -1), (norm, dict(y=None), -1),
    (norm, dict(q=P), -1),                       # codes without scales
    (norm, dict(M=0), -4), (norm, dict(K=0), -4), (norm, dict(K=49153), -5),
    (norm, dict(t=3), -8), (norm, dict(t=-1), -8), (norm, dict(eps=-1.0), -6),
    (norm, dict(eps=NAN), -6), (norm, dict(eps=float("inf")), -6),
    (norm, dict(r=ODD), -2), (norm, dict(h=ODD), -2), (norm, dict(rstd=ODD), -2),
    (norm, dict(q=ODD, s=P), -2),
    (grad, dict(gy=None), -1), (grad, dict(h=None), -1), (grad, dict(rstd=None), -1),
    (grad, dict(gx=None), -1), (grad, dict(ws=None), -1), (grad, dict(M=-1), -4),
    (grad, dict(K=50000), -5), (grad, dict(t=4), -8), (grad, dict(gh=ODD), -2),
    (grad, dict(ws=ODD), -2), (grad, dict(nbytes=256 + 4 * 64 - 1), -5),
    (quantize, dict(w=None), -1), (quantize, dict(scales=None), -1), (quantize, dict(bits=5), -3),
    (quantize, dict(bits=0), -3), (quantize, dict(bits=2), -8), (quantize, dict(group=48), -8),
    (quantize, dict(group=0), -4), (quantize, dict(N=0), -4), (quantize, dict(K=1 << 21), -5),
    (quantize, dict(t=3), -8), (quantize, dict(nbytes=127), -5), (quantize, dict(codes=ODD), -2),
    (values, dict(out=None), -1), (values, dict(off=0.25), -8), (values, dict(off=NAN), -6),
    (values, dict(group=33), -8), (values, dict(bits=3), -8), (values, dict(scales=ODD), -2),
    (linear, dict(X=None), -1), (linear, dict(Y=None), -1), (linear, dict(xt=3), -1),
    (linear, dict(xt=0), -8), (linear, dict(yt=3), -8), (linear, dict(rs=P), -8),
    (linear, dict(off=1.0), -8), (linear, dict(off=NAN), -6), (linear, dict(M=0), -4),
    (linear, dict(K=60), -2), (linear, dict(K=72, xt=3, rs=P), -2), (linear, dict(b=ODD), -2),
    (linear, dict(M=65535 * 64 + 1), -5), (linear, dict(bits=1), -8), (linear, dict(bits=6), -3),
    (linear, dict(xt=3, rs=P, K=1 << 17, group=1 << 17), -7),
])
def test_status(call, args, status):
    assert call(**args) == status


def test_sizes():
    assert dsq.dsq_group_count(1, 32) == 1 and dsq.dsq_group_count(64, 32) == 2
    assert dsq.dsq_group_count(65, 32) == 3 and dsq.dsq_group_count(0, 32) == 0
    assert dsq.dsq_group_count(1 << 20, 1 << 40) == 1
    small, large = (dsq.dsq_rmsnorm_bwd_workspace_bytes(m, 100) for m in (1, 1 << 20))
    assert 256 + 400 <= small < large <= 256 + 4 * 100 * 148 * 8
    assert dsq.dsq_rmsnorm_bwd_workspace_bytes(0, 100) == dsq.dsq_workspace_bytes()


def test_the_binding_refuses_other_tensors():
    x = torch.zeros(4, 64)                       # not on a GPU
    for call in (lambda: dsq.dsq_rmsnorm_fwd(x, torch.ones(64), 1e-5),
                 lambda: dsq.dsq_rmsnorm_bwd(x, x, torch.ones(64), torch.ones(4)),
                 lambda: dsq.dsq_quantize_groups(x, 4, 32),
                 lambda: dsq.dsq_dequantize_groups(x.byte(), torch.ones(2, 4), 4, 64),
                 lambda: dsq.dsq_wgemm_group(x.bfloat16(), x.byte(), 4, 4, 64, 4, 32, torch.ones(2, 4))):
        with pytest.raises(TypeError):
            call()
    assert set(B._DTYPES.values()) == {0, 1, 2}
