"""Refusals of the heads' norm and rotation: the status comes from the host before anything is
launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_1908_05033_b200 as dsq
from paper_1908_05033_b200 import binding as B

lib = dsq.lib
P, ODD = 0x1000, 0x1001         # never dereferenced
NAN = float("nan")


def fwd(q=True, x=P, y=P, w=None, heads=4, strides=(256, 64, 256, 64), k=None, tokens=3, rot=True, pos=P, freq=P,
        axis=None, D=64, R=64, axes=1, norm=1, eps=1e-6, t=1):
    h = B.dsq_heads_t(x, y, w, heads, *strides)
    r = B.dsq_rotary_t(pos, freq, axis, D, R, axes, 0)
    return lib.dsq_headnorm_fwd(C.byref(h) if q else None, C.byref(k) if k else None, tokens,
                                C.byref(r) if rot else None, norm, eps, t, None)


def bwd(gy=P, x=P, w=P, gx=P, gw=P, heads=4, strides=(256, 64) * 3, tokens=3, D=64, R=64, norm=1, eps=1e-6, t=1,
        ws=P, nbytes=1 << 30):
    h = B.dsq_heads_grad_t(gy, x, w, gx, gw, heads, *strides)
    r = B.dsq_rotary_t(P, P, None, D, R, 1, 0)
    return lib.dsq_headnorm_bwd(C.byref(h), None, tokens, C.byref(r), norm, eps, t, ws, nbytes, None)


@pytest.mark.parametrize("call,args,status", [
    (fwd, dict(q=False), -1), (fwd, dict(x=None), -1), (fwd, dict(y=None), -1), (fwd, dict(rot=False), -1),
    (fwd, dict(pos=None), -1), (fwd, dict(freq=None), -1),
    (fwd, dict(k=B.dsq_heads_t(None, P, None, 1, 64, 64, 64, 64)), -1),
    (fwd, dict(k=B.dsq_heads_t(P, P, None, 0, 64, 64, 64, 64)), -4),
    (fwd, dict(tokens=0), -4), (fwd, dict(heads=0), -4), (fwd, dict(D=0), -4), (fwd, dict(R=66), -4),
    (fwd, dict(R=3), -4), (fwd, dict(R=-2), -4), (fwd, dict(axes=0), -4), (fwd, dict(axes=256), -5),
    (fwd, dict(D=514, R=2), -5), (fwd, dict(heads=4097), -5), (fwd, dict(tokens=1 << 32), -5),
    (fwd, dict(D=63, R=62), -8), (fwd, dict(t=3), -8), (fwd, dict(t=-1), -8), (fwd, dict(w=P, norm=0), -8),
    (fwd, dict(eps=-1e-6), -6), (fwd, dict(eps=NAN), -6),
    (fwd, dict(x=ODD), -2), (fwd, dict(y=ODD), -2), (fwd, dict(pos=P + 4), -2), (fwd, dict(freq=P + 2), -2),
    (fwd, dict(w=P + 2), -2),
    # heads of y that overlap: too near, tokens too near, broadcast
    (fwd, dict(strides=(256, 64, 256, 63)), -4), (fwd, dict(strides=(256, 64, 255, 64)), -4),
    (fwd, dict(strides=(256, 64, 256, 0)), -4), (fwd, dict(strides=(256, 64, -256, 64)), -4),
    (fwd, dict(strides=(256, 64, 64, 191)), -4),
    (bwd, dict(gy=None), -1), (bwd, dict(gx=None), -1), (bwd, dict(x=None), -1), (bwd, dict(ws=None), -1),
    (bwd, dict(ws=P + 8), -2), (bwd, dict(nbytes=256 + 4 * 64), -5), (bwd, dict(norm=0), -8),
    (bwd, dict(strides=(256, 64, 256, 64, 256, 32)), -4), (bwd, dict(t=7), -8), (bwd, dict(gw=P + 2), -2),
])
def test_status(call, args, status):
    assert call(**args) == status


def test_sizes():
    assert dsq.dsq_headnorm_bwd_workspace_bytes(0) == dsq.dsq_workspace_bytes()
    assert dsq.dsq_headnorm_bwd_workspace_bytes(128) >= 256 + 128 * 4 * 148


def test_the_binding_refuses_other_tensors():
    x, pos, freq = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.long), torch.ones(32)
    with pytest.raises(TypeError):                # not on a GPU
        dsq.dsq_headnorm_fwd(x, x, pos, freq)
    with pytest.raises(TypeError):
        dsq.dsq_headnorm_bwd(x, x, x, x, pos, freq)
