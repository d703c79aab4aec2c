"""Refusals of the router's choice and of the layer of experts (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_1908_05033_b200 as dsq

lib = dsq.lib
P, ODD = C.c_void_p(0x1000), C.c_void_p(0x1008)      # never dereferenced
NAN = float("nan")


def route(z=P, T=4, E=8, k=2, ids=P, w=P):
    return lib.dsq_moe_route(z, T, E, k, 1, ids, w, None)


def layer(X=P, xt=1, ids=P, w=P, wi=P, si=P, wo=P, so=P, T=4, H=64, I=48, E=8, k=2, bits=4, group=32, off=0.5, act=0,
          res=None, yt=1, Y=P, ws=P, nbytes=1 << 30):
    return lib.dsq_moe_group(X, xt, ids, w, wi, si, wo, so, T, H, I, E, k, bits, group, off, act, res, yt, Y, ws,
                             nbytes, None)


@pytest.mark.parametrize("call,args,status", [
    (route, dict(z=None), -1), (route, dict(ids=None), -1), (route, dict(w=None), -1), (route, dict(T=0), -4),
    (route, dict(E=0), -4), (route, dict(k=0), -4), (route, dict(k=9), -4), (route, dict(k=33, E=64), -5),
    (route, dict(E=1 << 21), -5), (route, dict(T=1 << 29), -5), (route, dict(z=ODD), -2), (route, dict(ids=ODD), -2),
    *[(layer, {n: None}, -1) for n in ("X", "ids", "w", "wi", "si", "wo", "so", "Y", "ws")],
    *[(layer, {n: 0}, -4) for n in ("T", "H", "I", "E", "k")],
    (layer, dict(T=(1 << 20) + 1), -5), (layer, dict(E=1025), -5), (layer, dict(k=33), -5),
    (layer, dict(H=(1 << 20) + 8), -5), (layer, dict(I=(1 << 20) + 1), -5), (layer, dict(I=1 << 20, E=1024), -5),
    (layer, dict(bits=5), -3), (layer, dict(bits=3), -8), (layer, dict(group=48), -8), (layer, dict(group=0), -4),
    (layer, dict(off=NAN), -6), (layer, dict(off=0.25), -8), (layer, dict(act=2), -8), (layer, dict(xt=0), -8),
    (layer, dict(xt=3), -8), (layer, dict(yt=3), -8), (layer, dict(H=60), -2), (layer, dict(X=ODD), -2),
    (layer, dict(res=ODD), -2), (layer, dict(ws=ODD), -2), (layer, dict(nbytes=4 * 2 * 128 * 8), -5),
])
def test_status(call, args, status):
    assert call(**args) == status


def test_sizes():
    # digits of four bytes an element of x, eight bytes an element of mid, in chunks of 128
    need = 4 * 64 * 4 + 4 * 2 * 128 * 8
    assert need <= dsq.dsq_moe_workspace_bytes(4, 64, 48, 2) <= 256 + 2 * need + 9 * 256
    assert dsq.dsq_moe_workspace_bytes(64, 64, 100, 3) == dsq.dsq_moe_workspace_bytes(1 << 19, 64, 100, 3)
    for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, 33), (1, 1 << 21, 1, 1)):
        assert dsq.dsq_moe_workspace_bytes(*bad) == dsq.dsq_workspace_bytes()


def test_the_binding_refuses_other_tensors():
    with pytest.raises(TypeError):                # not on a GPU
        dsq.dsq_moe_route(torch.zeros(4, 8), 2)
    z = torch.zeros(1)
    with pytest.raises(TypeError):
        dsq.dsq_moe_group(z.bfloat16(), z.int(), z, z.byte(), z, z.byte(), z, 1, 1)
    with pytest.raises(ValueError):
        dsq.dsq_moe_group(z, z, z, z, z, z, z, 1, 1, activation="relu")
