"""Every argument that the gradient calls refuse (CPU: nothing is launched)."""
import ctypes
import os

import pytest
import torch

from paper_2607_08782_amd import moe


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(moe.LIB_PATH):
        from paper_2607_08782_amd import build
        build.build()
    return moe.load_library()


F = ctypes.c_void_p(0x1000)            # never dereferenced: every call below fails validation
ODD = ctypes.c_void_p(0x1008)


def test_combine_and_permute_backward_refuse(lib):
    def cb(**kw):
        a = dict(dy=F, y=F, t=1, row=F, gate=F, T=4, d=64, k=2, o=F, g=F)
        a.update(kw)
        return lib.moe_combine_backward(a["dy"], a["y"], a["t"], a["row"], a["gate"], a["T"], a["d"],
                                        a["k"], a["o"], a["g"], None)

    def pb(**kw):
        a = dict(x=F, t=1, row=F, add=None, T=4, d=64, k=2, o=F)
        a.update(kw)
        return lib.moe_permute_backward(a["x"], a["t"], a["row"], a["add"], a["T"], a["d"], a["k"],
                                        a["o"], None)
    sizes = [dict(t=2), dict(t=-1), dict(T=-1), dict(T=1 << 31), dict(d=0), dict(k=0), dict(k=17)]
    for bad in sizes + [dict(dy=None), dict(row=None), dict(y=None), dict(gate=None), dict(dy=ODD),
                        dict(y=ODD), dict(o=ODD)]:
        assert cb(**bad) == moe.MOE_ERR_ARG, bad
    for bad in sizes + [dict(x=None), dict(row=None), dict(o=None), dict(x=ODD), dict(add=ODD), dict(o=ODD)]:
        assert pb(**bad) == moe.MOE_ERR_ARG, bad
    assert cb(T=0, dy=None, y=None, row=None, gate=None) == moe.MOE_OK
    assert cb(o=None, g=None, y=None, gate=None) == moe.MOE_OK          # nothing asked for
    assert pb(T=0, x=None, row=None, o=None) == moe.MOE_OK


def test_route_backward_refuses(lib):
    def call(**kw):
        a = dict(dg=F, gate=F, idx=F, lg=F, x=F, w=F, t=1, T=40, d=64, E=8, k=2, fl=0, dl=F, dx=F, dw=F,
                 db=F, ws=0x100000)
        a.update(kw)
        need = lib.moe_route_topk_backward_ws_bytes(1, 40, 64, 8, 2, 0)
        return lib.moe_route_topk_backward(a["dg"], a["gate"], a["idx"], a["lg"], a["x"], a["w"], a["t"],
                                           a["T"], a["d"], a["E"], a["k"], a["fl"], a["dl"], a["dx"],
                                           a["dw"], a["db"], ctypes.c_void_p(a["ws"]), a.get("nb", need),
                                           None)
    for bad in (dict(t=2), dict(T=-1), dict(T=1 << 31), dict(d=0), dict(E=0), dict(E=257), dict(k=0),
                dict(k=9), dict(E=64, k=17), dict(fl=2), dict(fl=4), dict(dg=None), dict(gate=None),
                dict(idx=None), dict(lg=None), dict(x=None), dict(w=None), dict(x=ODD), dict(w=ODD),
                dict(dx=ODD)):
        assert call(**bad) == moe.MOE_ERR_ARG, bad
    for bad in (dict(d=60), dict(d=1 << 22), dict(ws=0), dict(ws=0x100010), dict(nb=1000)):
        assert call(**bad) == moe.MOE_ERR_SHAPE, bad
    assert call(dl=None, dx=None, dw=None, db=None) == moe.MOE_OK       # nothing asked for


def test_wrappers_refuse():
    T, k, d, E, n = 6, 2, 16, 8, 9
    dy, y, row = torch.zeros(T, d), torch.zeros(n, d), torch.zeros(T, k, dtype=torch.int32)
    gate = torch.zeros(T, k)
    cb = moe.moe_combine_backward
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        cb(dy, y, row, gate)
    for bad in (lambda: cb(dy, y[:, :8], row, gate), lambda: cb(dy, y.bfloat16(), row, gate),
                lambda: cb(dy, y, row[:5], gate), lambda: cb(dy, y, row, gate[:, :1]),
                lambda: cb(dy, y, row, gate.double()), lambda: cb(dy, None, row, gate),
                lambda: cb(dy, y, row, gate, dy_perm=y[:8]), lambda: cb(dy, y, row, gate, dgate=gate[:5]),
                lambda: cb(dy, y, row, gate, dy_perm=y.bfloat16())):
        with pytest.raises(ValueError):
            bad()
    pb = moe.moe_permute_backward
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        pb(y, row)
    for kw in (dict(dx_add=dy[:5]), dict(dx_add=dy.bfloat16()), dict(dx=dy[:, :8]), dict(dx=dy.bfloat16())):
        with pytest.raises(ValueError, match="must be torch"):
            pb(y, row, **kw)
    rb = moe.moe_route_topk_backward
    x, w, lg = torch.zeros(T, d), torch.zeros(E, d), torch.zeros(T, E)
    args = gate, gate, row, x, w
    for bad in (lambda: rb(gate[:5], gate, row, x, w), lambda: rb(gate, gate[:, :1], row, x, w),
                lambda: rb(gate, gate, row.long(), x, w), lambda: rb(gate, gate, row, x, w.bfloat16()),
                lambda: rb(gate, gate, row, x, w[:, :8]), lambda: rb(*args, renorm=False),
                lambda: rb(*args, renorm=False, logits=lg[:, :7]), lambda: rb(*args, dlogits=lg[:5]),
                lambda: rb(*args, dx=x.bfloat16()), lambda: rb(*args, dw=w[:7]),
                lambda: rb(*args, dbias=torch.zeros(7))):
        with pytest.raises(ValueError):
            bad()
