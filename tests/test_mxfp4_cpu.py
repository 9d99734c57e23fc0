"""MXFP4 on the CPU: the plain reference on hand-worked blocks, and every argument that the
conversions refuse (nothing is launched)."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import mxfp4 as om
from paper_2607_08782_amd import moe


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(moe.LIB_PATH):
        from paper_2607_08782_amd import build
        build.build()
    return moe.load_library()


def test_reference_on_hand_worked_blocks():
    v = np.zeros((1, 32), np.float32)
    # largest 5: exponent 2, scale 1
    v[0, :10] = [5.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.26, -5.0, 4.99]
    code, byte = om.encode(v)
    assert byte[0].tolist() == [127, 0, 0, 0]
    assert code[0, :10].tolist() == [6, 0, 2, 2, 4, 4, 6, 9, 14, 6]
    # largest 0.9 (exponent -1, scale 2^-3): 0.9 is 7.2 of it, past 6
    v = np.zeros((1, 33), np.float32)
    v[0, 0], v[0, 1], v[0, 32] = 0.9, 0.0625, 96.0
    code, byte = om.encode(v)
    assert byte[0].tolist() == [124, 131, 0, 0] and code.shape == (1, 128)
    assert om.values(code, byte, 33)[0, [0, 1, 32]].tolist() == [0.75, 0.0625, 96.0]
    # an infinity takes its block, not the next
    v = np.ones((1, 64), np.float32)
    v[0, 3] = np.inf
    got = om.rounded(v)
    assert np.isnan(got[0, :32]).all() and (got[0, 32:] == 1).all()
    packed = om.pack(code)
    np.testing.assert_array_equal(om.unpack(packed), code)


F = ctypes.c_void_p(0x1000)            # never dereferenced: every call below fails validation


def test_conversions_refuse(lib):
    for fn, order in ((lib.moe_quantize_mxfp4, "xdrcqs"), (lib.moe_dequantize_mxfp4, "qsrcdx")):
        def call(**kw):
            a = dict(x=F, d=1, r=4, c=64, q=F, s=F)
            a.update(kw)
            return fn(*[a[k] for k in order], None)
        for bad in (dict(x=None), dict(q=None), dict(s=None), dict(d=2), dict(d=-1), dict(r=-1),
                    dict(c=0), dict(c=-5), dict(x=ctypes.c_void_p(0x1001)),
                    dict(d=0, x=ctypes.c_void_p(0x1002)), dict(q=ctypes.c_void_p(0x1008)),
                    dict(s=ctypes.c_void_p(0x1002))):
            assert call(**bad) == moe.MOE_ERR_ARG, bad
        for bad in (dict(c=1 << 28), dict(r=1 << 41)):
            assert call(**bad) == moe.MOE_ERR_SHAPE, bad
        assert call(r=0, x=None, q=None, s=None) == moe.MOE_OK


def test_wrappers_refuse():
    x = torch.zeros(4, 100)
    u8 = dict(dtype=torch.uint8)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        moe.moe_quantize_mxfp4(x)
    with pytest.raises(ValueError, match="q must hold"):
        moe.moe_quantize_mxfp4(x, q=torch.zeros(4, 63, **u8))
    with pytest.raises(ValueError, match="scales must hold"):
        moe.moe_quantize_mxfp4(x, scales=torch.zeros(4, 3, **u8))
    q, s = torch.zeros(4, 64, **u8), torch.zeros(4, 4, **u8)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        moe.moe_dequantize_mxfp4(q, s, 100)
    for bad in ((q, s, 0), (q, s, 129), (q[:, :32], s, 100), (q, s[:3], 100)):
        with pytest.raises(ValueError):
            moe.moe_dequantize_mxfp4(*bad)
    with pytest.raises(ValueError, match="out must hold"):
        moe.moe_dequantize_mxfp4(q, s, 100, out=torch.zeros(4, 99, dtype=torch.bfloat16))


def _table(n, bad=None, value=None):
    """Four host arrays of device pointers (stand-ins), one entry of one of them replaced."""
    arrays = [[0x10000 * (i + 1) + 0x100 * j for j in range(n)] for i in range(4)]
    if bad is not None:
        arrays[bad[0]][bad[1]] = value
    keep = [(ctypes.c_void_p * n)(*a) for a in arrays]
    return keep, [ctypes.cast(a, ctypes.c_void_p) for a in keep]


def test_grouped_ffn_refuses(lib):
    need = lib.moe_grouped_ffn_mxfp4_ws_bytes(16, 40, 256, 96, 2)
    assert need >= 16 * 128 + 40 * 64

    def call(table=None, **kw):
        a = dict(x=F, T=16, tok=F, off=F, n=2, sh=0, d=256, f=96, cap=40, y=F, ws=0x100000, nb=need)
        a.update(kw)
        keep, p = table or _table(max(1, min(a["n"] + a["sh"], 200)))
        p = [a.get("p%d" % i, q) for i, q in enumerate(p)]
        return lib.moe_grouped_ffn_mxfp4(a["x"], a["T"], a["tok"], a["off"], a["n"], a["sh"], *p, a["d"],
                                         a["f"], a["cap"], a["y"], ctypes.c_void_p(a["ws"]), a["nb"], None)
    for bad in (dict(x=None), dict(off=None), dict(y=None), dict(T=-1), dict(n=-1), dict(n=0), dict(sh=-1),
                dict(n=129), dict(n=100, sh=29), dict(d=0), dict(f=0), dict(cap=-1), dict(cap=1 << 31),
                dict(T=1 << 31), dict(sh=1, tok=None), dict(sh=1, T=0), dict(T=1 << 30, sh=2, n=1),
                dict(x=ctypes.c_void_p(0x1008)), dict(y=ctypes.c_void_p(0x1008)),
                dict(p0=None), dict(p1=None), dict(p2=None), dict(p3=None)):
        assert call(**bad) == moe.MOE_ERR_ARG, bad
    for i in range(4):
        for value in (None, 0x10000 + (8 if i % 2 == 0 else 2)):
            assert call(_table(2, (i, 1), value)) == moe.MOE_ERR_ARG, (i, value)
    for bad in (dict(d=252), dict(d=1 << 21), dict(f=1 << 21), dict(T=1 << 25, nb=1 << 62), dict(nb=need - 1),
                dict(ws=0x100010), dict(ws=0), dict(tok=None, T=39)):
        assert call(**bad) == moe.MOE_ERR_SHAPE, bad
    assert call(cap=0, n=1, y=None, ws=0, nb=0) == moe.MOE_OK        # nothing to do


def test_lay_out_refuses(lib):
    def call(q=F, s=F, r=4, c=64, o=F, w=F):
        return lib.moe_mxfp4_lay_out(q, s, r, c, o, w, None)
    for bad in (dict(q=None), dict(s=None), dict(o=None), dict(w=None), dict(r=-1), dict(c=0),
                dict(q=ctypes.c_void_p(0x1008)), dict(s=ctypes.c_void_p(0x1001)),
                dict(o=ctypes.c_void_p(0x1008)), dict(w=ctypes.c_void_p(0x1002))):
        assert call(**bad) == moe.MOE_ERR_ARG, bad
    assert call(c=1 << 28) == moe.MOE_ERR_SHAPE and call(r=1 << 37) == moe.MOE_ERR_SHAPE
    assert call(r=0, q=None, s=None, o=None, w=None) == moe.MOE_OK
    u8 = dict(dtype=torch.uint8)
    q, s = torch.zeros(4, 64, **u8), torch.zeros(4, 4, **u8)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        moe.moe_mxfp4_lay_out(q, s, 100)
    for bad in ((q, s, 0), (q, s, 129), (q[:, :32], s, 100), (q, s[:3], 100)):
        with pytest.raises(ValueError):
            moe.moe_mxfp4_lay_out(*bad)


def test_ffn_wrapper_refuses():
    u8 = dict(dtype=torch.uint8)
    pair = (torch.zeros(64, 64, **u8), torch.zeros(64, 4, **u8))
    for bad in (([], []), ([pair], []), ([pair], [pair])):
        with pytest.raises(ValueError):
            moe.MxWeightTable(*bad, 100, 31)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        moe.MxWeightTable([pair], [pair], 100, 32)
    with pytest.raises(ValueError):
        moe.MxWeightTable.quantized([], [])
    table = moe.MxWeightTable.__new__(moe.MxWeightTable)
    table.d, table.f, table.w13 = 64, 32, [None, None]
    x, off = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    tok = torch.zeros(8, dtype=torch.int32)
    for bad in (dict(x=x.float()), dict(x=x[:, :32]), dict(off=off[:2]), dict(tok=tok), dict(n_shared=3),
                dict(tok=tok, cap_rows=9), dict(cap_rows=4, y_perm=torch.zeros(3, 64, dtype=torch.bfloat16))):
        a = dict(dict(x=x, off=off), **bad)
        with pytest.raises(ValueError):
            moe.moe_grouped_ffn_mxfp4(a.pop("x"), a.pop("off"), table, row_token=a.pop("tok", None), **a)
