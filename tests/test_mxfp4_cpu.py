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
