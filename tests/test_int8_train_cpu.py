"""Argument checks of the 8-bit rows', the norm's, the balance loss's and the clipping's calls that
need no GPU (every call fails validation, so nothing is launched and no pointer is read), and the
workspace sizes."""
import ctypes
import os

import pytest

from paper_2607_08782_amd import moe

FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1001)
ARG, SHAPE = moe.MOE_ERR_ARG, moe.MOE_ERR_SHAPE
BIG = 1 << 40
BF16, F32 = moe.MOE_BF16, moe.MOE_F32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(moe.LIB_PATH):
        from paper_2607_08782_amd import build
        build.build()
    return moe.load_library()


def _caller(fn, names, **ok):
    assert set(names) == set(ok)

    def call(**kw):
        a = dict(ok, **kw)
        return fn(*[a[n] for n in names])
    return call


def test_conversions(lib):
    for fn, names in ((lib.moe_quantize_int8, "m dtype rows cols q s stream"),
                      (lib.moe_dequantize_int8, "q s rows cols dtype m stream")):
        call = _caller(fn, names.split(), m=FAKE, dtype=BF16, rows=4, cols=100, q=FAKE, s=FAKE, stream=None)
        assert call(dtype=2) == ARG and call(rows=-1) == ARG and call(cols=0) == ARG
        assert call(m=None) == ARG and call(q=None) == ARG and call(s=None) == ARG
        assert call(m=ODD) == ARG and call(q=ctypes.c_void_p(0x1008)) == ARG and call(s=ODD) == ARG
        assert call(dtype=F32, m=ctypes.c_void_p(0x1002)) == ARG
        assert call(cols=1 << 28) == SHAPE and call(rows=1 << 60) == SHAPE
        assert call(rows=0, m=None, q=None, s=None) == moe.MOE_OK


def _groups(n, value=0x1000):
    return ctypes.cast((ctypes.c_void_p * max(n, 1))(*[value] * n), ctypes.c_void_p)


def test_grouped_ffn(lib):
    names = "xq xs T row_token offsets n_groups n_shared w13 s13 w2 s2 d f cap y ws ws_bytes stream".split()
    call = _caller(lib.moe_grouped_ffn_int8, names, xq=FAKE, xs=FAKE, T=16, row_token=FAKE, offsets=FAKE,
                   n_groups=3, n_shared=0, w13=_groups(3), s13=_groups(3), w2=_groups(3), s2=_groups(3), d=128,
                   f=96, cap=20, y=FAKE, ws=ctypes.c_void_p(0x100000), ws_bytes=BIG, stream=None)
    for kw in (dict(T=-1), dict(d=0), dict(f=0), dict(cap=-1), dict(n_groups=0), dict(n_groups=129),
               dict(n_shared=-1), dict(n_shared=127), dict(n_shared=1, row_token=None), dict(offsets=None),
               dict(w13=None), dict(s13=None), dict(w2=None), dict(s2=None), dict(xq=None), dict(xs=None),
               dict(y=None), dict(xq=ctypes.c_void_p(0x1008)), dict(xs=ODD), dict(y=ctypes.c_void_p(0x1008)),
               dict(w13=_groups(3, 0x1008)), dict(s2=_groups(3, 0x1002)), dict(w2=_groups(3, 0)),
               dict(T=1 << 31), dict(cap=1 << 31), dict(cap=0x7fffffff, n_shared=1)):
        assert call(**kw) == ARG, kw
    for kw in (dict(d=100), dict(d=(1 << 17) + 8), dict(f=(1 << 17) + 1), dict(T=1 << 24),
               dict(d=1 << 17, f=1 << 13), dict(d=1 << 16, f=1 << 15), dict(row_token=None), dict(ws=None),
               dict(ws=ctypes.c_void_p(0x100010)),
               dict(ws_bytes=lib.moe_grouped_ffn_int8_ws_bytes(20, 128, 96, 3) - 1)):
        assert call(**kw) == SHAPE, kw
    # nothing to do: no workspace, no rows
    assert call(cap=0, T=0, xq=None, xs=None, y=None, ws=None, ws_bytes=0) == moe.MOE_OK
    assert lib.moe_grouped_ffn_int8_ws_bytes(-1, 1, 1, 1) == 0
    assert lib.moe_grouped_ffn_int8_ws_bytes(10, 128, 96, 3) >= 10 * (128 * 3 + 4)


def test_norm(lib):
    names = "x residual dtype weight eps T d h y rstd q s stream".split()
    call = _caller(lib.moe_rmsnorm, names, x=FAKE, residual=FAKE, dtype=BF16, weight=FAKE, eps=1e-6, T=4, d=64,
                   h=ctypes.c_void_p(0x2000), y=ctypes.c_void_p(0x3000), rstd=FAKE, q=FAKE, s=FAKE, stream=None)
    for kw in (dict(dtype=2), dict(T=-1), dict(d=0), dict(x=None), dict(weight=None), dict(h=None), dict(q=None),
               dict(s=None), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(y=ctypes.c_void_p(0x2000)), dict(x=ODD), dict(residual=ODD), dict(weight=ODD), dict(h=ODD),
               dict(y=ODD), dict(rstd=ODD), dict(q=ctypes.c_void_p(0x1008)), dict(s=ODD)):
        assert call(**kw) == ARG, kw
    assert call(d=1 << 22) == SHAPE and call(T=1 << 31) == SHAPE
    assert call(T=0, x=None, weight=None, residual=None, h=None) == moe.MOE_OK


def test_norm_gradient(lib):
    names = "dy h dtype weight rstd add T d dh dw ws ws_bytes stream".split()
    call = _caller(lib.moe_rmsnorm_backward, names, dy=FAKE, h=FAKE, dtype=BF16, weight=FAKE, rstd=FAKE, add=FAKE,
                   T=4, d=64, dh=FAKE, dw=FAKE, ws=ctypes.c_void_p(0x100000), ws_bytes=BIG, stream=None)
    for kw in (dict(dtype=2), dict(T=-1), dict(d=0), dict(dy=None), dict(h=None), dict(weight=None),
               dict(rstd=None), dict(dy=ODD), dict(h=ODD), dict(add=ODD), dict(dh=ODD), dict(dw=ODD),
               dict(rstd=ODD)):
        assert call(**kw) == ARG, kw
    for kw in (dict(d=1 << 22), dict(T=1 << 31), dict(ws=None), dict(ws=ctypes.c_void_p(0x100010)),
               dict(ws_bytes=lib.moe_rmsnorm_backward_ws_bytes(BF16, 4, 64) - 1)):
        assert call(**kw) == SHAPE, kw
    assert call(dh=None, dw=None, ws=None) == moe.MOE_OK
    assert lib.moe_rmsnorm_backward_ws_bytes(BF16, -1, 64) == 0


def test_balance(lib):
    names = "logits idx mask T E k counts sums n loss ws ws_bytes stream".split()
    call = _caller(lib.moe_balance_loss, names, logits=FAKE, idx=FAKE, mask=None, T=4, E=16, k=2, counts=FAKE,
                   sums=FAKE, n=FAKE, loss=FAKE, ws=ctypes.c_void_p(0x100000), ws_bytes=BIG, stream=None)
    for kw in (dict(T=-1), dict(E=0), dict(E=257), dict(k=0), dict(k=17), dict(k=17, E=20), dict(T=1 << 30),
               dict(logits=None), dict(idx=None), dict(counts=None), dict(sums=None), dict(n=None),
               dict(loss=None), dict(logits=ODD), dict(idx=ODD), dict(loss=ODD)):
        assert call(**kw) == ARG, kw
    for kw in (dict(ws=None), dict(ws=ctypes.c_void_p(0x100010)),
               dict(ws_bytes=lib.moe_balance_loss_ws_bytes(4, 16) - 1)):
        assert call(**kw) == SHAPE, kw
    assert lib.moe_balance_loss_ws_bytes(4, 0) == 0
    names = "logits mask counts n T E k scale out stream".split()
    call = _caller(lib.moe_balance_loss_backward, names, logits=FAKE, mask=None, counts=FAKE, n=FAKE, T=4, E=16,
                   k=2, scale=1.0, out=FAKE, stream=None)
    for kw in (dict(T=-1), dict(E=257), dict(k=0), dict(k=17, E=30), dict(logits=None), dict(counts=None),
               dict(n=None), dict(out=None), dict(out=ODD), dict(counts=ODD)):
        assert call(**kw) == ARG, kw
    assert call(T=0, logits=None, out=None) == moe.MOE_OK


def test_gradient_norm_and_clipping(lib):
    ptrs = (ctypes.c_void_p * 2)(0x1000, 0x2000)
    sizes, types = (ctypes.c_int64 * 2)(5, 1 << 20), (ctypes.c_int * 2)(F32, BF16)
    call = _caller(lib.moe_grad_norm, "g sizes types n norm ws ws_bytes stream".split(), g=ptrs, sizes=sizes,
                   types=types, n=2, norm=FAKE, ws=ctypes.c_void_p(0x100000), ws_bytes=BIG, stream=None)
    clip = _caller(lib.moe_clip_grads, "g sizes types n norm most out stream".split(), g=ptrs, sizes=sizes,
                   types=types, n=2, norm=FAKE, most=1.0, out=ptrs, stream=None)
    for c in (call, clip):
        for kw in (dict(n=-1), dict(g=None), dict(sizes=None), dict(types=None), dict(norm=None), dict(norm=ODD),
                   dict(g=(ctypes.c_void_p * 2)(0x1000, None)), dict(g=(ctypes.c_void_p * 2)(0x1002, 0x2000)),
                   dict(sizes=(ctypes.c_int64 * 2)(-1, 4)), dict(types=(ctypes.c_int * 2)(F32, 2))):
            assert c(**kw) == ARG, kw
        assert c(sizes=(ctypes.c_int64 * 2)(1 << 45, 4)) == SHAPE
    assert call(ws=None) == SHAPE and call(ws=ctypes.c_void_p(0x100010)) == SHAPE
    assert call(ws_bytes=lib.moe_grad_norm_ws_bytes(sizes, 2) - 1) == SHAPE
    for kw in (dict(most=-1.0), dict(most=float("nan")), dict(out=None),
               dict(out=(ctypes.c_void_p * 2)(0x1000, None)), dict(out=(ctypes.c_void_p * 2)(0x1000, 0x2001))):
        assert clip(**kw) == ARG, kw
    assert clip(n=0, norm=None, out=None) == moe.MOE_OK
    assert lib.moe_grad_norm_ws_bytes((ctypes.c_int64 * 2)(-1, 4), 2) == 0
