"""MXFP4 matrices on the GPU (marked `gpu`) against the plain reference: codes and scale
bytes bit for bit, values exactly, at every rounding boundary and over the whole
exponent range, for every layout of the rows.
"""
import numpy as np
import pytest
import torch

from oracle import mxfp4 as om
from paper_2607_08782_amd import moe

from parity import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


def _np(t):
    return t.float().cpu().numpy()


def _check(x):
    rows, cols = x.shape
    q, s = moe.moe_quantize_mxfp4(x.cuda())
    code, byte = om.encode(_np(x))
    np.testing.assert_array_equal(s.cpu().numpy(), byte)
    np.testing.assert_array_equal(q.cpu().numpy(), om.pack(code))
    want = om.values(code, byte, cols)
    got = moe.moe_dequantize_mxfp4(q, s, cols, dtype=torch.float32)
    np.testing.assert_array_equal(got.double().cpu().numpy(), want)
    low = moe.moe_dequantize_mxfp4(q, s, cols)
    assert torch.equal(low.cpu().nan_to_num(1.5), torch.from_numpy(want).float().bfloat16().nan_to_num(1.5))


def _boundaries(dtype):
    mid = (om.GRID[1:] + om.GRID[:-1]) / 2
    p = np.concatenate([om.GRID, mid, [7.0, 7.96875]]).astype(np.float32)
    t = torch.from_numpy(p).to(dtype)
    up = torch.nextafter(t, torch.tensor(100.0, dtype=dtype))
    down = torch.nextafter(t, torch.tensor(0.0, dtype=dtype))
    p = torch.cat([t, up, down]).float().numpy()
    return np.concatenate([p, -p])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(64, 1024), (33, 1000), (40, 77), (19, 128), (7, 33), (5, 1),
                                       (1, 8), (300, 264)])
def test_codes_at_every_boundary_and_scale(dtype, rows, cols):
    say("[mxfp4]", dtype, rows, cols)
    rng = np.random.RandomState(rows + cols)
    v = rng.choice(_boundaries(dtype), size=(rows, cols)).astype(np.float32)
    v[:, ::32] = 4.0                                     # the block's scale is 1 ...
    # ... times a power of two: from where values and scales are subnormal to the largest
    e = rng.randint(-135, 125, size=(rows, cols // 32 + 1)).repeat(32, 1)[:, :cols]
    v = np.ldexp(v.astype(np.float64), e)
    v = np.where(np.abs(v) < 3e38, v, 1.0).astype(np.float32)
    _check(torch.from_numpy(v).to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 4096), (1000, 515), (129, 2048), (3, 14336)])
def test_random_rows(dtype, rows, cols):
    say("[mxfp4 random]", dtype, rows, cols)
    g = torch.Generator().manual_seed(rows * cols)
    x = torch.randn(rows, cols, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))
    _check(x.to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [256, 200, 203])
def test_blocks_that_are_zero_or_not_finite(dtype, cols):
    say("[mxfp4 special]", dtype, cols)
    x = torch.randn(9, cols, generator=torch.Generator().manual_seed(cols))
    x[0] = 0.0
    x[1, 32:64] = -0.0
    x[2, 5] = float("inf")
    x[3, 40] = float("-inf")
    x[4, 70] = float("nan")
    x[5, cols - 1] = float("nan")
    x[6] = 1e-39                                         # subnormal as a float
    x[7, :32] = torch.tensor(3.3e38)
    x[8] = float("inf")
    _check(x.to(dtype))


def test_rows_at_any_address_and_nothing_outside_is_written():
    say("[mxfp4 address]")
    rows, cols = 37, 264
    flat = torch.randn(rows * cols + 3, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    for shift in (1, 2, 3):
        x = flat[shift:shift + rows * cols].view(rows, cols)
        P = moe.mxfp4_cols(cols)
        qb = torch.full((rows * P // 2 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        sb = torch.full((rows * P // 32 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        q, s = qb[32:-32].view(rows, -1), sb[32:-32].view(rows, -1)
        moe.moe_quantize_mxfp4(x, q=q, scales=s)
        code, byte = om.encode(_np(x))
        np.testing.assert_array_equal(q.cpu().numpy(), om.pack(code))
        np.testing.assert_array_equal(s.cpu().numpy(), byte)
        for b in (qb, sb):
            assert (b[:32] == 0xA5).all() and (b[-32:] == 0xA5).all()
        yb = torch.full((rows * cols + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
        y = yb[shift:shift + rows * cols].view(rows, cols)
        moe.moe_dequantize_mxfp4(q, s, cols, out=y)
        np.testing.assert_array_equal(y.double().cpu().numpy(), om.values(code, byte, cols))
        assert (yb[:shift] == 7).all() and (yb[shift + rows * cols:] == 7).all()


def test_no_rows():
    x = torch.empty(0, 100, device="cuda")
    q, s = moe.moe_quantize_mxfp4(x)
    assert q.shape == (0, 64) and s.shape == (0, 4)
    assert moe.moe_dequantize_mxfp4(q, s, 100).shape == (0, 100)


def test_on_another_stream():
    x = torch.randn(512, 1024, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        q, s = moe.moe_quantize_mxfp4(x)
        y = moe.moe_dequantize_mxfp4(q, s, 1024, dtype=torch.float32)
    side.synchronize()
    np.testing.assert_array_equal(y.double().cpu().numpy(), om.rounded(x.cpu().numpy()))


@pytest.mark.parametrize("rows,cols", [(1, 5), (33, 128), (70, 4500), (1000, 264), (31, 1024), (64, 14336)])
def test_step_major_layout(rows, cols):
    P = moe.mxfp4_cols(cols)
    q = torch.randint(0, 256, (rows, P // 2), dtype=torch.uint8, device="cuda")
    s = torch.randint(0, 256, (rows, P // 32), dtype=torch.uint8, device="cuda")
    codes, words = moe.moe_mxfp4_lay_out(q, s, cols)
    np.testing.assert_array_equal(codes.cpu().numpy(),
                                  q.cpu().numpy().reshape(rows, P // 128, 64).transpose(1, 0, 2))
    np.testing.assert_array_equal(words.cpu().numpy().view(np.uint32), s.cpu().numpy().view(np.uint32).T)
