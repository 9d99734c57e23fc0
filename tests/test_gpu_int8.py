"""Rows in 8-bit integers (marked `gpu`): codes, scales and values bit for bit against
oracle.int8 on the same bf16 / fp32 values."""
import numpy as np
import pytest
import torch

from oracle import int8 as oi
from paper_2607_08782_amd import moe

from parity import np32, say

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


def _check(x):
    rows, cols = x.shape
    q, s = moe.moe_quantize_int8(x)
    y = moe.moe_dequantize_int8(q, s, cols, dtype=x.dtype)
    torch.cuda.synchronize()
    want, scale = oi.quantize_rows(np32(x))
    np.testing.assert_array_equal(s.cpu().numpy(), scale)
    np.testing.assert_array_equal(q.cpu().numpy(), want)
    v = want[:, :cols].astype(np.float32) * scale[:, None]
    np.testing.assert_array_equal(np32(y), oi.bf16(v) if x.dtype == torch.bfloat16 else v)


def _rows(rows, cols, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (0, 64), (7, 72), (5, 100), (300, 256), (1025, 130), (33, 4096),
                                       (3, 20000), (1100, 2048), (2, 127), (4, 129), (1500, 1031)])
def test_rows(dtype, rows, cols):
    say("[int8]", dtype, rows, cols)
    _check(_rows(rows, cols, dtype, rows * 7 + cols).cuda())


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_at_the_edges(dtype):
    x = _rows(24, 264, dtype, 1)
    x[0] = 0.0
    x[1] *= 1e-44                                    # subnormal: the smallest scale
    x[2] *= 1e-38
    x[3, 5] = float("nan")
    x[4, 263] = float("inf")
    x[5, 0] = float("-inf")
    x[6] = torch.arange(264) - 127.0                 # 137 the largest: quotients near ties
    x[7] = (torch.arange(264) % 255 - 127).float()   # scale 1: every code
    x[8] = (torch.arange(264) % 254 - 127).float() + 0.5
    x[8, 0] = 127.0                                  # scale 1: ties, to the even code
    x[9] *= 1e30
    x[10] = 3.3e38
    x[11] = -0.0
    x[12] *= 1e-20
    x[13] = 127 * 2.0 ** -126
    _check(x.cuda())


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_are_not_16_byte_aligned(dtype):
    flat = _rows(1, 9 * 256 + 1, dtype, 5).cuda().flatten()
    x = flat[1:].view(9, 256)
    assert x.is_contiguous() and x.data_ptr() % 16 != 0
    _check(x)


@pytest.mark.parametrize("dtype", DTYPES)
def test_every_quotient_near_a_tie(dtype):
    """Values that lie as near to code + 1/2 as the type allows, over scales of all magnitudes."""
    rng = np.random.RandomState(3)
    top = (2.0 ** rng.randint(-100, 100, 200) * (1 + rng.rand(200))).astype(np.float32)
    top = oi.bf16(top) if dtype == torch.bfloat16 else top
    scale = (top / np.float32(127)).astype(np.float32)
    tie = (scale[:, None].astype(np.float64) * (np.arange(126) + 0.5)).astype(np.float32)
    near = np.stack([tie, np.nextafter(tie, np.float32(0)), np.nextafter(tie, np.float32(np.inf))], 2)
    x = np.concatenate([top[:, None], near.reshape(200, -1), -near.reshape(200, -1)], 1)
    _check(torch.from_numpy(x).to(dtype).cuda())


def test_far_rows():
    """Rows past 2^31 codes, and 2^32 bytes of values."""
    cols, rows = 4096, (1 << 31) // 4096 + 40
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    last = _rows(32, cols, torch.bfloat16, 8)
    x[-32:] = last.cuda()
    q, s = moe.moe_quantize_int8(x)
    y = moe.moe_dequantize_int8(q, s, cols)
    want, scale = oi.quantize_rows(np32(last))
    np.testing.assert_array_equal(q[-32:].cpu().numpy(), want)
    np.testing.assert_array_equal(s[-32:].cpu().numpy(), scale)
    np.testing.assert_array_equal(np32(y[-32:]), oi.bf16(want.astype(np.float32) * scale[:, None]))
    assert not q[:-32].any() and (s[:-32] == 2.0 ** -126).all() and not y[:-32].any()


def test_outputs_of_another_shape_are_refused():
    x = torch.zeros(4, 100, device="cuda")
    new = lambda *shape, dtype=torch.int8: torch.zeros(shape, dtype=dtype, device="cuda")
    with pytest.raises(ValueError, match="q must be"):
        moe.moe_quantize_int8(x, q=new(4, 100))
    with pytest.raises(ValueError, match="scales must be"):
        moe.moe_quantize_int8(x, scales=new(3, dtype=torch.float32))
    with pytest.raises(ValueError, match="q must be"):
        moe.moe_dequantize_int8(new(4, 256), new(4, dtype=torch.float32), 100)
    with pytest.raises(ValueError, match="cols"):
        moe.moe_dequantize_int8(new(4, 128), new(4, dtype=torch.float32), 0)
    with pytest.raises(TypeError):
        moe.moe_quantize_int8(x.half())
    with pytest.raises(ValueError, match="contiguous"):
        moe.moe_quantize_int8(torch.zeros(100, 4, device="cuda").t())
