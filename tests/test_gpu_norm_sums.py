"""The norm's weight gradient over many rows (marked `gpu`): what small parts add to a large one is
kept."""
import pytest
import torch

from paper_2607_08782_amd import moe

from parity import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 200, 1000, 2048, 4096, 4100, 9000])
def test_small_parts_beside_a_large_one(dtype, d):
    """n is 1 everywhere; dy is 2^25 in the first row and 1 in 255 others, of other ranges: in 32 bits
    2^25 + 1 is 2^25.  dw is 2^25 + 255, whose fp32 value is 2^25 + 256."""
    say("[dw]", dtype, d)
    T = 4096
    one = torch.ones(T, d, dtype=dtype, device="cuda")
    dy = torch.zeros_like(one)
    dy[16::16] = 1.0
    dy[0] = 2.0 ** 25
    _, dw = moe.moe_rmsnorm_backward(dy, one, one[0].clone(), torch.ones(T, device="cuda"), want_dh=False)
    assert (dw == 2.0 ** 25 + 256).all(), dw[dw != 2.0 ** 25 + 256][:4]
