"""Every MXFP4 element under every scale byte (marked `gpu`), those that no quantization gives
among them: exact, infinite past the range of a float, NaN under byte 255."""
import numpy as np
import pytest
import torch

from oracle import mxfp4 as om
from paper_2607_08782_amd import moe

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_all_codes_under_all_scales(dtype):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    code = np.zeros((256, 128), np.uint8)
    code[:, :16] = np.arange(16)
    byte = np.zeros((256, 4), np.uint8)
    byte[:, 0] = np.arange(256)
    got = moe.moe_dequantize_mxfp4(torch.from_numpy(om.pack(code)).cuda(), torch.from_numpy(byte).cuda(), 128,
                                   dtype=dtype)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(om.values(code, byte, 128).astype(np.float32)).to(dtype)
    assert torch.equal(got.cpu().isnan(), want.isnan())
    assert torch.equal(got.cpu()[:255], want[:255])      # all but byte 255's
    assert int(want.isinf().sum()) == 12                 # 4 and 6 under 253; 2 to 6 under 254, both signs
