"""Gradients of a batch of which no row is here (marked `gpu`): the rows' tensor is empty."""
import pytest
import torch

from paper_2607_08782_amd import moe

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(5, 64), (5, 33), (5000, 512)])
def test_tokens_without_rows(T, d, dtype):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    k = 3
    dy = torch.randn(T, d, device="cuda").to(dtype)
    rows = torch.empty(0, d, dtype=dtype, device="cuda")
    here = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    dy_perm, dgate = moe.moe_combine_backward(dy, rows, here, torch.rand(T, k, device="cuda"),
                                              dgate=torch.full((T, k), 7.0, device="cuda"))
    assert dy_perm.shape == (0, d) and not dgate.any()
    assert not moe.moe_permute_backward(rows, here, dx=torch.full_like(dy, 7.0)).any()
    assert torch.equal(moe.moe_permute_backward(rows, here, dx_add=dy), dy)
