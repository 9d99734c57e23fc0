"""The 8-bit FFN's 256 x 256 down tiles without slices of K, the long prompt's own kernel (marked
`gpu`): at 2^24 outputs and more over a K of fewer than 64 steps of 64 columns, at 2^25 over any."""
import numpy as np
import pytest
import torch

from paper_2607_08782_amd import moe

from parity import say
from test_gpu_ffn_int8 import _expected, _experts, _numbers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


@pytest.mark.parametrize("sizes,d,f", [
    ([4097], 4096, 64),                              # one group, a row past its tiles
    ([2000, 0, 1, 1900, 300], 4096, 136),            # ragged ones, one without rows
    ([16500, 290], 1000, 200),                       # columns that end inside a tile
    ([8200], 4096, 4100),                            # a long K, too many outputs to cut it
])
def test_down_product_of_many_rows(sizes, d, f):
    """Every row has the bits that a call over 1500 rows or fewer gives it, by other tiles (what a row's
    bits do not depend on); rows around the tiles' borders are within the definition's tolerance."""
    say("[int8 large]", sizes, d, f)
    rows, E = sum(sizes), len(sizes)
    assert rows * d >= (1 << 25 if moe.int8_cols(f) >= 4096 else 1 << 24)
    w13, w2 = _experts(E, d, f, rows)
    x = torch.randn(rows, d, generator=torch.Generator().manual_seed(rows)).bfloat16()
    q, s = moe.moe_quantize_int8(x.cuda())
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32), device="cuda")
    y = torch.full((rows + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_grouped_ffn_int8(q, s, off, moe.Int8WeightTable(w13, w2, d, f), cap_rows=rows, y_perm=y)
    torch.cuda.synchronize()
    assert (y[rows] == 7.0).all()
    at = 0
    for e, size in enumerate(sizes):
        one = moe.Int8WeightTable([w13[e]], [w2[e]], d, f)
        for first in range(0, size, 1500):
            n = min(1500, size - first)
            part = slice(at + first, at + first + n)
            few = moe.moe_grouped_ffn_int8(q[part], s[part].clone(), torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                                           one)
            assert torch.equal(y[part], few), (e, first)
        if size:
            some = sorted({r for b in (0, 256, size // 512 * 256, size) for r in range(b - 4, b + 4) if 0 <= r < size})
            r = torch.tensor(some, device="cuda") + at
            want, tol = _expected(*_numbers((q[r], s[r]), d), _numbers(w13[e], d), _numbers(w2[e], f), f)
            bad = ~(np.abs(y[r].double().cpu().numpy() - want) <= tol)
            assert not bad.any(), (e, np.argwhere(bad)[:5])
        at += size
