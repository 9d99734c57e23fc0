"""Grouped FFN of MXFP4 experts (marked `gpu`) at the sizes that choose its kernels: token
rows quantized by the strips or before them, tiles of 256 x 256 with ragged, half-filled and
halved last ones, and more tiles a workgroup than it lists at once.

The checks and their tolerance are those of test_gpu_ffn_mxfp4.py: every row against the
definition in float64.
"""
import numpy as np
import pytest
import torch

from oracle import mxfp4 as om
from paper_2607_08782_amd import moe

from parity import say
from test_gpu_ffn_mxfp4 import _expected, _experts, _run, _values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


@pytest.mark.parametrize("sizes,d,f,T", [
    ([16, 3, 0, 9], 2048, 96, 16), ([13, 1], 2040, 64, 13),          # by the strips
    ([16, 3, 0, 9], 4096, 96, 16), ([9, 2], 4104, 40, 9),            # before them
    ([1], 4104, 2500, 1), ([8, 8], 4096, 2048, 8),                   # few steps a wave, and more
])
def test_few_rows(sizes, d, f, T):
    say("[ffn mxfp4 few rows]", sizes, d, f, T)
    _run(sizes, d, f, T, seed=11)
    _run(sizes, d, f, 0, gather=False, cap=sum(sizes), seed=12)


@pytest.mark.parametrize("sizes,d,f,T", [
    ([700, 129, 0, 385, 128], 384, 12512, 700),       # gate/up: whole tiles and half-filled ones
    ([1000, 400], 256, 12544, 1000),                  # what is left of a round in halves
    ([700, 1, 300, 343, 40], 12544, 160, 700),        # down
    ([1000, 400], 12544, 128, 1000),
])
def test_large_tiles(sizes, d, f, T):
    say("[ffn mxfp4 large tiles]", sizes, d, f, T)
    _run(sizes, d, f, T, seed=13)


@pytest.mark.parametrize("d,f,cap", [(128, 8192, 1500), (256, 8192, 1500), (384, 8192, 1500), (512, 8192, 1500),
                                     (128, 16640, 1500), (256, 16640, 1500), (384, 16640, 1500)])
def test_products_of_fewer_steps_than_the_ring(d, f, cap):
    """Token rows of the next tile, several tiles a workgroup, 1 to 4 steps a tile."""
    say("[ffn mxfp4 short products]", d, f)
    _run([700, 130, 601], d, f, 900, cap=cap, seed=17)


def test_a_buffer_much_longer_than_the_rows():
    say("[ffn mxfp4 long buffer]")
    _run([768], 128, 12544, 900, cap=1400, seed=14)
    _run([0, 0], 128, 12544, 900, cap=1400, seed=14)


def test_more_tiles_than_a_workgroup_lists():
    say("[ffn mxfp4 many tiles]")
    n, d, f, T, cap = 120, 128, 8192, 300, 2100
    rng = np.random.RandomState(5)
    sizes = rng.randint(0, 4, n)
    sizes[7], sizes[60], sizes[119] = 300, 257, 130
    token = np.concatenate([np.sort(rng.choice(T, s, replace=False)) for s in sizes])
    N = len(token)
    assert N <= cap
    (w13,), (w2,) = _experts(1, d, f, 15)
    table = moe.MxWeightTable([w13] * n, [w2] * n, d, f)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(15)).bfloat16()
    row_token = torch.zeros(cap, dtype=torch.int32)
    row_token[:N] = torch.from_numpy(token)
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    y = torch.full((cap, d), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_grouped_ffn_mxfp4(x.cuda(), off, table, row_token=row_token.cuda(), cap_rows=cap, y_perm=y)
    got = y.double().cpu().numpy()
    want, tol = _expected(om.rounded(x.float().numpy()), _values(w13, d), _values(w2, f), f)
    bad = ~(np.abs(got[:N] - want[token]) <= tol[token])
    assert not bad.any(), np.argwhere(bad)[:5]
    assert (got[N:] == 7.0).all()


@pytest.mark.parametrize("T", [20, 300])
def test_rows_far_into_a_long_buffer(T):
    """Two steps of hidden codes lie 1.1 GB apart: offsets past 31 bits."""
    say("[ffn mxfp4 far rows]", T)
    d, f, cap = 8, 256, 17 << 20
    n, start = T - 3, cap - T
    (w13,), (w2,) = _experts(1, d, f, 16)
    table = moe.MxWeightTable([w13], [w2], d, f)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(16)).bfloat16()
    row_token = torch.zeros(cap, dtype=torch.int32, device="cuda")
    row_token[start:start + n] = torch.arange(n, dtype=torch.int32, device="cuda")
    off = torch.tensor([start, start + n], dtype=torch.int32, device="cuda")
    y = torch.full((cap, d), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_grouped_ffn_mxfp4(x.cuda(), off, table, row_token=row_token, cap_rows=cap, y_perm=y)
    got = y[start:].double().cpu().numpy()
    want, tol = _expected(om.rounded(x.float().numpy()), _values(w13, d), _values(w2, f), f)
    assert (np.abs(got[:n] - want[:n]) <= tol[:n]).all()
    assert (got[n:] == 7.0).all() and bool((y[:start] == 7.0).all())
