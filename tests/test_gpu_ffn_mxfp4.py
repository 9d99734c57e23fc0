"""Grouped FFN of MXFP4 experts (marked `gpu`) against its definition in float64.

Tolerance, per output: bf16's unit roundoff (8 significant bits: 2^-8 of it), 2^-20 of
the sum of magnitudes for fp32 accumulation over up to 2^14 terms, and for every hidden
value that lies within 1e-5 of a rounding boundary of its 4-bit grid (or whose block's
largest magnitude lies so near a power of two) what the output would change by if it fell
to the other side.
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


def _experts(n, d, f, seed, std=0.05):
    g = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda r, c: moe.moe_quantize_mxfp4(torch.randn(r, c, generator=g, device="cuda") * std)
    return [mk(2 * f, d) for _ in range(n)], [mk(d, f) for _ in range(n)]


def _values(pair, cols):
    return om.values(om.unpack(pair[0].cpu().numpy()), pair[1].cpu().numpy(), cols)


def _expected(xq, w13, w2, f):
    """(y, tolerance) of one group's rows."""
    a, b = xq @ w13[:f].T, xq @ w13[f:].T
    with np.errstate(over="ignore"):
        h = a / (1 + np.exp(-a)) * b
    h = h.astype(np.float32).astype(np.float64)
    code, byte = om.encode(h)
    hq = om.values(code, byte, f)
    P = om.padded(f)
    pad = np.zeros((h.shape[0], P))
    pad[:, :f] = np.abs(h)
    blocks = pad.reshape(-1, P // 32, 32)
    scale = np.exp2(byte.astype(np.float64) - 127)[..., None]
    u = blocks / scale
    mid = (om.GRID[1:] + om.GRID[:-1]) / 2
    near = np.abs(u[..., None] - mid).min(-1) < 1e-5 * np.maximum(u, 0.25)
    may = np.where(near, 2.0 * scale, 0.0)
    most = blocks.max(-1, keepdims=True)
    frac = np.frexp(most)[0]
    edge = (np.minimum(np.abs(frac - 0.5), np.abs(frac - 1.0)) < 1e-5) & (most > 0)
    may = np.maximum(may, np.where(edge, blocks, 0.0)).reshape(h.shape[0], P)[:, :f]
    y = hq @ w2.T
    tol = 2.0 ** -8 * np.abs(y) + 2.0 ** -20 * (np.abs(hq) @ np.abs(w2).T) + may @ np.abs(w2).T
    return y, tol


def _run(sizes, d, f, T, *, gather=True, n_shared=0, seed=0, cap=None, x=None):
    """One call over groups of these sizes; every row checked, and that rows past the last
    group's keep their contents."""
    rng = np.random.RandomState(seed)
    n = len(sizes)
    w13, w2 = _experts(n_shared + n, d, f, seed)
    table = moe.MxWeightTable(w13, w2, d, f)
    N = int(sum(sizes))
    cap = N + 3 if cap is None else cap
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    if x is None:
        x = torch.randn(T if gather else cap, d, generator=torch.Generator().manual_seed(seed)).bfloat16()
    rows = n_shared * T + cap
    if gather:
        token = [np.arange(T)] * n_shared + [np.sort(rng.choice(T, s, replace=False)) for s in sizes]
        token = np.concatenate(token + [np.full(cap - N, 0)]).astype(np.int32)
        row_token = torch.from_numpy(token).cuda()
    else:
        token, row_token = np.arange(cap), None
    y = torch.full((rows + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((moe.moe_grouped_ffn_mxfp4_ws_bytes(x.shape[0], rows, d, f, n_shared + n) + 256,),
                    0xFF, dtype=torch.uint8, device="cuda")
    moe.moe_grouped_ffn_mxfp4(x.cuda(), torch.from_numpy(offsets).cuda(), table, row_token=row_token,
                              n_shared=n_shared, cap_rows=cap, y_perm=y, ws=ws[:-256])
    torch.cuda.synchronize()
    assert (ws[-256:] == 0xFF).all()
    got = y.double().cpu().numpy()
    xq = om.rounded(x.float().numpy())
    starts = [s * T for s in range(n_shared)] + [n_shared * T + o for o in offsets[:-1]]
    for i, (start, size) in enumerate(zip(starts, [T] * n_shared + list(sizes))):
        if size == 0:
            continue
        want, tol = _expected(xq[token[start:start + size]], _values(w13[i], d), _values(w2[i], f), f)
        off = np.abs(got[start:start + size] - want)
        bad = ~(off <= tol)
        assert not bad.any(), (i, np.argwhere(bad)[:5], (off / np.maximum(tol, 1e-30)).max())
    assert (got[n_shared * T + N:] == 7.0).all()
    return y


@pytest.mark.parametrize("sizes,d,f,T", [
    ([1], 128, 32, 1), ([1], 8, 1, 1), ([1, 0, 1], 256, 96, 1), ([0, 0], 64, 64, 4),
    ([5, 0, 16, 1, 11], 1000, 328, 16), ([17, 32, 0, 3], 136, 200, 33), ([64, 63, 1], 2048, 1408, 64),
    ([40, 7], 4096, 1024, 50), ([3, 2], 512, 4500, 5), ([65, 2, 128], 384, 257, 130),
    ([500, 115, 0, 260], 512, 640, 777), ([256, 257, 255, 1, 0, 513], 256, 384, 600),
    ([129], 1920, 72, 129), ([1000, 3], 640, 128, 1000), ([300] * 6, 128, 128, 300),
])
def test_groups(sizes, d, f, T):
    say("[ffn mxfp4]", sizes, d, f, T)
    _run(sizes, d, f, T, seed=d + f)


@pytest.mark.parametrize("sizes,d,f", [([3, 0, 9], 264, 160), ([70, 300, 1], 512, 192), ([0, 0], 128, 64)])
def test_packaged_rows(sizes, d, f):
    say("[ffn mxfp4 packaged]", sizes, d, f)
    _run(sizes, d, f, 0, gather=False, seed=3)


@pytest.mark.parametrize("sizes,d,f,T,n_shared", [([2, 0, 5], 256, 96, 6, 2), ([100, 40], 128, 256, 140, 1),
                                                  ([], 256, 64, 5, 1), ([300, 2], 384, 128, 310, 3)])
def test_shared_leading_groups(sizes, d, f, T, n_shared):
    say("[ffn mxfp4 shared]", sizes, d, f, T, n_shared)
    _run(sizes, d, f, T, n_shared=n_shared, seed=5)


@pytest.mark.parametrize("T,sizes", [(9, [4, 9, 2]), (400, [350, 20])])
def test_rows_that_are_not_finite_keep_to_themselves(T, sizes):
    say("[ffn mxfp4 nonfinite]", T)
    d, f = 384, 200
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(9)).bfloat16()
    rows = np.arange(T) if T < 20 else None
    bad = [1, T // 2, T - 1]
    dirty = x.clone()
    dirty[bad[0], 5] = float("nan")
    dirty[bad[1], d - 1] = float("inf")
    dirty[bad[2], 0] = float("-inf")
    w13, w2 = _experts(len(sizes), d, f, 4)
    table = moe.MxWeightTable(w13, w2, d, f)
    rng = np.random.RandomState(1)
    token = np.concatenate([np.sort(rng.choice(T, s, replace=False)) for s in sizes]).astype(np.int32)
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    out = [moe.moe_grouped_ffn_mxfp4(v.cuda(), off, table, row_token=torch.from_numpy(token).cuda(),
                                     cap_rows=len(token)).float().cpu().numpy() for v in (x, dirty)]
    hit = np.isin(token, bad)
    assert hit.any() and np.isnan(out[1][hit]).all()
    np.testing.assert_array_equal(out[1][~hit], out[0][~hit])


@pytest.mark.parametrize("T,sizes", [(7, [3, 0, 7]), (300, [299, 10])])
def test_zero_rows_and_large_values(T, sizes):
    say("[ffn mxfp4 values]", T)
    d, f = 256, 128
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(2))
    x[0] = 0.0
    x[1] *= 1e4                                     # gates past the range of exp
    x[2] *= 1e-6
    _run(sizes, d, f, T, x=x.bfloat16(), seed=8)


@pytest.mark.parametrize("T,sizes", [(40, [40, 3]), (500, [480, 100, 1])])
def test_the_same_bits_every_time_and_on_another_stream(T, sizes):
    say("[ffn mxfp4 repeat]", T)
    d, f = 512, 320
    w13, w2 = _experts(len(sizes), d, f, 6)
    table = moe.MxWeightTable(w13, w2, d, f)
    x = torch.randn(T, d, device="cuda").bfloat16()
    token = torch.cat([torch.arange(s) for s in sizes]).int().cuda()
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    call = lambda: moe.moe_grouped_ffn_mxfp4(x, off, table, row_token=token, cap_rows=len(token))
    ref = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            got = call()
            side.synchronize()
            assert torch.equal(got, ref)
