"""Grouped FFN of 8-bit experts (marked `gpu`) against its definition in float64.

Tolerance, per output.  The sums of products are whole numbers and exact.  a and b keep three
roundings of 2^-24 (the sum to fp32, two scales); SiLU adds those of an exponential whose
argument is off by 2^-24 |a| and a division, the product one more: h is within
(16 + 2 |a|) 2^-24 of its value.  Where that interval holds a boundary between two bf16 values
the stored h may be either, and the 8-bit value, which lies within half a step of it, may differ
by a step and the 2^-8 of h; a row whose largest |h| is such a place may differ so in every
value.  y then keeps three fp32 roundings and one to bf16 (2^-8).
"""
import numpy as np
import pytest
import torch

from oracle import int8 as oi
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

    def mk(r, c):
        w = torch.randn(r, c, generator=g, device="cuda") * std
        return moe.moe_quantize_int8(w * torch.exp(0.3 * torch.randn(r, 1, generator=g, device="cuda")))
    return [mk(2 * f, d) for _ in range(n)], [mk(d, f) for _ in range(n)]


def _numbers(pair, cols):
    return pair[0].cpu().numpy()[:, :cols].astype(np.float64), pair[1].double().cpu().numpy()


def _expected(xq, sx, w13, w2, f):
    """(y, tolerance) of one group's rows."""
    ab = (xq @ w13[0].T) * sx[:, None] * w13[1]
    a, b = ab[:, :f], ab[:, f:]
    with np.errstate(over="ignore"):
        h = a / (1 + np.exp(-a)) * b
    off = np.abs(h) * (16 + 2 * np.abs(a)) * 2.0 ** -24
    hb = oi.bf16(h.astype(np.float32))
    ends = [oi.bf16((h + s * off).astype(np.float32)) for s in (-1, 1)]
    may = (ends[0] != hb) | (ends[1] != hb)
    codes, sh = oi.quantize_rows(hb)
    top = np.abs(hb).max(1, keepdims=True)
    near = np.maximum(np.abs(ends[0]), np.abs(ends[1])) >= top * (1 - 2.0 ** -8)
    may |= (may & near).any(1, keepdims=True)
    step = sh[:, None] * 1.01 + np.abs(hb) * 2.0 ** -7
    q = codes[:, :f].astype(np.float64)
    y = (q @ w2[0].T) * sh[:, None].astype(np.float64) * w2[1]
    tol = (2.0 ** -8 + 2.0 ** -22) * np.abs(y) + (may * step) @ np.abs(w2[0] * w2[1][:, None]).T
    return y, tol


def _run(sizes, d, f, T, *, gather=True, n_shared=0, seed=0, cap=None, x=None, std=0.05):
    """One call over groups of these sizes; every row checked, and that rows past the last
    group's keep their contents."""
    rng = np.random.RandomState(seed)
    n = len(sizes)
    w13, w2 = _experts(n_shared + n, d, f, seed, std)
    table = moe.Int8WeightTable(w13, w2, d, f)
    N = int(sum(sizes))
    cap = N + 3 if cap is None else cap
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    if x is None:
        x = torch.randn(T if gather else cap, d, generator=torch.Generator().manual_seed(seed)).bfloat16()
    xq, sx = moe.moe_quantize_int8(x.cuda())
    rows = n_shared * T + cap
    if gather:
        token = [np.arange(T)] * n_shared + [np.sort(rng.choice(T, s, replace=False)) for s in sizes]
        token = np.concatenate(token + [np.full(cap - N, 0)]).astype(np.int32)
        row_token = torch.from_numpy(token).cuda()
    else:
        token, row_token = np.arange(cap), None
    y = torch.full((rows + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((moe.moe_grouped_ffn_int8_ws_bytes(rows, d, f, n_shared + n) + 256,), 0xFF,
                    dtype=torch.uint8, device="cuda")
    moe.moe_grouped_ffn_int8(xq, sx, torch.from_numpy(offsets).cuda(), table, row_token=row_token,
                             n_shared=n_shared, cap_rows=cap, y_perm=y, ws=ws[:-256])
    torch.cuda.synchronize()
    assert (ws[-256:] == 0xFF).all()
    got = y.double().cpu().numpy()
    xv, sv = _numbers((xq, sx), d)
    starts = [s * T for s in range(n_shared)] + [n_shared * T + o for o in offsets[:-1]]
    for i, (start, size) in enumerate(zip(starts, [T] * n_shared + list(sizes))):
        if size == 0:
            continue
        t = token[start:start + size]
        want, tol = _expected(xv[t], sv[t], _numbers(w13[i], d), _numbers(w2[i], f), f)
        off = np.abs(got[start:start + size] - want)
        bad = ~(off <= tol)
        assert not bad.any(), (i, np.argwhere(bad)[:5], (off / np.maximum(tol, 1e-30)).max())
    assert (got[n_shared * T + N:] == 7.0).all()
    return y


@pytest.mark.parametrize("sizes,d,f,T", [
    ([1], 128, 32, 1), ([1], 8, 1, 1), ([1, 0, 1], 256, 96, 1), ([0, 0], 64, 64, 4),
    ([5, 0, 16, 1, 11], 1000, 328, 16), ([17, 32, 0, 3], 136, 200, 33), ([64, 63, 1], 2048, 1408, 64),
    ([40, 7], 4096, 1024, 50), ([3, 2], 512, 4500, 5), ([65, 2, 128], 384, 257, 130), ([9, 1], 24, 131, 9),
    ([500, 115, 0, 260], 512, 640, 777), ([256, 257, 255, 1, 0, 513], 256, 384, 600),
    ([129], 1920, 72, 129), ([1000, 3], 640, 128, 1000), ([300] * 6, 128, 128, 300), ([700, 129], 40, 520, 700),
    # few strips, and few tiles, over a long K: slices of it
    ([20, 1], 264, 4100, 20), ([70, 0, 300, 1], 512, 4224, 310), ([650, 30], 264, 8200, 700),
    # a token alone, two tokens: hidden rows quantized by the strips, also past what LDS holds
    ([1, 0, 1, 1], 520, 1000, 1), ([2, 1], 64, 15000, 2), ([2, 2], 128, 20000, 2),
    # wide strips of a long K that go round from another step each, of other widths by the rounds
    ([20, 7], 2104, 4590, 27), ([1], 4096, 1000, 1), ([2, 0, 1], 2304, 648, 2), ([30, 61], 2304, 4660, 64),
    # waves side by side that share a long K's rows: one to all of their row blocks, columns past the end
    # of which most or all waves lie, slices of K
    ([33, 1, 0, 49], 2304, 2312, 50), ([64, 17, 32], 4096, 72, 64), ([40, 100, 7], 2056, 3000, 100),
    ([97, 128], 2304, 2600, 128), ([40], 8, 9000, 40), ([36, 3], 24, 3000, 36), ([90], 2104, 1, 90),
    # a long K and as many tokens, but few rows a group on average
    ([3, 0, 9, 16, 1, 2, 5, 33], 2304, 2400, 50), ([0, 64, 1, 0, 18, 0, 0, 2], 2104, 4200, 64),
])
def test_groups(sizes, d, f, T):
    say("[ffn int8]", sizes, d, f, T)
    _run(sizes, d, f, T, seed=d + f)


@pytest.mark.parametrize("sizes,d,f", [([3, 0, 9], 264, 160), ([70, 300, 1], 512, 192), ([0, 0], 128, 64)])
def test_packaged_rows(sizes, d, f):
    say("[ffn int8 packaged]", sizes, d, f)
    _run(sizes, d, f, 0, gather=False, seed=3)


@pytest.mark.parametrize("sizes,d,f,T,n_shared", [([2, 0, 5], 256, 96, 6, 2), ([100, 40], 128, 256, 140, 1),
                                                  ([], 256, 64, 5, 1), ([300, 2], 384, 128, 310, 3)])
def test_shared_leading_groups(sizes, d, f, T, n_shared):
    say("[ffn int8 shared]", sizes, d, f, T, n_shared)
    _run(sizes, d, f, T, n_shared=n_shared, seed=5)


@pytest.mark.parametrize("d,f", [(512, 1408), (1000, 328), (256, 4500), (2304, 4660)])
def test_a_row_has_the_same_bits_in_every_batch(d, f):
    """Whatever kernels a batch takes: alone (strips that quantize), in a few rows (strips), in many
    (tiles of both sizes, slices of K)."""
    say("[ffn int8 batches]", d, f)
    g = torch.Generator().manual_seed(d)
    xq, sx = moe.moe_quantize_int8(torch.randn(5000, d, generator=g).bfloat16().cuda())
    w13, w2 = _experts(1, d, f, 3)
    table = moe.Int8WeightTable(w13, w2, d, f)

    def run(n):
        off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        return moe.moe_grouped_ffn_int8(xq[:n], sx[:n], off, table)
    want = run(5000)
    for n in (1, 2, 3, 16, 17, 33, 64, 65, 90, 128, 300, 2000):
        assert torch.equal(run(n), want[:n]), n


@pytest.mark.parametrize("T,n,d,f", [(1, 40, 256, 12000), (2, 21, 256, 12000), (40, 300, 2304, 3000),
                                     (100, 290, 2304, 3000)])
def test_a_group_that_names_a_token_more_than_once(T, n, d, f):
    """More rows in a group than tokens: every one is computed."""
    xq, sx = moe.moe_quantize_int8(torch.randn(T, d, generator=torch.Generator().manual_seed(4)).cuda())
    w13, w2 = _experts(2, d, f, 3)
    table = moe.Int8WeightTable(w13, w2, d, f)
    one = [moe.moe_grouped_ffn_int8(xq, sx, torch.tensor([0, T * (s == 0), T], dtype=torch.int32, device="cuda"), table)
           for s in (0, 1)]
    token = torch.tensor([i % T for i in range(n)] * 2, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
    y = moe.moe_grouped_ffn_int8(xq, sx, off, table, row_token=token, cap_rows=2 * n)
    for s in (0, 1):
        assert torch.equal(y[s * n:(s + 1) * n], one[s][token[:n].long()])


@pytest.mark.parametrize("T,sizes", [(7, [3, 0, 7]), (40, [33, 40]), (300, [299, 10])])
def test_zero_rows_and_large_values(T, sizes):
    say("[ffn int8 values]", T)
    d, f = 256, 128
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(2))
    x[0] = 0.0
    x[1] *= 1e4                                     # gates past the range of exp
    x[2] *= 1e-6
    _run(sizes, d, f, T, x=x.bfloat16(), seed=8)


@pytest.mark.parametrize("T,sizes", [(9, [4, 9, 2]), (70, [64, 40]), (400, [350, 20])])
def test_rows_that_are_not_finite_keep_to_themselves(T, sizes):
    say("[ffn int8 nonfinite]", T)
    d, f = 384, 200
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(9)).bfloat16()
    bad = [1, T // 2, T - 1]
    dirty = x.clone()
    dirty[bad[0], 5] = float("nan")
    dirty[bad[1], d - 1] = float("inf")
    dirty[bad[2]] *= 3e36                           # h past what bf16 holds
    w13, w2 = _experts(len(sizes), d, f, 4)
    table = moe.Int8WeightTable(w13, w2, d, f)
    rng = np.random.RandomState(1)
    token = np.concatenate([np.sort(rng.choice(T, s, replace=False)) for s in sizes]).astype(np.int32)
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    out = [moe.moe_grouped_ffn_int8(*moe.moe_quantize_int8(v.cuda()), off, table,
                                    row_token=torch.from_numpy(token).cuda(),
                                    cap_rows=len(token)).float().cpu().numpy() for v in (x, dirty)]
    hit = np.isin(token, bad)
    assert hit.any() and np.isnan(out[1][hit]).all()
    np.testing.assert_array_equal(out[1][~hit], out[0][~hit])


@pytest.mark.parametrize("T", [5, 200])
def test_largest_sums(T):
    """Every code at its largest, of one sign: sums of 127 x 127 K, and of 127 x -128 K at the longest
    K there is, the largest that a product has."""
    d, f = 8, 1 << 17
    full = lambda rows, cols, v: torch.full((rows, moe.int8_cols(cols)), v, dtype=torch.int8, device="cuda")
    one = lambda n, v: torch.full((n,), v, dtype=torch.float32, device="cuda")
    table = moe.Int8WeightTable([(full(2 * f, d, 127), one(2 * f, 1e-4))], [(full(d, f, -128), one(d, 1e-6))], d, f)
    xq, sx = full(T, d, 127), one(T, 1e-3)
    xq[:, d:] = 0
    off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    y = moe.moe_grouped_ffn_int8(xq, sx, off, table).double().cpu().numpy()
    a = 127.0 * 127.0 * 8 * 1e-3 * 1e-4
    h = float(oi.bf16(np.float32([a / (1 + np.exp(-a)) * a]))[0])
    want = -128.0 * 127.0 * f * float(np.float32(h) / np.float32(127)) * 1e-6
    assert np.abs(y - want).max() <= 2.0 ** -7 * abs(want)


@pytest.mark.parametrize("T,sizes", [(3, [3, 2]), (40, [40, 3]), (500, [480, 100, 1])])
def test_the_same_bits_every_time_on_another_stream_and_from_a_graph(T, sizes):
    say("[ffn int8 repeat]", T)
    d, f = 512, 320
    w13, w2 = _experts(len(sizes), d, f, 6)
    table = moe.Int8WeightTable(w13, w2, d, f)
    xq, sx = moe.moe_quantize_int8(torch.randn(T, d, device="cuda").bfloat16())
    token = torch.cat([torch.arange(s) for s in sizes]).int().cuda()
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    ws = moe.workspace(moe.moe_grouped_ffn_int8_ws_bytes(len(token), d, f, len(sizes)), "cuda")
    y = torch.zeros(len(token), d, dtype=torch.bfloat16, device="cuda")
    call = lambda **kw: moe.moe_grouped_ffn_int8(xq, sx, off, table, row_token=token, cap_rows=len(token), **kw)
    ref = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            got = call()
            side.synchronize()
            assert torch.equal(got, ref)
    got = call(stream=side)
    side.synchronize()
    assert torch.equal(got, ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(y_perm=y, ws=ws)
    for n in range(4):
        fresh = moe.moe_quantize_int8(torch.randn(T, d, device="cuda").bfloat16())
        xq.copy_(fresh[0])
        sx.copy_(fresh[1])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, call()), n


def test_codes_and_scales_of_the_quantized_table():
    d, f = 136, 72
    g = torch.Generator(device="cuda").manual_seed(1)
    w13 = [torch.randn(2 * f, d, generator=g, device="cuda").bfloat16() for _ in range(2)]
    w2 = [torch.randn(d, f, generator=g, device="cuda").bfloat16() for _ in range(2)]
    t = moe.Int8WeightTable.quantized(w13, w2)
    assert len(t) == 2 and (t.d, t.f) == (d, f)
    for (q, s), w in zip(t.w13 + t.w2, w13 + w2):
        want, scale = oi.quantize_rows(w.float().cpu().numpy())
        np.testing.assert_array_equal(q.cpu().numpy(), want)
        np.testing.assert_array_equal(s.cpu().numpy(), scale)


def test_refusals():
    d, f = 128, 64
    w13, w2 = _experts(2, d, f, 0)
    table = moe.Int8WeightTable(w13, w2, d, f)
    xq, sx = moe.moe_quantize_int8(torch.zeros(4, d, device="cuda"))
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    token = torch.zeros(4, dtype=torch.int32, device="cuda")
    call = moe.moe_grouped_ffn_int8
    with pytest.raises(ValueError, match="xq must be"):
        call(xq.float(), sx, off, table)
    with pytest.raises(ValueError, match="xq must be"):
        call(xq[:, :64], sx, off, table)
    with pytest.raises(ValueError, match="x_scale must be"):
        call(xq, sx[:3], off, table)
    with pytest.raises(ValueError, match="group_offsets"):
        call(xq, sx, off[:2], table)
    with pytest.raises(ValueError, match="cap_rows"):
        call(xq, sx, off, table, row_token=token)
    with pytest.raises(ValueError, match="row_token must hold"):
        call(xq, sx, off, table, row_token=token, cap_rows=5)
    with pytest.raises(ValueError, match="y_perm must hold"):
        call(xq, sx, off, table, y_perm=torch.zeros(3, d, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(moe.MoeError, match="workspace"):
        call(xq, sx, off, table, ws=torch.zeros(512, dtype=torch.uint8, device="cuda"))
    with pytest.raises(moe.MoeError, match="shape"):
        call(xq, sx, off, table, cap_rows=5)         # without a row map, more rows than xq has
    with pytest.raises(ValueError, match="w13 codes"):
        moe.Int8WeightTable([(w13[0][0][:, :64], w13[0][1])], w2[:1], d, f)
    with pytest.raises(ValueError, match="w2 scales"):
        moe.Int8WeightTable(w13[:1], [(w2[0][0], w2[0][1].double())], d, f)
    with pytest.raises(ValueError, match="pair"):
        moe.Int8WeightTable([], [], d, f)
