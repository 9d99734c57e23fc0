"""The norm in front of a layer and its gradient (marked `gpu`) against their definition in
float64, and against differences.

Tolerances.  A sum in fp32 over a row of d values runs over at most C = ceil(d / 64) of them in one
thread and a tree of 10 steps: an error of (C + 10) 2^-24 of the sum of magnitudes.  rstd, whose
squares are summed in 64 bits, keeps at most half of that and 4 roundings; y that, two more
and its own rounding (half a step: eps / 2 of its type).  dw's chains are a range's rows (at most
ceil(T / 512), four at least) and 160 parts.
"""
import numpy as np
import pytest
import torch

from oracle import int8 as oi
from paper_2607_08782_amd import moe

from parity import np32, say

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]
U = 2.0 ** -24
SIZES = [(1, 1), (0, 64), (3, 7), (7, 4096), (333, 1000), (1100, 256), (1030, 2048), (5, 4100), (2, 40000),
         (1500, 130), (64, 8192), (2049, 520), (4, 16392)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


def _rows(T, d, dtype, seed, spread=0.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, d, generator=g) * torch.exp(spread * torch.randn(T, 1, generator=g))).to(dtype).cuda()


def _weight(d, dtype, seed):
    return (1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(seed))).to(dtype).cuda()


def _half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _sum_bound(d):
    return (-(-d // 64) + 10) * U


def _check(x, residual, w, eps, h, y, rstd, q, s):
    """Outputs (None: not wanted) of one call, on these inputs."""
    T, d = x.shape
    if residual is not None:
        assert torch.equal(h, (x.float() + residual.float()).to(x.dtype))
    v = np32(h).astype(np.float64)
    want = 1 / np.sqrt((v * v).mean(1) + eps) if T else np.zeros(0)
    tol = _sum_bound(d) / 2 + 4 * U
    if rstd is not None:
        assert (np.abs(rstd.double().cpu().numpy() - want) <= tol * want).all()
    full = v * want[:, None] * w.double().cpu().numpy()
    if y is not None:
        off = np.abs(y.double().cpu().numpy() - full)
        assert (off <= (tol + 2 * U + _half_step(x.dtype)) * np.abs(full) + 1e-44).all()
        if q is not None:
            again = moe.moe_quantize_int8(y)
            assert torch.equal(again[0], q) and torch.equal(again[1], s)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d", SIZES)
def test_norm(dtype, T, d):
    say("[norm]", dtype, T, d)
    x, r, w = _rows(T, d, dtype, T + d), _rows(T, d, dtype, T + d + 1, 0.0), _weight(d, dtype, d)
    for residual in (None, r):
        keep = x.clone()
        h, y, rstd, q, s = moe.moe_rmsnorm(x, w, residual=residual, want_rstd=True, want_q=True)
        assert torch.equal(x, keep) and (residual is not None or h is x)
        _check(x, residual, w, 1e-6, h, y, rstd, q, s)
        # each output alone is the same
        only_q = moe.moe_rmsnorm(x, w, residual=residual, want_y=False, want_q=True)
        assert only_q[1] is None and only_q[2] is None
        assert torch.equal(only_q[3], q) and torch.equal(only_q[4], s)
        only_y = moe.moe_rmsnorm(x, w, residual=residual)
        assert torch.equal(only_y[1], y) and only_y[3] is None


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d", [(5, 264), (1100, 512), (3, 20000), (6, 77)])
def test_norm_in_place(dtype, T, d):
    """h over x or the residual, y over the other or over x."""
    x, r, w = _rows(T, d, dtype, 1), _rows(T, d, dtype, 2), _weight(d, dtype, 3)
    h, y, _, q, s = moe.moe_rmsnorm(x, w, residual=r, want_q=True)
    plain = moe.moe_rmsnorm(x, w)[1]
    for to_h, to_y in (("x", None), ("r", None), ("x", "r"), ("r", "x"), (None, "x"), (None, "r")):
        b = {"x": x.clone(), "r": r.clone(), None: None}
        got = moe.moe_rmsnorm(b["x"], w, residual=b["r"], h=b[to_h], y=b[to_y], want_q=True)
        for a, c in zip((got[0], got[1], got[3], got[4]), (h, y, q, s)):
            assert torch.equal(a, c), (to_h, to_y)
    over = x.clone()
    assert torch.equal(moe.moe_rmsnorm(over, w, y=over)[1], plain)


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_of_rows_at_the_edges(dtype):
    T, d = 9, 384
    x, w = _rows(T, d, dtype, 4), _weight(d, dtype, 5)
    clean = moe.moe_rmsnorm(x, w, want_rstd=True, want_q=True)
    x[1] = 0.0
    x[2, 7] = float("nan")
    x[3, 0] = float("inf")
    x[4] *= 1e-30                                    # squares vanish: rstd is eps's
    h, y, rstd, q, s = moe.moe_rmsnorm(x, w, want_rstd=True, want_q=True)
    assert not y[1].any() and not q[1].any() and float(rstd[1]) == pytest.approx(1e3, rel=1e-6)
    assert torch.isnan(y[2]).all() and torch.isnan(s[2]) and not q[2].any()
    assert torch.isnan(y[3, 0]) and not y[3, 1:].any() and torch.isnan(s[3])
    assert float(rstd[4]) == pytest.approx(1e3, rel=1e-6)
    _check(x[4:5], None, w, 1e-6, x[4:5], y[4:5], rstd[4:5], q[4:5], s[4:5])
    for a, b in zip((y, rstd, q, s), (clean[1], clean[2], clean[3], clean[4])):
        assert torch.equal(a[5:], b[5:]) and torch.equal(a[0], b[0])
    # eps 0 of a row of zeros: 0 * infinity
    assert torch.isnan(moe.moe_rmsnorm(x[1:2], w, eps=0.0)[1]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1e18, 1e25, 1e36])
@pytest.mark.parametrize("d", [384, 77])
def test_norm_of_rows_whose_squares_pass_32_bits(dtype, scale, d):
    x, w = (_rows(4, d, torch.float32, 8, 0.0) * scale).to(dtype), _weight(d, dtype, 5)
    h, y, rstd, q, s = moe.moe_rmsnorm(x, w, want_rstd=True, want_q=True)
    assert float(y.abs().max()) > 1.0
    _check(x, None, w, 1e-6, x, y, rstd, q, s)


def test_norm_of_rows_that_are_not_16_byte_aligned():
    d = 256
    for dtype in DTYPES:
        flat = _rows(1, 6 * d + 1, dtype, 6).flatten()
        x, w = flat[1:].view(6, d), _weight(d, dtype, 7)
        assert x.data_ptr() % 16
        h, y, rstd, q, s = moe.moe_rmsnorm(x, w, want_rstd=True, want_q=True)
        _check(x, None, w, 1e-6, x, y, rstd, q, s)


def _backward_check(dy, h, w, rstd, add, dh, dw):
    T, d = dy.shape
    n64 = lambda t: t.double().cpu().numpy()
    up, r, v = n64(dy), n64(rstd)[:, None], n64(w)
    n = n64(h) * r
    g = up * v
    mean = (g * n).mean(1, keepdims=True) if T else np.zeros((0, 1))
    extra = n64(add) if add is not None else np.zeros_like(up)
    if dh is not None:
        want = r * (g - n * mean) + extra
        # n, g w, the mean, its product, the difference, r, the addition
        size = np.abs(r * g) + np.abs(r * n) * (np.abs(mean) + np.abs(g * n).mean(1, keepdims=True)
                                                if T else 0.0) + np.abs(extra)
        tol = (_sum_bound(d) + 8 * U) * size + _half_step(dy.dtype) * np.abs(want) + 1e-44
        off = np.abs(n64(dh) - want)
        assert (off <= tol).all(), (off / tol).max()
    if dw is not None:
        chain = max(-(-T // 512), 4) + 160
        off = np.abs(n64(dw) - (up * n).sum(0))
        assert (off <= (chain + 2) * U * np.abs(up * n).sum(0)).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d", SIZES)
def test_gradient(dtype, T, d):
    say("[norm grad]", dtype, T, d)
    h, w = _rows(T, d, dtype, T + d), _weight(d, dtype, d)
    dy, add = _rows(T, d, dtype, T + d + 2, 0.0), _rows(T, d, dtype, T + d + 3, 0.0)
    rstd = moe.moe_rmsnorm(h, w, want_rstd=True)[2]
    dh, dw = moe.moe_rmsnorm_backward(dy, h, w, rstd, dh_add=add)
    _backward_check(dy, h, w, rstd, add, dh, dw)
    bare, same = moe.moe_rmsnorm_backward(dy, h, w, rstd)
    _backward_check(dy, h, w, rstd, None, bare, same)
    assert torch.equal(same, dw)
    one, none = moe.moe_rmsnorm_backward(dy, h, w, rstd, dh_add=add, want_dw=False)
    assert none is None and torch.equal(one, dh)
    none, one = moe.moe_rmsnorm_backward(dy, h, w, rstd, want_dh=False)
    assert none is None and torch.equal(one, dw)
    over = add.clone()
    assert torch.equal(moe.moe_rmsnorm_backward(dy, h, w, rstd, dh_add=over, dh=over)[0], dh)
    assert T or not dw.any()


def test_gradient_against_differences():
    """The loss sum(dy * y) of the norm in float64, a step of 1e-6 up and down."""
    T, d, eps = 5, 24, 1e-3
    g = torch.Generator().manual_seed(0)
    x, w, dy = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((T, d), (d,), (T, d)))

    def loss(x, w):
        return (x / (x.square().mean(1, keepdim=True) + eps).sqrt() * w * dy).sum()
    f = lambda t: t.float().cuda()
    rstd = moe.moe_rmsnorm(f(x), f(w), eps=eps, want_rstd=True)[2]
    dh, dw = moe.moe_rmsnorm_backward(f(dy), f(x), f(w), rstd)
    for t, got in ((x, dh), (w, dw)):
        for i in range(t.numel()):
            step = torch.zeros_like(t).view(-1)
            step[i] = 1e-6
            step = step.view_as(t)
            num = (loss(x + step, w) - loss(x - step, w)) / 2e-6 if t is x else \
                  (loss(x, w + step) - loss(x, w - step)) / 2e-6
            # differences: 1e-12 / 1e-6 of the loss's rounding and third derivatives; fp32: 1e-5
            assert abs(float(got.flatten()[i]) - float(num)) <= 1e-5 * (1 + abs(float(num)))


@pytest.mark.parametrize("T", [3, 1500])
def test_captured_and_on_another_stream(T):
    d = 512
    x, r, w = _rows(T, d, torch.bfloat16, 1), _rows(T, d, torch.bfloat16, 2), _weight(d, torch.bfloat16, 3)
    dy = _rows(T, d, torch.bfloat16, 4)
    ws = moe.workspace(moe.moe_rmsnorm_backward_ws_bytes(moe.MOE_BF16, T, d), "cuda")

    def both(**kw):
        h, y, rstd, q, s = moe.moe_rmsnorm(x, w, residual=r, want_rstd=True, want_q=True, **kw)
        return [h, y, rstd, q, s, *moe.moe_rmsnorm_backward(dy, h, w, rstd, dh_add=dy, ws=ws, **kw)]
    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(stream=side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = both()
    for n in range(4):
        x.copy_(_rows(T, d, torch.bfloat16, 10 + n))
        dy.copy_(_rows(T, d, torch.bfloat16, 20 + n))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, both()):
            assert torch.equal(a, b), n


def test_far_rows():
    """Rows past 2^32 bytes."""
    T, d = (1 << 31) // 4096 + 20, 4096
    x = torch.ones(T, d, dtype=torch.bfloat16, device="cuda")
    last, w = _rows(16, d, torch.bfloat16, 1), _weight(d, torch.bfloat16, 2)
    x[-16:] = last
    want = moe.moe_rmsnorm(last, w, want_rstd=True, want_q=True)
    h, y, rstd, q, s = moe.moe_rmsnorm(x, w, want_rstd=True, want_q=True)
    for a, b in zip((y, rstd, q, s), want[1:]):
        # (short batches sum a row in four waves, long ones in another order)
        assert (a[-16:].double() - b.double()).abs().max() <= (1 if a.dtype == torch.int8 else 2 ** -7 * b.double().abs().max())
    del q, s
    dh, dw = moe.moe_rmsnorm_backward(x, x, w, rstd, dh=y)
    want = moe.moe_rmsnorm_backward(last, last, w, rstd[-16:].contiguous())[0]
    assert (dh[-16:].double() - want.double()).abs().max() <= 2 ** -7 * want.double().abs().max()


def test_refusals():
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    with pytest.raises(ValueError, match="weight must be"):
        moe.moe_rmsnorm(x, w.bfloat16())
    with pytest.raises(ValueError, match="residual must be"):
        moe.moe_rmsnorm(x, w, residual=x[:3])
    with pytest.raises(ValueError, match="x itself"):
        moe.moe_rmsnorm(x, w, h=x)
    with pytest.raises(ValueError, match="together"):
        moe.moe_rmsnorm(x, w, q=torch.zeros(4, 128, dtype=torch.int8, device="cuda"))
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(moe.MoeError, match="argument"):
            moe.moe_rmsnorm(x, w, eps=eps)
    with pytest.raises(moe.MoeError, match="argument"):
        over = x.clone()
        moe.moe_rmsnorm(x, w, residual=x, h=over, y=over)
    with pytest.raises(TypeError):
        moe.moe_rmsnorm(x.half(), w.half())
    r = torch.ones(4, device="cuda")
    with pytest.raises(ValueError, match="rstd must be"):
        moe.moe_rmsnorm_backward(x, x, w, r[:3])
    with pytest.raises(ValueError, match="h must be"):
        moe.moe_rmsnorm_backward(x, x.bfloat16(), w, r)
    with pytest.raises(moe.MoeError, match="workspace"):
        moe.moe_rmsnorm_backward(x, x, w, r, ws=torch.zeros(256, dtype=torch.uint8, device="cuda"))
