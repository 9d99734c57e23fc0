"""The norm over many gradients and their clipping (marked `gpu`).

The norm against float64 (summed there in another order: both are within n 2^-53 of the sum) within
the one rounding to fp32, 2^-24; the clipped values bit for bit against fp32 products by the factor
that the GPU's own norm gives."""
import math

import numpy as np
import pytest
import torch

from oracle import int8 as oi
from paper_2607_08782_amd import moe

from parity import np32, say

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


def _grads(shapes, seed, std=1e-2):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(s, generator=g) * std).to(dt).cuda() for s, dt in shapes]


def _clipped(g, factor):
    v = np32(g) * np.float32(factor)
    return oi.bf16(v) if g.dtype == BF else v


def _check(grads, share):
    """Norm and clipping to `share` of the norm, beside and in place."""
    exact = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    most = share * exact
    out = [torch.full_like(g, 7.0) for g in grads]
    table = moe.GradTable(grads, out=out)
    norm = moe.moe_grad_norm(table)
    assert abs(float(norm) - exact) <= 2.0 ** -23 * exact
    keep = [g.clone() for g in grads]
    assert moe.moe_clip_grads(table, norm, most) is table.out
    torch.cuda.synchronize()
    n = np.float32(float(norm))
    factor = np.float32(1.0) if n <= np.float32(most) else np.float32(most) / n
    for g, k, o in zip(grads, keep, out):
        assert torch.equal(g, k)
        np.testing.assert_array_equal(np32(o), _clipped(g, factor))
    here = moe.GradTable(grads)
    again = moe.moe_grad_norm(here)
    assert torch.equal(again, norm)
    moe.moe_clip_grads(here, again, most)
    for g, o in zip(grads, out):
        assert torch.equal(g, o)


@pytest.mark.parametrize("shapes", [
    [((1,), F)], [((1,), BF)], [((3, 5), BF), ((7,), F)],
    [((64, 2048), F), ((64,), F), ((2048,), F)] * 27,
    [((2816, 512), BF), ((512, 1408), BF), ((33, 77), F)],
    [((0,), F), ((5,), F), ((0, 4), BF), ((16384,), F), ((16385,), BF), ((16383,), F)],
    [((i % 13 + 1,), BF if i % 3 else F) for i in range(300)],
    [((40000 + i,), F) for i in range(100)],
])
@pytest.mark.parametrize("share", [0.3, 1.2, 0.0])
def test_norm_and_clipping(shapes, share):
    say("[clip]", len(shapes), share)
    _check(_grads(shapes, len(shapes)), share)


def test_elements_that_are_not_16_byte_aligned():
    flat = [torch.randn(50001, generator=torch.Generator().manual_seed(i)).to(dt).cuda() for i, dt in enumerate((F, BF))]
    _check([t[1:] for t in flat], 0.5)
    # an output that is not, of a gradient that is
    g = flat[0][:50000]
    out = torch.zeros(50001, device="cuda")[1:]
    table = moe.GradTable([g], out=[out])
    norm = moe.moe_grad_norm(table)
    moe.moe_clip_grads(table, norm, 1.0)
    np.testing.assert_array_equal(np32(out), _clipped(g, np.float32(1.0) / np.float32(float(norm))))


def test_large_and_small_values():
    """Squares past what fp32 holds, and below."""
    for v in (1e30, 1e-30, 3e38):
        g = torch.full((1000,), v, device="cuda")
        norm = moe.moe_grad_norm(moe.GradTable([g]))
        want = float(np.float32(v)) * math.sqrt(1000)
        assert (math.isinf(float(norm)) if want > 3.41e38 else abs(float(norm) - want) <= 2.0 ** -23 * want)


def test_gradients_that_are_not_finite():
    g = _grads([((100,), F), ((50,), BF)], 1)
    g[1][7] = float("inf")
    table = moe.GradTable(g)
    norm = moe.moe_grad_norm(table)
    assert math.isinf(float(norm))
    moe.moe_clip_grads(table, norm, 1.0)
    assert not g[0].any() and torch.isnan(g[1][7]) and not g[1][:7].any()
    g = _grads([((100,), F), ((50,), BF)], 1)
    g[0][3] = float("nan")
    table = moe.GradTable(g)
    norm = moe.moe_grad_norm(table)
    assert math.isnan(float(norm))
    moe.moe_clip_grads(table, norm, 1.0)
    assert torch.isnan(g[0]).all() and torch.isnan(g[1]).all()


def test_zeros_and_nothing():
    g = [torch.zeros(10, device="cuda")]
    norm = moe.moe_grad_norm(moe.GradTable(g))
    assert float(norm) == 0.0
    moe.moe_clip_grads(moe.GradTable(g), norm, 0.0)
    assert not g[0].any()
    out = torch.full((1,), 5.0, device="cuda")
    assert float(moe.moe_grad_norm(moe.GradTable([]), norm=out)) == 0.0
    moe.moe_clip_grads(moe.GradTable([]), out, 1.0)
    with pytest.raises(ValueError, match="needs norm"):
        moe.moe_grad_norm(moe.GradTable([]))


def test_a_tensor_past_2_31_elements():
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=BF, device="cuda")
    g[-3:] = torch.tensor([3.0, 0.0, 4.0])
    g[0] = 12.0
    table = moe.GradTable([g])
    norm = moe.moe_grad_norm(table)
    assert float(norm) == 13.0
    moe.moe_clip_grads(table, norm, 6.5)
    assert float(g[0]) == 6.0 and g[-3:].tolist() == [1.5, 0.0, 2.0]


def test_the_same_bits_on_another_stream_and_captured():
    grads = _grads([((300, 500), F), ((70000,), BF), ((9,), F)], 2)
    out = [torch.zeros_like(g) for g in grads]
    table = moe.GradTable(grads, out=out)
    ws = moe.workspace(moe.moe_grad_norm_ws_bytes(table), "cuda")
    norm = moe.moe_grad_norm(table)
    moe.moe_clip_grads(table, norm, 0.5)
    want = [norm.clone()] + [o.clone() for o in out]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    again = moe.moe_grad_norm(table, stream=side)
    moe.moe_clip_grads(table, again, 0.5, stream=side)
    side.synchronize()
    for a, b in zip([again] + out, want):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        moe.moe_grad_norm(table, norm=norm, ws=ws)
        moe.moe_clip_grads(table, norm, 0.5)
    for n in range(4):
        for t, f in zip(grads, _grads([(t.shape, t.dtype) for t in grads], 30 + n)):
            t.copy_(f)
        g.replay()
        torch.cuda.synchronize()
        got = [norm.clone()] + [o.clone() for o in out]
        eager = moe.moe_grad_norm(table)
        moe.moe_clip_grads(table, eager, 0.5)
        for a, b in zip(got, [eager] + out):
            assert torch.equal(a, b), n


def test_refusals():
    g = _grads([((10,), F), ((4,), BF)], 0)
    with pytest.raises(TypeError):
        moe.GradTable([g[0].half()])
    with pytest.raises(ValueError, match="one output"):
        moe.GradTable(g, out=g[:1])
    with pytest.raises(ValueError, match="types and shapes"):
        moe.GradTable(g, out=[g[0], g[1].float()])
    with pytest.raises(ValueError, match="contiguous"):
        moe.GradTable([torch.zeros(4, 6, device="cuda").t()])
    with pytest.raises(ValueError, match="GPU"):
        moe.GradTable([torch.zeros(4)])
    table = moe.GradTable(g)
    norm = moe.moe_grad_norm(table)
    for most in (-1.0, float("nan")):
        with pytest.raises(moe.MoeError, match="argument"):
            moe.moe_clip_grads(table, norm, most)
    with pytest.raises(ValueError, match="norm must be"):
        moe.moe_clip_grads(table, norm.double(), 1.0)
    with pytest.raises(moe.MoeError, match="workspace"):
        moe.moe_grad_norm(table, ws=torch.zeros(8, dtype=torch.uint8, device="cuda"))


def test_a_gradient_that_is_listed_twice():
    """It counts twice in the norm; clipped in place it would be scaled twice, or once, by chance."""
    g = _grads([((9000,), F), ((0,), F), ((0,), F)], 3)
    table = moe.GradTable(g + g[:1])
    norm = moe.moe_grad_norm(table)
    assert abs(float(norm) - 2 ** 0.5 * float(moe.moe_grad_norm(moe.GradTable(g)))) <= 2 ** -22 * float(norm)
    with pytest.raises(ValueError, match="twice"):
        moe.moe_clip_grads(table, norm, 1.0)
    out = [torch.empty_like(t) for t in g + g[:1]]
    moe.moe_clip_grads(moe.GradTable(g + g[:1], out=out), norm, 1.0)
    assert torch.equal(out[0], out[-1]) and torch.equal(out[0], g[0] * (1.0 / norm))
    moe.moe_clip_grads(moe.GradTable(g), norm, 1.0)
    assert torch.equal(g[0], out[0])
