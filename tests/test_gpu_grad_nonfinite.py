"""Gates' gradients that are not finite, through the router's products (marked `gpu`): sums
are what the same sums in 32 bits are, infinities with their signs, and no other entry
changes."""
import numpy as np
import pytest
import torch

from paper_2607_08782_amd import moe

from parity import say
from test_gpu_grad import DT, _np, _rand, _routing

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


def _sum64(a, b):
    """a [n, K] times b [K, m] with infinities and NaN as sums have them, term by term."""
    out = np.zeros((a.shape[0], b.shape[1]))
    with np.errstate(invalid="ignore"):
        for i in range(a.shape[1]):
            out += a[:, i, None] * b[i]
    return out


@pytest.mark.parametrize("T,E,k,d", [(1, 4, 2, 8), (70, 24, 3, 136), (300, 65, 2, 64), (130, 200, 4, 72)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("renorm", [True, False])
def test_infinite_dlogits(T, E, k, d, dtype, renorm):
    """An infinite dgate: NaN for its expert's score, infinities for the token's others."""
    say("[route grad infinite]", T, E, k, d, dtype, renorm)
    logits, idx, gate = _routing(T, E, k, renorm, T + E, spread=1.0)
    dgate, w = _rand((T, k), 1), _rand((E, d), 3, dtype, 0.02)
    # no zeros or overflows: an infinity times any entry has a sign
    x = (_rand((T, d), 2) * 0.5 + torch.sign(_rand((T, d), 2))).to(DT[dtype])
    kw = dict(logits=None if renorm else logits.cuda(), renorm=renorm)
    call = lambda: moe.moe_route_topk_backward(dgate.cuda(), gate, idx, x.cuda(), w.cuda(), **kw)
    clean = call()
    t = T // 2
    dgate[t, 0] = float("inf")
    dl, dx, dw, dbias = call()
    e0 = int(idx[t, 0])
    hit = idx[t].tolist() if renorm else range(E)
    assert np.isnan(_np(dl)[t, e0]) and np.isneginf(_np(dl)[t, [e for e in hit if e != e0]]).all()
    for got, want in ((dw, _sum64(_np(dl).T, _np(x))), (dbias, _np(dl).sum(0)), (dx, _sum64(_np(dl), _np(w)))):
        got = _np(got)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        np.testing.assert_array_equal(np.where(np.isinf(got), np.sign(got), 0),
                                      np.where(np.isinf(want), np.sign(want), 0))
    rows = np.arange(T) != t
    experts = ~np.isin(np.arange(E), list(hit))
    for got, ref, keep in ((dl, clean[0], rows), (dx, clean[1], rows), (dw, clean[2], experts),
                           (dbias, clean[3], experts)):
        np.testing.assert_array_equal(_np(got)[keep], _np(ref)[keep])


@pytest.mark.parametrize("E,k", [(2, 2), (40, 2), (150, 2)])
@pytest.mark.parametrize("renorm", [True, False])
def test_scores_gradients_past_the_range_to_an_infinity(E, k, renorm):
    """Two gates' gradients whose difference overflows: an infinite dlogit beside finite ones
    (no NaN among the token's), so dx has infinities with signs too."""
    T, d = 33, 64
    say("[route grad overflow]", E, renorm)
    logits = torch.zeros(T, E)
    logits[:, 0], logits[:, 1] = 12.0, 10.0
    _, idx, gate = moe.moe_route_topk(None, None, None, k, logits=logits.cuda(), logits_in=True, renorm=renorm)
    dgate = _rand((T, k), 1)
    dgate[4] = torch.tensor([3e38, -3e38])           # mean 2.3e38: the second's difference is -inf
    x, w = _rand((T, d), 2, "bf16"), _rand((E, d), 3, "bf16", 0.02)
    dl, dx, dw, _ = moe.moe_route_topk_backward(dgate.cuda(), gate, idx, x.cuda(), w.cuda(),
                                                logits=None if renorm else logits.cuda(), renorm=renorm)
    dl = _np(dl)
    assert np.isneginf(dl[4, 1]) and np.isfinite(np.delete(dl, 4, 0)).all() and np.isfinite(dl[4, 0])
    want = -np.sign(_np(w)[1]) * np.where(_np(w)[1] == 0, np.nan, np.inf)
    np.testing.assert_array_equal(_np(dx)[4], want)
    want = -np.sign(_np(x)[4]) * np.where(_np(x)[4] == 0, np.nan, np.inf)
    np.testing.assert_array_equal(_np(dw)[1], want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,renorm", [(40, False), (40, True), (200, False)])
def test_rows_and_weights_that_are_not_finite(E, renorm, dtype):
    """They reach the sums that they enter, and no others."""
    T, k, d = 100, 3, 136
    say("[route grad operands]", E, renorm, dtype)
    logits, idx, gate = _routing(T, E, k, renorm, 9, spread=1.0)
    dgate, x, w = _rand((T, k), 1), _rand((T, d), 2, dtype), _rand((E, d), 3, dtype, 0.02)
    call = lambda x, w: moe.moe_route_topk_backward(dgate.cuda(), gate, idx, x.cuda(), w.cuda(), renorm=renorm,
                                                    logits=None if renorm else logits.cuda())
    clean = call(x, w)
    x2, w2 = x.clone(), w.clone()
    x2[7, 5], x2[99, 64], x2[50, 135] = float("inf"), float("-inf"), float("nan")
    e = int(idx[3, 0])
    w2[e, 9], w2[e, 70] = float("inf"), float("nan")
    _, dx, dw, _ = call(x2, w2)
    used = _np(clean[0]) != 0
    for got, ref, cols, rows in ((dx, clean[1], [9, 70], [used[:, e]] * 2),
                                 (dw, clean[2], [5, 64, 135], [used[7], used[99], used[50]])):
        got, ref = _np(got), _np(ref)
        keep = ~np.isin(np.arange(d), cols)
        np.testing.assert_array_equal(got[:, keep], ref[:, keep])
        for c, r in zip(cols, rows):
            assert not np.isfinite(got[r, c]).any()
