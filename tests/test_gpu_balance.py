"""The balance loss and its gradient (marked `gpu`) against their definition in float64, and
against differences.

Tolerances.  A score's p keeps the rounding of score - top (2^-24 of it, which the exponential
turns into as much of p), an exponential's 2 ulp (4 times 2^-24), a sum over E scores of at most 15
additions in a lane and 4 between lanes, a reciprocal and a product: (|l - top| + 26) 2^-24 of p, and
of any sum of p the largest of these; prob_sum adds chains of at most ceil(T / 256) (16 at least)
tokens and 34 more.  The gradient is f p (c - sum p c): its two terms keep p's error, the counts'
rounding and ten more.
"""
import numpy as np
import pytest
import torch

from paper_2607_08782_amd import moe

from parity import say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


def _batch(T, E, k, seed, padding=0.0):
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn(T, E, generator=g) + torch.linspace(1.0, -1.0, E)
    idx = torch.topk(logits, k, 1)[1].int()
    mask = torch.rand(T, generator=g) >= padding if padding else None
    return logits, idx, mask


def _check(logits, idx, mask, scale=1.0):
    T, E = logits.shape
    k = idx.shape[1]
    c = lambda t: None if t is None else t.cuda()
    L, I, M = c(logits), c(idx), c(mask)
    loss, counts, prob_sum, n = moe.moe_balance_loss(L, I, mask=M)
    dl = moe.moe_balance_loss_backward(L, counts, n, k, scale=scale, mask=M)
    torch.cuda.synchronize()
    live = np.ones(T, bool) if mask is None else mask.numpy() != 0
    l = logits.double().numpy()[live]
    top = l.max(1, keepdims=True) if len(l) else l[:, :1]
    p = np.exp(l - top)
    p /= p.sum(1, keepdims=True)
    want = np.bincount(idx.numpy()[live].ravel(), minlength=E)
    N = int(live.sum())
    assert int(n) == N
    np.testing.assert_array_equal(counts.cpu().numpy(), want)
    fin = np.where(np.isfinite(l), np.abs(l - top), 0.0)
    rho = (fin.max(1, keepdims=True) + 26) * U if N else np.zeros((0, 1))
    S = p.sum(0)
    tol = (p * rho).sum(0) + (max(-(-T // 256), 16) + 34) * U * S
    assert (np.abs(prob_sum.double().cpu().numpy() - S) <= tol).all()
    exact = E * (want / (k * N) * S / N).sum() if N else 0.0
    slack = E * (want / (k * N) * tol / N).sum() + 4 * U * exact if N else 0.0
    assert abs(float(loss) - exact) <= slack
    full = np.zeros((T, E))
    bound = np.zeros((T, E))
    if N:
        f = scale * E / (k * N * N)
        centred = want - want.mean()
        dot = (p * centred).sum(1, keepdims=True)
        full[live] = f * p * (centred - dot)
        size = np.abs(centred) + 1.0 + (p * (np.abs(centred) + 1.0)).sum(1, keepdims=True)
        bound[live] = abs(f) * p * size * (2 * rho + 16 * U) + 1e-44
    off = np.abs(dl.double().cpu().numpy() - full)
    assert (off <= bound).all()
    return loss, counts, prob_sum, n, dl


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (0, 16, 4), (7, 8, 8), (64, 24, 3), (333, 60, 4), (777, 64, 6),
                                   (1000, 128, 8), (5000, 128, 8), (300, 200, 16), (257, 256, 1), (20000, 9, 2),
                                   (4097, 33, 5)])
@pytest.mark.parametrize("padding", [0.0, 0.4])
def test_loss_and_gradient(T, E, k, padding):
    say("[balance]", T, E, k, padding)
    _check(*_batch(T, E, k, T + E, padding), scale=0.25)


def test_what_the_masked_tokens_hold_is_not_read():
    logits, idx, mask = _batch(500, 40, 4, 3, 0.5)
    mask[7], mask[499] = False, False
    ref = _check(logits, idx, mask)
    logits[~mask] = float("nan")
    logits[7] = float("inf")
    bad = idx.clone()
    bad[~mask] = 1 << 30
    c = lambda t: t.cuda()
    loss, counts, prob_sum, n = moe.moe_balance_loss(c(logits), c(bad), mask=c(mask))
    dl = moe.moe_balance_loss_backward(c(logits), counts, n, 4, mask=c(mask))
    for a, b in zip((loss, counts, prob_sum, n, dl), ref):
        assert torch.equal(a, b)
    # bytes, and any value but 0
    loss = moe.moe_balance_loss(c(logits), c(bad), mask=c(mask.to(torch.uint8) * 3))[0]
    assert torch.equal(loss, ref[0])


def test_no_token_counts():
    logits, idx, _ = _batch(100, 16, 2, 1)
    out = _check(logits, idx, torch.zeros(100, dtype=torch.bool))
    for t in out:
        assert not t.any()


def test_scores_at_the_edges():
    logits, idx, _ = _batch(64, 12, 2, 2)
    logits[0] = 3e38
    logits[1] = -3e38
    logits[2] = 0.0
    logits[3, 1:] = float("-inf")                    # one expert left
    logits[4, :6] = float("-inf")
    logits[5] *= 60                                  # nearly one-hot
    idx = torch.topk(logits, 2, 1)[1].int()
    _check(logits, idx, None)


def test_even_routing_costs_one_and_all_on_one_expert_costs_more():
    E, k, T = 16, 2, 160
    logits = torch.zeros(T, E)
    idx = torch.stack([torch.arange(T) % E, (torch.arange(T) + 5) % E], 1).int()
    loss, *_, dl = _check(logits, idx, None)
    assert abs(float(loss) - 1.0) <= 8 * U and not dl.any()
    logits[:, 3] = 20.0
    loss = _check(logits, torch.tensor([[3, 4]] * T).int(), None)[0]
    assert float(loss) == pytest.approx(E / 2, rel=1e-4)


def test_gradient_against_differences():
    T, E, k = 6, 10, 2
    logits, idx, mask = _batch(T, E, k, 9, 0.3)
    counts = torch.bincount(idx[mask].flatten().long(), minlength=E).double()
    n = int(mask.sum())

    def loss(l):
        p = torch.softmax(l[mask].double(), 1).sum(0)
        return float(E * (counts * p).sum() / (k * n * n))
    _, c, _, m = moe.moe_balance_loss(logits.cuda(), idx.cuda(), mask=mask.cuda())
    dl = moe.moe_balance_loss_backward(logits.cuda(), c, m, k, mask=mask.cuda()).cpu()
    base = logits.double()
    for i in range(T * E):
        step = torch.zeros(T * E, dtype=torch.float64)
        step[i] = 1e-5
        num = (loss(base + step.view(T, E)) - loss(base - step.view(T, E))) / 2e-5
        assert abs(float(dl.flatten()[i]) - num) <= 1e-6


def test_counts_of_two_gpus_batches():
    """Two batches' counts, sums and tokens added: the loss and gradient of them as one batch."""
    logits, idx, _ = _batch(300, 24, 3, 5)
    cut = 130
    whole = _check(logits, idx, None)
    parts = [moe.moe_balance_loss(l.contiguous().cuda(), i.contiguous().cuda())
             for l, i in ((logits[:cut], idx[:cut]), (logits[cut:], idx[cut:]))]
    counts, n = parts[0][1] + parts[1][1], parts[0][3] + parts[1][3]
    assert torch.equal(counts, whole[1]) and torch.equal(n, whole[3])
    dl = torch.cat([moe.moe_balance_loss_backward(l.contiguous().cuda(), counts, n, 3)
                    for l in (logits[:cut], logits[cut:])])
    assert torch.equal(dl, whole[4])


def test_in_place_on_another_stream_and_captured():
    T, E, k = 900, 48, 4
    logits, idx, mask = (t.cuda() for t in _batch(T, E, k, 4, 0.2))
    ws = moe.workspace(moe.moe_balance_loss_ws_bytes(T, E), "cuda")

    def both(**kw):
        out = moe.moe_balance_loss(logits, idx, mask=mask, ws=ws, **kw)
        return [*out, moe.moe_balance_loss_backward(logits, out[1], out[3], k, mask=mask, **kw)]
    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(stream=side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    over = logits.clone()
    assert torch.equal(moe.moe_balance_loss_backward(over, want[1], want[3], k, mask=mask, dlogits=over), want[4])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = both()
    for n in range(4):
        fresh = _batch(T, E, k, 50 + n, 0.2)
        for t, f in zip((logits, idx, mask), fresh):
            t.copy_(f)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, both()):
            assert torch.equal(a, b), n


def test_refusals():
    logits, idx, _ = (None if t is None else t.cuda() for t in _batch(8, 16, 2, 0))
    with pytest.raises(ValueError, match="topk_idx must be"):
        moe.moe_balance_loss(logits, idx[:7])
    with pytest.raises(ValueError, match="logits must be"):
        moe.moe_balance_loss(logits.double(), idx)
    for mask in (torch.ones(7, dtype=torch.bool, device="cuda"), torch.ones(8, device="cuda")):
        with pytest.raises(ValueError, match="mask must be"):
            moe.moe_balance_loss(logits, idx, mask=mask)
    with pytest.raises(moe.MoeError, match="argument"):
        moe.moe_balance_loss(logits, torch.zeros(8, 17, dtype=torch.int32, device="cuda"))
    with pytest.raises(moe.MoeError, match="workspace"):
        moe.moe_balance_loss(logits, idx, ws=torch.zeros(64, dtype=torch.uint8, device="cuda"))
    _, counts, _, n = moe.moe_balance_loss(logits, idx)
    with pytest.raises(ValueError, match="counts must be"):
        moe.moe_balance_loss_backward(logits, counts.float(), n, 2)
    with pytest.raises(moe.MoeError, match="argument"):
        moe.moe_balance_loss_backward(logits, counts, n, 0)
