"""What masked tokens hold changes no output of the balance loss or its gradient (marked `gpu`): by one
launch (up to 2^14 scores) and by three, for every number of lanes that a token has."""
import pytest
import torch

from paper_2607_08782_amd import moe

from parity import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


@pytest.mark.parametrize("E,k", [(2, 1), (8, 8), (7, 3), (16, 4), (13, 5), (32, 16), (30, 2), (64, 6), (61, 4),
                                 (128, 8), (127, 9), (256, 16), (253, 3)])
@pytest.mark.parametrize("scores", [1 << 10, 1 << 14, (1 << 14) + 1, 1 << 16])
def test_what_masked_tokens_hold(E, k, scores):
    T = scores // E if scores <= 1 << 14 else -(-scores // E)
    assert (T * E <= 1 << 14) == (scores <= 1 << 14)
    say("[masked]", T, E, k)
    g = torch.Generator().manual_seed(T + E)
    logits = torch.randn(T, E, generator=g)
    idx = torch.topk(logits, k, 1)[1].int()
    mask = torch.rand(T, generator=g) < 0.6
    mask[0], mask[T - 1] = False, False
    logits[~mask], idx[~mask] = 0.0, 0

    def run(l, i, m):
        l, i, m = l.cuda(), i.cuda(), m.cuda()
        out = moe.moe_balance_loss(l, i, mask=m)
        over = l.clone()
        dl = moe.moe_balance_loss_backward(l, out[1], out[3], k, mask=m)
        assert torch.equal(moe.moe_balance_loss_backward(over, out[1], out[3], k, mask=m, dlogits=over), dl)
        return [t.cpu() for t in (*out, dl)]
    want = run(logits, idx, mask)
    live = torch.bincount(idx[mask].flatten().long(), minlength=E)
    assert torch.equal(want[1].long(), live) and int(want[3]) == int(mask.sum())
    assert all(torch.isfinite(t).all() for t in want) and not want[4][~mask].any()
    for value, index in ((float("nan"), 1 << 30), (float("inf"), -1), (float("-inf"), -(1 << 31)), (3e38, E)):
        logits[~mask], idx[~mask] = value, index
        for a, b in zip(run(logits, idx, mask), want):
            assert torch.equal(a, b), (value, index)
    # bytes, and any value but 0
    for a, b in zip(run(logits, idx, mask.to(torch.uint8) * 200), want):
        assert torch.equal(a, b)
    # no token counts
    logits[:], idx[:] = float("nan"), 1 << 30
    assert not any(t.any() for t in run(logits, idx, torch.zeros(T, dtype=torch.bool)))
