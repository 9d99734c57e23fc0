"""moe_route_topk_backward_aux (marked `gpu`): the router's gradient with a gradient that reaches the
scores another way.  dlogits is the sum of two fp32 values, rounded once, so it is checked bit for
bit; dx, dw and dbias against float64 products of it, with the bounds that the call without it
keeps: E + 4 (T + 4) times 2^-24 of the sum of magnitudes, and dx's own rounding."""
import numpy as np
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


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,E,k,d", [(1, 8, 2, 64), (64, 8, 2, 4096), (333, 24, 3, 1000), (777, 64, 6, 256),
                                     (515, 129, 5, 64), (2050, 128, 8, 256)])
def test_added_gradient(T, E, k, d, dtype, renorm):
    say("[route grad aux]", T, E, k, d, dtype, renorm)
    g = torch.Generator().manual_seed(T + E)
    rnd = lambda *s: torch.randn(*s, generator=g)
    logits, add = rnd(T, E).cuda(), rnd(T, E).cuda()
    _, idx, gate = moe.moe_route_topk(None, None, None, k, logits=logits, logits_in=True, renorm=renorm)
    args = rnd(T, k).cuda(), gate, idx, rnd(T, d).to(dtype).cuda(), (0.02 * rnd(E, d)).to(dtype).cuda()
    kw = dict(logits=None if renorm else logits, renorm=renorm)
    alone = moe.moe_route_topk_backward(*args, **kw)
    got = moe.moe_route_topk_backward(*args, **kw, dlogits_add=add)
    assert torch.equal(got[0], alone[0] + add)
    dl, x, w = (t.double().cpu().numpy() for t in (got[0], args[3], args[4]))
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    # (bf16: dlogits enter dx with 16 bits)
    entry = 2.0 ** -16 if dtype == torch.bfloat16 else 0.0
    for name, out, want, tol in (
            ("dx", got[1], dl @ w, (entry + (E + 4) * 2.0 ** -24) * (np.abs(dl) @ np.abs(w)) + half * np.abs(dl @ w)),
            ("dw", got[2], dl.T @ x, (T + 4) * 2.0 ** -24 * (np.abs(dl).T @ np.abs(x))),
            ("dbias", got[3], dl.sum(0), (T + 4) * 2.0 ** -24 * np.abs(dl).sum(0))):
        off = np.abs(out.double().cpu().numpy() - want)
        assert (off <= tol + 1e-44).all(), (name, (off / tol).max())
    # in place, and every output alone
    over = add.clone()
    assert torch.equal(moe.moe_route_topk_backward(*args, **kw, dlogits_add=over, dlogits=over)[0], got[0])
    for i, name in enumerate(("dlogits", "dx", "dw", "dbias")):
        want = {"want_" + n: n == name for n in ("dlogits", "dx", "dw", "dbias")}
        assert torch.equal(moe.moe_route_topk_backward(*args, **kw, dlogits_add=add, **want)[i], got[i]), name


def test_refusals():
    z = lambda *s: torch.zeros(*s, device="cuda")
    args = z(4, 2), z(4, 2), z(4, 2).int(), z(4, 16), z(8, 16)
    for bad in (z(4, 7), z(3, 8), z(4, 8).double()):
        with pytest.raises(ValueError, match="dlogits_add must be"):
            moe.moe_route_topk_backward(*args, dlogits_add=bad)
