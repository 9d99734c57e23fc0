"""Calls of more workgroups than one grid holds (marked `gpu`): every row is there, and the
rows around the end of the first launch and the last ones are right."""
import pytest
import torch

from oracle import mxfp4 as om
from paper_2607_08782_amd import moe

from parity import say
from test_gpu_ffn_mxfp4 import _expected, _experts, _values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield
    torch.cuda.empty_cache()


def test_4_bit_ffn_of_a_long_batch():
    """2^24 token rows and some: the first ones, those around the end of a launch, the last."""
    say("[ffn mxfp4 long batch]")
    d, f, T = 8, 96, (1 << 24) + 100
    (w13,), (w2,) = _experts(1, d, f, 21)
    table = moe.MxWeightTable([w13], [w2], d, f)
    x = torch.randn(T, d, generator=torch.Generator(device="cuda").manual_seed(21), device="cuda").bfloat16()
    token = torch.cat([torch.arange(0, 40), torch.arange((1 << 24) - 60, T)]).int().cuda()
    n = len(token)
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    ws = torch.full((moe.moe_grouped_ffn_mxfp4_ws_bytes(T, n, d, f, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    got = moe.moe_grouped_ffn_mxfp4(x, off, table, row_token=token, cap_rows=n, ws=ws)
    want, tol = _expected(om.rounded(x[token.long()].float().cpu().numpy()), _values(w13, d), _values(w2, f), f)
    assert (abs(got[:n].double().cpu().numpy() - want) <= tol).all()


def test_conversions_of_many_rows():
    """Rows of one value that 4 bits hold exactly: to MXFP4, step-major (of one step: in the
    same order) and back."""
    say("[mxfp4 many rows]")
    rows, part = (1 << 30) + 37, 1 << 26
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 3.0, 6.0, -0.75, -48.0, 2.0 ** 100, -2.0 ** -90], device="cuda")
    order = torch.randint(0, len(values), (9973,), generator=torch.Generator().manual_seed(1)).cuda()
    x = torch.empty(rows, 1, dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, part):
        at = torch.arange(r, min(r + part, rows), device="cuda") % len(order)
        x[r:r + part, 0] = values[order[at]]
    q = torch.full((rows, 64), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, 4), 0xA5, dtype=torch.uint8, device="cuda")
    moe.moe_quantize_mxfp4(x, q=q, scales=scales)
    y = torch.full((rows, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_dequantize_mxfp4(q, scales, 1, out=y)
    steps, words = moe.moe_mxfp4_lay_out(q, scales, 1)
    for r in range(0, rows, part):
        e = min(r + part, rows)
        assert torch.equal(x[r:e], y[r:e]), r
        assert torch.equal(steps[0, r:e].view(torch.int64), q[r:e].view(torch.int64)), r
        assert torch.equal(words[0, r:e], scales[r:e].view(torch.int32)[:, 0]), r
        assert not q[r:e, 1:].view(torch.uint8).any() and not scales[r:e, 1:].any(), r


@pytest.mark.parametrize("T,d", [((1 << 20) + 900, 4097), ((1 << 23) + 900, 4096)])
def test_packaging_gradient_of_a_long_batch(T, d):
    """More elements than work-items of a grid, by either of the kernels: each token's row is
    one of few, its number tells which."""
    say("[permute grad long batch]", T, d)
    n = 97
    rows = torch.randn(n, d, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    row = (torch.arange(T, device="cuda") % n).int().view(T, 1)
    dx = torch.full((T, d), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_permute_backward(rows, row, dx=dx)
    part = n * 10000
    want = rows.repeat(10000, 1)
    for t in range(0, T, part):
        got = dx[t:t + part]
        assert torch.equal(got, want[:len(got)]), t


def test_combine_and_gate_gradients_of_a_long_batch():
    """2^26 tokens and some, of one column each: dy_perm and dgate of the last token of every
    2^20 and of those around the end of a launch; dlogits of all."""
    say("[combine grad long batch]")
    T, n = (1 << 26) + 77, 200
    tokens = torch.cat([torch.arange((1 << 20) - 1, T, 1 << 20), torch.arange((1 << 26) - 60, (1 << 26) - 1),
                        torch.arange(T - 60, T)]).cuda()
    m = len(tokens)
    assert m <= n and len(tokens.unique()) == m
    row = torch.full((T, 1), -1, dtype=torch.int32, device="cuda")
    row[tokens, 0] = torch.arange(m, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(6)
    # products of bf16 values are exact in 32 bits
    dy = torch.randn(T, 1, generator=g, device="cuda").bfloat16()
    y = torch.randn(n, 1, generator=g, device="cuda").bfloat16()
    gate = torch.rand(T, 1, generator=g, device="cuda")
    out = torch.full((n, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    dgate = torch.full((T, 1), 7.0, device="cuda")
    moe.moe_combine_backward(dy, y, row, gate, dy_perm=out, dgate=dgate)
    want = torch.zeros(T, 1, device="cuda")
    want[tokens, 0] = dy[tokens, 0].float() * y[:m, 0].float()
    assert torch.equal(dgate, want)
    assert torch.equal(out[:m], (gate[tokens] * dy[tokens].float()).bfloat16()) and bool((out[m:] == 7.0).all())
    # one expert, not renormalised: the softmax is 1 and its gradient 0; two, one half each
    zeros = torch.zeros(T, 2, device="cuda")
    idx = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    x, w = torch.empty(T, 1, device="cuda"), torch.empty(2, 1, device="cuda")
    dl = torch.full((T, 2), 7.0, device="cuda")
    moe.moe_route_topk_backward(gate, torch.full_like(gate, 0.5), idx, x, w, logits=zeros, renorm=False,
                                want_dx=False, want_dw=False, want_dbias=False, dlogits=dl)
    assert torch.equal(dl[:, :1], 0.25 * gate) and torch.equal(dl[:, 1:], -0.25 * gate)


def test_router_gradient_of_the_longest_rows():
    """fp32 dx over more column tiles than a grid has along its second dimension."""
    say("[route grad long rows]")
    T, E, d = 3, 2, (1 << 22) - 5
    g = torch.Generator(device="cuda").manual_seed(7)
    w = torch.randn(E, d, generator=g, device="cuda")
    x = torch.empty(T, d, device="cuda")
    dgate, gate = torch.randn(T, 1, generator=g, device="cuda"), torch.full((T, 1), 0.5, device="cuda")
    idx = torch.tensor([[0], [1], [0]], dtype=torch.int32, device="cuda")
    dl, dx, _, _ = moe.moe_route_topk_backward(dgate, gate, idx, x, w, logits=torch.zeros(T, E, device="cuda"),
                                               renorm=False, want_dw=False, want_dbias=False,
                                               dx=torch.full_like(x, 7.0))
    want = (dl.double()[:, :, None] * w.double()).sum(1)
    size = (dl.double()[:, :, None] * w.double()).abs().sum(1)
    assert bool(((dx.double() - want).abs() <= (E + 4) * 2.0 ** -24 * size).all())
