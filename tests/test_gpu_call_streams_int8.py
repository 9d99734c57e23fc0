"""Calls on a given stream that allocate for themselves, of 8-bit rows and experts, the norm, the
balance loss, the router's gradient with another added and the gradients' norm (marked `gpu`):
outputs and workspaces lie in that stream's memory."""
import numpy as np
import pytest
import torch

from paper_2607_08782_amd import moe

from parity import say
from test_gpu_call_streams import SLEEP, _owner, _tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


T, E, k, d, f, G = 300, 12, 3, 256, 128, 2
LONG = 3000                                          # tokens whose balance loss takes three launches


def _calls():
    """(name, call(stream)) on inputs made here."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, w = rand(T, d).bfloat16(), (rand(E, d) * 0.05).bfloat16()
    logits, idx, gate = moe.moe_route_topk(x, w, None, k)
    counts = moe.moe_expert_histogram(idx, E)[0]
    placement = np.zeros((E, G), np.uint8)
    placement[np.arange(E), np.arange(E) % G] = 1
    cap = T * k
    maps = moe.moe_permute(x, idx, gate, counts, placement, 0, E=E, cap_rows=cap)
    n = E // G
    table = moe.Int8WeightTable.quantized([(rand(2 * f, d) * 0.05).bfloat16() for _ in range(n)],
                                          [(rand(d, f) * 0.05).bfloat16() for _ in range(n)])
    wide = moe.Int8WeightTable.quantized([(rand(256, 2304) * 0.05).bfloat16()], [(rand(2304, 128) * 0.05).bfloat16()])
    off, tok = maps["group_offsets"], maps["row_token"]
    N = int(off[-1])
    q, s = moe.moe_quantize_int8(x)
    q60, s60 = moe.moe_quantize_int8(rand(60, 2304).bfloat16())
    off60 = torch.tensor([0, 60], dtype=torch.int32, device="cuda")
    weight, residual, dy = rand(d).bfloat16(), rand(T, d).bfloat16(), rand(T, d).bfloat16()
    h, _, rstd, _, _ = moe.moe_rmsnorm(x, weight, want_rstd=True)
    _, bcounts, _, bn = moe.moe_balance_loss(logits, idx)
    long_logits = rand(LONG, E)
    long_idx = torch.topk(long_logits, k, 1)[1].int()
    mask = rand(LONG) > 0
    dgate, add = rand(T, k), rand(T, E)
    grads = moe.GradTable([rand(90000), rand(77).bfloat16(), rand(3, 5)])
    return [
        ("quantize_int8", lambda st: moe.moe_quantize_int8(x, stream=st)),
        ("dequantize_int8", lambda st: moe.moe_dequantize_int8(q, s, d, stream=st)),
        ("dequantize_int8 fp32", lambda st: moe.moe_dequantize_int8(q, s, d, dtype=torch.float32, stream=st)),
        ("ffn_int8", lambda st: moe.moe_grouped_ffn_int8(q, s, off, table, row_token=tok, cap_rows=cap, stream=st)[:N]),
        ("ffn_int8 long K", lambda st: moe.moe_grouped_ffn_int8(q60, s60, off60, wide, stream=st)),
        ("rmsnorm", lambda st: moe.moe_rmsnorm(x, weight, want_rstd=True, want_q=True, stream=st)[1:]),
        ("rmsnorm residual", lambda st: moe.moe_rmsnorm(x, weight, residual=residual, want_rstd=True, want_q=True,
                                                        stream=st)),
        ("rmsnorm_backward", lambda st: moe.moe_rmsnorm_backward(dy, h, weight, rstd, dh_add=residual, stream=st)),
        ("balance_loss", lambda st: moe.moe_balance_loss(logits, idx, stream=st)),
        ("balance_loss long", lambda st: moe.moe_balance_loss(long_logits, long_idx, mask=mask, stream=st)),
        ("balance_loss_backward", lambda st: moe.moe_balance_loss_backward(logits, bcounts, bn, k, stream=st)),
        ("route_backward add", lambda st: moe.moe_route_topk_backward(dgate, gate, idx, x, w, dlogits_add=add, stream=st)),
        ("grad_norm", lambda st: moe.moe_grad_norm(grads, stream=st)),
    ]


@pytest.mark.parametrize("handle", [False, True])
def test_what_a_call_allocates_belongs_to_its_stream(handle):
    say("[call streams int8]", handle)
    calls = _calls()
    side = torch.cuda.Stream()
    want = [_tensors(call(None)) for _, call in calls]
    torch.cuda.synchronize()
    for (name, call), ref in zip(calls, want):
        with torch.cuda.stream(side):
            torch.cuda._sleep(SLEEP)
        got = _tensors(call(side.cuda_stream if handle else side))
        # what the call dropped, if the current stream could have it, is overwritten now
        junk = [torch.full((1 << n,), 0xA5, dtype=torch.uint8, device="cuda") for n in range(9, 24) for _ in (0, 1)]
        assert len(got) == len(ref) and all(_owner(t) == side.cuda_stream for t in got), name
        torch.cuda.synchronize()
        for a, b in zip(got, ref):
            assert torch.equal(a, b), name
        del junk
