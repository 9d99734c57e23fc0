"""Calls on a given stream that allocate for themselves (marked `gpu`): outputs and workspaces
lie in that stream's memory, so that work queued on the current stream, before the call or
after it, shares none of it."""
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


T, E, k, d, f, G = 300, 12, 3, 256, 128, 2
SLEEP = 20_000_000                                   # clocks: about 10 ms


def _calls():
    """(name, call(stream)): every entry point that allocates, on inputs made here."""
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
    w13, w2 = [(rand(2 * f, d) * 0.05).bfloat16() for _ in range(n)], [(rand(d, f) * 0.05).bfloat16() for _ in range(n)]
    table, mx = moe.WeightTable(w13, w2), moe.MxWeightTable.quantized(w13, w2)
    off, tok, row = maps["group_offsets"], maps["row_token"], maps["token_row"]
    N = int(off[-1])
    y = moe.moe_grouped_ffn(maps["x_perm"], off, table, cap_rows=cap)
    q, s = moe.moe_quantize_mxfp4(x)
    dgate = rand(T, k)
    first = lambda t: t[:N]                          # rows past the groups' end are not written
    return [
        ("route_topk", lambda st: moe.moe_route_topk(x, w, None, k, stream=st)),
        ("histogram", lambda st: moe.moe_expert_histogram(idx, E, want_coact=True, stream=st)),
        ("permute", lambda st: moe.moe_permute(x, idx, gate, counts, placement, 0, E=E, cap_rows=cap,
                                               stream=st)["token_row"]),
        ("ffn", lambda st: first(moe.moe_grouped_ffn(maps["x_perm"], off, table, cap_rows=cap, stream=st))),
        ("ffn_rows", lambda st: first(moe.moe_grouped_ffn_rows(x, tok, off, table, cap_rows=cap, stream=st))),
        ("combine", lambda st: moe.moe_combine(y, row, gate, None, T=T, d=d, stream=st)),
        ("quantize_e4m3", lambda st: moe.moe_quantize_e4m3(x, stream=st)),
        ("quantize_mxfp4", lambda st: moe.moe_quantize_mxfp4(x, stream=st)),
        ("dequantize_mxfp4", lambda st: moe.moe_dequantize_mxfp4(q, s, d, stream=st)),
        ("lay_out", lambda st: moe.moe_mxfp4_lay_out(q, s, d, stream=st)),
        ("ffn_mxfp4", lambda st: first(moe.moe_grouped_ffn_mxfp4(x, off, mx, row_token=tok, cap_rows=cap, stream=st))),
        ("combine_backward", lambda st: moe.moe_combine_backward(x, y, row, gate, want_dy_perm=False, stream=st)[1]),
        ("combine_backward rows", lambda st: first(moe.moe_combine_backward(x, y, row, gate, stream=st)[0])),
        ("permute_backward", lambda st: moe.moe_permute_backward(y, row, stream=st)),
        ("permute_backward add", lambda st: moe.moe_permute_backward(y, row, dx_add=x, stream=st)),
        ("route_backward", lambda st: moe.moe_route_topk_backward(dgate, gate, idx, x, w, stream=st)),
    ]


def _tensors(out):
    return [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]


def _owner(t):
    """Handle of the stream that a tensor's memory belongs to."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("no such memory")


@pytest.mark.parametrize("handle", [False, True])
def test_what_a_call_allocates_belongs_to_its_stream(handle):
    say("[call streams]", handle)
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
        assert all(_owner(t) == side.cuda_stream for t in got), name
        torch.cuda.synchronize()
        for a, b in zip(got, ref):
            assert torch.equal(a, b), name
        del junk
