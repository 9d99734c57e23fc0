"""Swaps of the placement of a share with 4-bit experts (marked `gpu`) beside runs on other
streams and captured ones."""
import numpy as np
import pytest
import torch

from paper_2607_08782_amd import moe, synth
from paper_2607_08782_amd.layer import LayerShare

from parity import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


CFG = dict(d=256, E=16, k=4, f=192, G=3, replicas=2, zipf=1.2)
SLEEP = 20_000_000                                   # clocks: about 10 ms


def _layers(T):
    """Two layers' experts on the same inputs, and the output with either's."""
    cfg = synth.custom_config(**CFG)
    i, other = (synth.make_layer(cfg, T, seed=s, device="cuda") for s in (0, 9))
    make = lambda e: LayerShare(i.X, i.Wr, i.bias, cfg.k, i.placement, 0, e.w13, e.w2, mxfp4=True)
    want = [make(e).run().clone() for e in (i, other)]
    torch.cuda.synchronize()
    assert not torch.equal(*want)
    return i, other, make(i), want


def _overwrite_free_memory(table):
    """Tensors of the sizes of a table's, twice over, filled."""
    tensors = table.w13 + table.s13 + table.w2 + table.s2
    return [torch.full_like(t, 77) for t in tensors + tensors]


@pytest.mark.parametrize("T", [40, 300])
def test_runs_on_another_stream_around_a_swap(T):
    """A run still waiting on its stream when the swap is made on another keeps the old experts;
    the next one there has the new ones, though nothing made it wait for the swap's stream."""
    say("[mxfp4 swap streams]", T)
    i, other, share, (old, new) = _layers(T)
    runs, swaps = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(runs):
        torch.cuda._sleep(SLEEP)
        first = share.run().clone()
    with torch.cuda.stream(swaps):
        torch.cuda._sleep(SLEEP)
        share.set_placement(i.placement, other.w13, other.w2)
        keep = _overwrite_free_memory(share.weights)
    with torch.cuda.stream(runs):
        second = share.run().clone()
    torch.cuda.synchronize()
    assert torch.equal(first, old) and torch.equal(second, new)
    del keep


@pytest.mark.parametrize("T", [16, 300])
def test_a_captured_run_replays_with_its_experts_after_swaps(T):
    """As with experts in bf16, which belong to the caller: a graph from before a swap computes
    what it did, whatever the memory that is free by then holds."""
    say("[mxfp4 swap graph]", T)
    i, other, share, (old, new) = _layers(T)
    share.run()
    torch.cuda.synchronize()
    graphs = []
    for e, want in ((i, old), (other, new)):
        share.set_placement(i.placement, e.w13, e.w2)
        graphs.append((torch.cuda.CUDAGraph(), want))
        with torch.cuda.graph(graphs[-1][0]):
            share.run()
            share.run()
    assert len(share.captured_tables) == 2 and share.captured_tables[1] is share.weights
    share.set_placement(i.placement, i.w13, i.w2)
    keep = _overwrite_free_memory(share.weights)
    for _ in range(3):
        for g, want in graphs:
            g.replay()
            assert torch.equal(share.y, want)
        assert torch.equal(share.run(), old)
        torch.cuda.synchronize()
    del keep
    assert len(share.captured_tables) == 2               # eager runs add none


@pytest.mark.parametrize("mxfp4", [False, True])
def test_a_share_without_experts_takes_a_swap(mxfp4):
    cfg = synth.custom_config(**CFG)
    i = synth.make_layer(cfg, 20, device="cuda")
    nothing = np.concatenate([i.placement, np.zeros_like(i.placement[:, :1])], 1)    # on one GPU more
    share = LayerShare(i.X, i.Wr, i.bias, cfg.k, nothing, cfg.G, [], [], mxfp4=mxfp4)
    share.set_placement(nothing, [], [])
    assert not share.run().any()
