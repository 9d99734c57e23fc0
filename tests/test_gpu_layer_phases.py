"""A share stepped phase by phase, and by the step that migrates experts (marked `gpu`): the rows
that a norm or 8-bit experts need are the present batch's there too."""
import numpy as np
import pytest
import torch

from paper_2607_08782_amd import moe, synth
from paper_2607_08782_amd.layer import LayerShare
from paper_2607_08782_amd.migration import ExpertStore, Migrator, run_step

from parity import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


CFG = dict(d=256, E=16, k=4, f=192, G=3, replicas=2, zipf=1.2)
FRONTS = {"plain": (), "int8": ("int8",), "norm": ("norm",), "norm mxfp4": ("norm", "mxfp4"),
          "norm int8": ("norm", "int8"), "residual": ("norm", "residual"),
          "residual int8": ("norm", "residual", "int8")}
MADE = [f for f in FRONTS if f != "plain"]


def _rows(T, d, seed):
    return torch.randn(T, d, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def _options(front, T, d):
    kw = {name: True for name in FRONTS[front] if name in ("int8", "mxfp4")}
    if "norm" in FRONTS[front]:
        kw["norm"] = (1 + 0.2 * _rows(1, d, 3)[0]).contiguous()
    if "residual" in FRONTS[front]:
        kw["residual"] = _rows(T, d, 4)
    return kw


def _share(front, T, shared_f=(), cfg=CFG):
    """A share, and one of the same layer with a batch of its own."""
    cfg = synth.custom_config(**cfg, shared_f=shared_f)
    i = synth.make_layer(cfg, T, device="cuda")

    def make(X=i.X, **kw):
        return LayerShare(X, i.Wr, i.bias, cfg.k, i.placement, 0, i.w13, i.w2, shared=i.shared, fuse_combine=False,
                          **dict(_options(front, T, cfg.d), **kw))
    return make(), make


def _next(share, front, n):
    """The share's next batch, as its arguments."""
    kw = {"residual": _rows(share.T, share.d, 200 + n)} if "residual" in FRONTS[front] else {}
    return dict(X=_rows(share.T, share.d, 100 + n), **kw)


def _phases(share):
    share.route()
    moe.moe_expert_histogram(share.topk_idx, share.E, counts=share.counts)
    share.package()
    share.routed_ffn()
    share._shared_ffn()
    share.combine()


def _packaged_phases(share):
    share._route_package()
    share.routed_ffn()
    share._shared_ffn()
    share.combine()


def _same(share, make, batch):
    """What the share holds is what a share of this batch's own gives by `run`."""
    fresh = make(**batch)
    y = fresh.run()
    torch.cuda.synchronize()
    assert torch.equal(share.topk_idx, fresh.topk_idx) and torch.equal(share.rows, fresh.rows)
    assert torch.equal(share.y, y)
    return fresh


@pytest.mark.parametrize("T,shared_f", [(1, ()), (40, (64,)), (300, ())])
@pytest.mark.parametrize("front", list(FRONTS))
@pytest.mark.parametrize("step", [lambda s: run_step(s, None), _phases, _packaged_phases])
def test_steps_after_the_next_batch_s_inputs_are_set(T, shared_f, front, step):
    say("[phases]", T, shared_f, front)
    share, make = _share(front, T, shared_f)
    share.run()
    for n in range(2):
        batch = _next(share, front, n)
        share.set_inputs(**batch)
        step(share)
        fresh = _same(share, make, batch)
        dy = _rows(T, share.d, 300 + n)
        got, want = share.backward(dy), fresh.backward(dy)
        for name in want:
            # (rows past the groups' end are not written)
            end = int(share.perm["group_offsets"][-1]) if name == "dy_perm" else None
            assert torch.equal(got[name][:end], want[name][:end]), name


@pytest.mark.parametrize("front", list(FRONTS))
@pytest.mark.parametrize("step", [lambda s: run_step(s, None), _phases])
def test_steps_after_a_batch_is_written_over_the_last(front, step):
    """No set_inputs: X and the residual get new values where they are."""
    share, make = _share(front, 33)
    share.run()
    batch = _next(share, front, 5)
    share.X.copy_(batch["X"])
    if "residual" in batch:
        share.residual.copy_(batch["residual"])
    step(share)
    _same(share, make, batch)


@pytest.mark.parametrize("front", list(FRONTS))
@pytest.mark.parametrize("step", [lambda s: run_step(s, None), _phases, _packaged_phases])
def test_the_first_step_of_a_share(front, step):
    share, make = _share(front, 17)
    step(share)
    _same(share, make, {})


@pytest.mark.parametrize("front", MADE)
def test_rows_of_an_earlier_batch_are_refused(front):
    share, make = _share(front, 24, (64,))
    for phase in (share.package, share.routed_ffn, share._shared_ffn):
        with pytest.raises(ValueError, match="prepare_rows"):
            phase()                                  # of no batch yet
    share.run()
    share.routed_ffn()                               # again, over the same rows
    share.set_inputs(**_next(share, front, 1))
    for phase in (share.package, share.routed_ffn, share._shared_ffn):
        with pytest.raises(ValueError, match="prepare_rows"):
            phase()
    share.prepare_rows()
    share._shared_ffn()                              # before the routing
    _phases(share)
    _same(share, make, _next(share, front, 1))


@pytest.mark.parametrize("front", [f for f in MADE if "norm" in FRONTS[f]])
def test_gradients_through_rows_that_were_made_anew_are_refused(front):
    """The rows that the last routing read are gone: what they were multiplied with is not theirs."""
    share, _ = _share(front, 24)
    dy = _rows(24, share.d, 9)
    share.run()
    want = {n: t.clone() for n, t in share.backward(dy).items()}
    share.set_inputs(**_next(share, front, 2))
    for name, t in share.backward(dy).items():       # still the run's
        assert torch.equal(t, want[name]), name
    share.prepare_rows()
    with pytest.raises(ValueError, match="made anew"):
        share.backward(dy)
    share.run()
    share.backward(dy)


@pytest.mark.parametrize("front", ["int8", "residual int8"])
def test_8_bit_experts_that_migrate(front):
    """Batch after batch while two experts move in: each what a share of the old placement gives;
    after the switch, of the new one."""
    cfg = synth.custom_config(d=256, E=16, k=4, f=256, G=4, zipf=1.2)
    T = 48
    i = synth.make_layer(cfg, T, seed=2, device="cuda", experts="all")
    old = np.ascontiguousarray(i.placement, dtype=np.uint8)
    only = lambda j: [e for e in range(cfg.E) if old[e].sum() == 1 and old[e, j]]
    new = old.copy()
    for a, b in zip(only(0)[:2], only(1)[:2]):
        new[a, 0], new[a, 1], new[b, 0], new[b, 1] = 0, 1, 1, 0
    mig = Migrator(ExpertStore(i.w13, i.w2), old, 0, spare=2, chunk_bytes=64 << 10)

    def make(placement, w13, w2, X=i.X, **kw):
        return LayerShare(X, i.Wr, i.bias, cfg.k, placement, 0, w13, w2, **dict(_options(front, T, cfg.d), **kw))
    share = make(old, *mig.weights())
    held = lambda P: [[w[e] for e in np.nonzero(P[:, 0])[0]] for w in (i.w13, i.w2)]
    mig.plan(new)
    n = 0
    while not mig.finished:
        batch = _next(share, front, n)
        share.set_inputs(**batch)
        run_step(share, mig, budget_bytes=256 << 10)
        _same(share, lambda **kw: make(old, *held(old), **kw), batch)
        n += 1
    assert n > 1
    share.set_placement(new, *mig.switch())
    batch = _next(share, front, n)
    share.set_inputs(**batch)
    run_step(share, None)
    _same(share, lambda **kw: make(new, *held(new), **kw), batch)


@pytest.mark.parametrize("front", list(FRONTS))
def test_phases_replay_from_a_graph(front):
    """The rows are made within the graph: each replay's are those of what X and the residual hold."""
    share, make = _share(front, 40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        share.prepare_rows()
        _phases(share)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _phases(share)
    for n in range(4):
        batch = _next(share, front, 10 + n)
        share.X.copy_(batch["X"])
        if "residual" in batch:
            share.residual.copy_(batch["residual"])
        g.replay()
        _same(share, make, batch)
        share.run()                                  # eager work between the replays
        _same(share, make, batch)
