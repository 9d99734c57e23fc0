"""What a share's gradient goes back through (marked `gpu`): the scores and token rows of the
last routing, whatever the share was given since.

Tolerances: an fp32 sum of n products is within (n + 4) 2^-24 of the sum of its terms'
magnitudes, a softmax gradient within (E + 16) 2^-24 + 2^-19 of its own."""
import numpy as np
import pytest
import torch

from paper_2607_08782_amd import moe, synth
from paper_2607_08782_amd.layer import LayerShare

from parity import say
from test_gpu_grad import _np, _want_route

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


T = 150
CFG = dict(dtype="f32", d=64, E=12, k=3, f=32, zipf=1.0)


def _share(**kw):
    cfg = synth.custom_config(**CFG)
    i = synth.make_layer(cfg, T, device="cuda")
    return i, LayerShare(i.X, i.Wr, i.bias, cfg.k, i.placement, 0, i.w13, i.w2, fuse_combine=False, **kw)


def _normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()


def _check_router(share, g, X, logits, renorm):
    """dx, dw and dbias of a share's backward against the formulas on X and these scores."""
    dl, size, dx, dx_size, dw, dw_size = _want_route(logits, share.topk_idx, share.topk_gate, g["dgate"], X,
                                                     share.Wr, renorm)
    E = share.E
    rel = (E + 16) * 2.0 ** -24 + 2.0 ** -19
    for name, want, tol in (("dx", dx, (rel + (E + 4) * 2.0 ** -24) * dx_size),
                            ("dw", dw, (rel + (T + 4) * 2.0 ** -24) * dw_size),
                            ("dbias", dl.sum(0), (rel + (T + 4) * 2.0 ** -24) * size.sum(0))):
        off = np.abs(_np(g[name]) - want)
        assert (off <= tol + 2.0 ** -24 * np.abs(want)).all(), (name, off.max(), np.abs(want).max())


def test_gradients_without_a_run_are_refused():
    """The row maps hold no rows yet: nothing is read by them."""
    _, share = _share()
    with pytest.raises(ValueError, match="run"):
        share.backward(_normal(5, T, share.d))
    with pytest.raises(ValueError, match="run"):
        share.backward_rows(_normal(6, *share.y_perm.shape))


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("phases", [False, True])
def test_backward_takes_the_scores_that_were_handed_in(renorm, phases):
    """run(logits_in=...) and route(logits_in=...) choose by the caller's scores; the share's
    own hold an earlier batch's."""
    say("[backward of given scores]", renorm, phases)
    _, share = _share(renorm=renorm)
    share.run()
    given = _normal(1, T, share.E)
    if phases:
        share.route(logits_in=given)
        share.package()
        share.routed_ffn()
        share.combine()
    else:
        share.run(logits_in=given)
    g = share.backward(_normal(2, T, share.d))
    _check_router(share, g, share.X, given, renorm)
    share.run()                                      # and its own again
    g = share.backward(_normal(3, T, share.d))
    _check_router(share, g, share.X, share.logits, renorm)


def test_given_scores_need_none_of_the_share_s_own():
    _, share = _share(renorm=False, want_logits=False)
    dy = _normal(2, T, share.d)
    given = _normal(1, T, share.E)
    share.run(logits_in=given)
    _check_router(share, share.backward(dy), share.X, given, False)
    share.run()
    with pytest.raises(ValueError, match="want_logits"):
        share.backward(dy)


def test_backward_after_the_next_batch_s_inputs_are_set():
    """set_inputs for the next batch between run and backward: the gradient is the run's."""
    i, share = _share()
    share.run()
    share.set_inputs(_normal(4, T, share.d))
    _check_router(share, share.backward(_normal(5, T, share.d)), i.X, share.logits, True)


def test_backward_rows_adds_no_earlier_batch_s_gradient():
    """run, backward, run, backward_rows: dx is the rows' alone; after a backward of the same
    run it is on top of that one's."""
    _, share = _share()
    dx_perm = _normal(6, *share.y_perm.shape)
    rows = lambda: moe.moe_permute_backward(dx_perm, share.perm["token_row"])
    share.run()
    dx = share.backward(_normal(7, T, share.d))["dx"]
    both = moe.moe_permute_backward(dx_perm, share.perm["token_row"], dx_add=dx)
    assert torch.equal(share.backward_rows(dx_perm), both) and not torch.equal(both, rows())
    share.set_inputs(_normal(8, T, share.d))
    assert torch.equal(share.backward_rows(dx_perm), both)           # still the last run's
    share.run()
    assert torch.equal(share.backward_rows(dx_perm), rows())
    share.backward(_normal(9, T, share.d))
    assert not torch.equal(share.backward_rows(dx_perm), rows())
    share.route()
    assert torch.equal(share.backward_rows(dx_perm), rows())
