"""What a share's gradient goes back through (marked `gpu`): the last run."""
import pytest
import torch

from paper_2607_08782_amd import moe, synth
from paper_2607_08782_amd.layer import LayerShare

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


def test_gradients_without_a_run_are_refused():
    """The row maps hold no rows yet: nothing is read by them."""
    _, share = _share()
    with pytest.raises(ValueError, match="run"):
        share.backward(_normal(5, T, share.d))
    with pytest.raises(ValueError, match="run"):
        share.backward_rows(_normal(6, *share.y_perm.shape))
