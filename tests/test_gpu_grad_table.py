"""Tables whose outputs overlap are refused before anything is launched (marked `gpu`)."""
import pytest
import torch

from paper_2607_08782_amd import moe

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


def _refused(grads, out=None):
    before = [g.clone() for g in grads]
    table = moe.GradTable(grads, out=out)
    norm = moe.moe_grad_norm(table)
    exact = torch.cat([g.double().flatten() for g in grads]).norm()
    assert abs(float(norm) - float(exact)) <= 2.0 ** -23 * float(exact)    # a norm writes none of them
    with pytest.raises(ValueError, match="overlap"):
        moe.moe_clip_grads(table, norm, 0.5)
    for a, b in zip(grads, before):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_outputs_that_overlap_are_refused(dtype):
    a, b = (torch.randn(20000, generator=torch.Generator().manual_seed(n)).to(dtype).cuda() for n in (1, 2))
    room = torch.ones(40000, dtype=dtype, device="cuda")
    _refused([a, b], [b, a])                         # swapped
    _refused([a, b], [room[:20000], a])              # over another's gradient
    _refused([a, b], [room[:20000], room[16000:36000]])
    _refused([a, b[:8]], [room[:20000], room[64:72]])
    _refused([room[:20000].copy_(a), room[16000:36000]])
    _refused([room[:20000].copy_(a)], [room[8:20008]])
    _refused([a, a], [a, room[:20000]])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_outputs_side_by_side_are_clipped(dtype):
    """One behind the other, in place or not, and of one gradient twice."""
    a, b = (torch.randn(9001, generator=torch.Generator().manual_seed(n)).to(dtype).cuda() for n in (1, 2))
    room = torch.empty(3 * 9001, dtype=dtype, device="cuda")
    out = list(room.split(9001))
    table = moe.GradTable([a, b, a], out=out)
    norm = moe.moe_grad_norm(table)
    moe.moe_clip_grads(table, norm, 0.5)
    want = [(g.float() * (0.5 / norm)).to(dtype) for g in (a, b, a)]
    assert torch.equal(room, torch.cat(want))
    room[:18002].copy_(torch.cat([a, b]))
    table = moe.GradTable(out[:2])
    moe.moe_clip_grads(table, norm, 0.5)
    assert torch.equal(room, torch.cat(want))
