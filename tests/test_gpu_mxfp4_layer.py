"""A share with 4-bit experts, and the gradient of a share around its experts (marked `gpu`)."""
import dataclasses

import numpy as np
import pytest
import torch

from paper_2607_08782_amd import moe, synth
from paper_2607_08782_amd.gate_tuning import main
from paper_2607_08782_amd.layer import LayerShare

from parity import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    moe.load_library()
    yield


def _share(cfg, T, seed=0, **kw):
    i = synth.make_layer(cfg, T, seed=seed, device="cuda")
    return i, LayerShare(i.X, i.Wr, i.bias, cfg.k, i.placement, 0, i.w13, i.w2, shared=i.shared,
                         coact=cfg.coact, **kw)


CFG = dict(d=256, E=16, k=4, f=192, G=3, replicas=2, zipf=1.2)


@pytest.mark.parametrize("T,shared_f", [(1, ()), (40, ()), (40, (64,)), (700, (64, 128))])
def test_share_with_4_bit_experts_is_its_calls(T, shared_f):
    """The share's y from 4-bit experts against its parts: routing as the bf16 share's bit for
    bit, y the combine of moe_grouped_ffn_mxfp4's rows and the bf16 shared experts."""
    say("[mxfp4 share]", T, shared_f)
    cfg = synth.custom_config(**CFG, shared_f=shared_f)
    i, plain = _share(cfg, T, shared_in_ffn=False)
    _, share = _share(cfg, T, mxfp4=True)
    plain.run()
    y = share.run()
    torch.cuda.synchronize()
    for a, b in ((share.topk_idx, plain.topk_idx), (share.topk_gate, plain.topk_gate),
                 (share.counts, plain.counts), (share.perm["token_row"], plain.perm["token_row"])):
        assert torch.equal(a, b)
    N = int(share.perm["group_offsets"][-1])
    rows = moe.moe_grouped_ffn_mxfp4(i.X, share.perm["group_offsets"],
                                     moe.MxWeightTable.quantized(i.w13, i.w2),
                                     row_token=share.perm["row_token"], cap_rows=max(N, 1))
    assert torch.equal(rows[:N], share.y_perm[:N])
    want = moe.moe_combine(share.y_perm, share.perm["token_row"], share.topk_gate, share.y_shared, T=T, d=cfg.d)
    assert torch.equal(y[:T], want)
    if shared_f:
        assert torch.equal(share.y_shared[:T], plain.y_shared[:T])


@pytest.mark.parametrize("T", [16, 300])
def test_share_replays_from_a_graph(T):
    say("[mxfp4 graph]", T)
    cfg = synth.custom_config(**CFG)
    _, share = _share(cfg, T, mxfp4=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        share.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    dy = torch.randn(T, cfg.d, device="cuda").bfloat16()
    share.backward(dy)                               # allocates its buffers
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        share.run()
        grads = share.backward(dy)
    for n in range(4):
        share.X.copy_(torch.randn(T, cfg.d, device="cuda"))
        dy.copy_(torch.randn(T, cfg.d, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        got = [share.y.clone()] + [grads[k].clone() for k in sorted(grads)]
        share.run()
        again = share.backward(dy)
        torch.cuda.synchronize()
        for a, b in zip(got, [share.y] + [again[k] for k in sorted(again)]):
            assert torch.equal(a, b), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("renorm", [True, False])
def test_backward_of_a_whole_layer(dtype, renorm):
    """One GPU with every expert: the share's gradients, with the experts' own gradient from
    elementary products, against autograd of the layer's definition in float64 (the choice of
    experts as the share made it).  fp32: 1e-5 of the largest value.  bf16: four roundings
    (h, y_perm, dy_perm, the output) of 2^-8 each on the way, whose errors are independent
    over sums of hundreds of terms: 2^-6 of the largest value."""
    say("[layer grad]", dtype, renorm)
    T = 200
    cfg = synth.custom_config(dtype=dtype, d=128, E=12, k=3, f=64, zipf=1.0)
    i, share = _share(cfg, T, renorm=renorm, fuse_combine=False)
    share.run()
    dt = cfg.torch_dtype
    dy = torch.randn(T, cfg.d, generator=torch.Generator().manual_seed(5)).to(dt).cuda()
    g = share.backward(dy)
    off = share.perm["group_offsets"].tolist()
    tok = share.perm["row_token"].long()
    dx_perm = torch.zeros_like(share.y_perm)
    for s in range(cfg.E):                           # the experts' gradient, by plain products
        if off[s] == off[s + 1]:
            continue
        x = i.X[tok[off[s]:off[s + 1]]].float().requires_grad_()
        a, b = x @ i.w13[s][:cfg.f].float().t(), x @ i.w13[s][cfg.f:].float().t()
        ((torch.nn.functional.silu(a) * b) @ i.w2[s].float().t()).backward(g["dy_perm"][off[s]:off[s + 1]].float())
        dx_perm[off[s]:off[s + 1]] = x.grad.to(dt)
    dx = share.backward_rows(dx_perm)
    torch.cuda.synchronize()

    X = i.X.double().cpu().requires_grad_()
    W = i.Wr.double().cpu().requires_grad_()
    b = i.bias.double().cpu().requires_grad_()
    logits = X @ W.t() + b
    idx = share.topk_idx.long().cpu()
    gate = torch.softmax(logits.gather(1, idx), 1) if renorm else torch.softmax(logits, 1).gather(1, idx)
    y = torch.zeros(T, cfg.d, dtype=torch.float64)
    for e in range(cfg.E):
        h = torch.nn.functional.silu(X @ i.w13[e][:cfg.f].double().cpu().t()) * (X @ i.w13[e][cfg.f:].double().cpu().t())
        y = y + (h @ i.w2[e].double().cpu().t()) * (gate * (idx == e)).sum(1, keepdim=True)
    y.backward(dy.double().cpu())
    for name, got, want in (("dx", dx, X.grad), ("dw", g["dw"], W.grad), ("dbias", g["dbias"], b.grad)):
        err = float((got.double().cpu() - want).abs().max() / want.abs().max())
        say("  ", name, "%.2e" % err)
        assert err <= (1e-5 if dtype == "f32" else 2.0 ** -6), (name, err)


def test_reduction_of_the_gates_gradient_over_gpus():
    """Two GPUs' shares of one layer (run one after the other here): dgate summed over them is
    the whole layer's, and so is the router's gradient then."""
    T = 128
    cfg = synth.custom_config(dtype="f32", d=64, E=8, k=2, f=64, G=2)
    whole_cfg = dataclasses.replace(cfg, G=1)
    i = synth.make_layer(cfg, T, device="cuda", experts="all")
    dy = torch.randn(T, cfg.d, device="cuda")
    one = synth.make_layer(whole_cfg, T, device="cuda")
    whole = LayerShare(one.X, one.Wr, one.bias, cfg.k, one.placement, 0, one.w13, one.w2, fuse_combine=False)
    whole.run()
    want = whole.backward(dy)
    shares = []
    for dev in (0, 1):
        here = np.nonzero(i.placement[:, dev])[0]
        s = LayerShare(i.X, i.Wr, i.bias, cfg.k, i.placement, dev, [i.w13[e] for e in here],
                       [i.w2[e] for e in here], fuse_combine=False)
        s.run()
        shares.append(s)
    alone = [s.backward(dy)["dgate"].clone() for s in shares]
    assert ((alone[0] != 0) & (alone[1] != 0)).sum() == 0
    for n, s in enumerate(shares):
        g = s.backward(dy, reduce_dgate=lambda t: t.add_(alone[1 - n]))
        for k in ("dgate", "dw", "dbias", "dx"):
            assert torch.equal(g[k], want[k]), k


def test_refusals():
    cfg = synth.custom_config(d=64, E=8, k=2, f=64)
    i = synth.make_layer(cfg, 8, device="cuda")
    mk = lambda **kw: LayerShare(i.X, i.Wr, i.bias, cfg.k, i.placement, 0, i.w13, i.w2, **kw)
    for kw in (dict(gather_in_ffn=False), dict(fuse_combine=True), dict(shared_in_ffn=True)):
        with pytest.raises(ValueError, match="mxfp4"):
            mk(mxfp4=True, **kw)
    with pytest.raises(ValueError, match="bfloat16"):
        f = synth.make_layer(dataclasses.replace(cfg, dtype="f32"), 8, device="cuda")
        LayerShare(f.X, f.Wr, f.bias, cfg.k, f.placement, 0, f.w13, f.w2, mxfp4=True)
    dy = torch.zeros(8, 64, device="cuda", dtype=torch.bfloat16)
    fused = mk(fuse_combine=True)
    assert fused.fused_combine
    with pytest.raises(ValueError, match="y_perm"):
        fused.backward(dy)
    share = mk(mxfp4=True, renorm=False, want_logits=False)
    with pytest.raises(ValueError, match="want_logits"):
        share.backward(dy)
    share = mk(mxfp4=True)
    for bad in (dy.float(), dy[:7], dy[:, :32]):
        with pytest.raises(ValueError, match="dy must be"):
            share.backward(bad)


def test_placement_switch_quantizes_the_new_experts():
    cfg = synth.custom_config(**CFG)
    i, share = _share(cfg, 50, mxfp4=True)
    other = synth.make_layer(cfg, 50, seed=9, device="cuda")
    share.set_placement(i.placement, other.w13, other.w2)
    y = share.run().clone()
    fresh = LayerShare(i.X, i.Wr, i.bias, cfg.k, i.placement, 0, other.w13, other.w2, mxfp4=True)
    assert torch.equal(y, fresh.run())


def test_training_a_router_over_4_bit_experts(capsys):
    """From a router that starts off, held-out batches come closer to the original layer."""
    assert main(["--config", "qwen15_moe_a27b", "--tokens", "1024", "--steps", "25"]) == 0
    line = capsys.readouterr().out.strip().splitlines()[-1]
    say(line)
    before, after = (float(w) for w in line.replace(",", "").split() if w[0].isdigit())
    assert after < 0.8 * before
