"""A share with 8-bit experts, a norm in front of it and a balance loss on its routing: run and
gradient, alone, from a graph and in a stack (marked `gpu`)."""
import dataclasses

import numpy as np
import pytest
import torch

from paper_2607_08782_amd import moe, synth
from paper_2607_08782_amd.gate_tuning import GateTuner, main
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


def _weight(d, dtype=torch.bfloat16, seed=3):
    return (1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(seed))).to(dtype).cuda()


def _rows(T, d, dtype=torch.bfloat16, seed=4):
    return torch.randn(T, d, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


CFG = dict(d=256, E=16, k=4, f=192, G=3, replicas=2, zipf=1.2)


@pytest.mark.parametrize("T,shared_f", [(1, ()), (40, ()), (40, (64,)), (700, (64, 128))])
@pytest.mark.parametrize("front", ["rows", "norm", "residual"])
def test_share_with_8_bit_experts_is_its_calls(T, shared_f, front):
    say("[int8 share]", T, shared_f, front)
    cfg = synth.custom_config(**CFG, shared_f=shared_f)
    kw = {} if front == "rows" else dict(norm=_weight(cfg.d), norm_eps=1e-5)
    if front == "residual":
        kw["residual"] = _rows(T, cfg.d)
    i, share = _share(cfg, T, int8=True, **kw)
    y = share.run()
    torch.cuda.synchronize()
    rows, q, s = i.X, *moe.moe_quantize_int8(i.X)
    if kw:
        h, rows, rstd, q, s = moe.moe_rmsnorm(i.X, kw["norm"], residual=kw.get("residual"), eps=1e-5,
                                              want_rstd=True, want_q=True)
        assert torch.equal(share.hidden, h) and torch.equal(share.rstd, rstd)
    assert torch.equal(share.rows, rows) and torch.equal(share.xq, q) and torch.equal(share.x_scale, s)
    plain = LayerShare(rows, i.Wr, i.bias, cfg.k, i.placement, 0, i.w13, i.w2, shared=i.shared, shared_in_ffn=False)
    plain.run()
    for a, b in ((share.topk_idx, plain.topk_idx), (share.topk_gate, plain.topk_gate),
                 (share.counts, plain.counts), (share.perm["token_row"], plain.perm["token_row"])):
        assert torch.equal(a, b)
    N = int(share.perm["group_offsets"][-1])
    want = moe.moe_grouped_ffn_int8(q, s, share.perm["group_offsets"], moe.Int8WeightTable.quantized(i.w13, i.w2),
                                    row_token=share.perm["row_token"], cap_rows=max(N, 1))
    assert torch.equal(want[:N], share.y_perm[:N])
    want = moe.moe_combine(share.y_perm, share.perm["token_row"], share.topk_gate, share.y_shared, T=T, d=cfg.d)
    assert torch.equal(y[:T], want)
    if shared_f:
        assert torch.equal(share.y_shared[:T], plain.y_shared[:T])


@pytest.mark.parametrize("kw", [dict(), dict(mxfp4=True), dict(fuse_combine=False)])
def test_other_experts_behind_a_norm(kw):
    """bf16 and 4-bit shares: what a share of the normed rows gives."""
    cfg = synth.custom_config(**CFG)
    w, r = _weight(cfg.d), _rows(60, cfg.d)
    i, share = _share(cfg, 60, norm=w, residual=r, **kw)
    rows = moe.moe_rmsnorm(i.X, w, residual=r)[1]
    plain = LayerShare(rows, i.Wr, i.bias, cfg.k, i.placement, 0, i.w13, i.w2, **kw)
    assert torch.equal(share.run(), plain.run())
    torch.cuda.synchronize()


@pytest.mark.parametrize("T", [1, 16, 300])
def test_share_replays_from_a_graph(T):
    """A step and its gradient, balance loss included, beside eager steps of the same share."""
    say("[int8 graph]", T)
    cfg = synth.custom_config(**CFG)
    w, r = _weight(cfg.d), _rows(T, cfg.d)
    _, share = _share(cfg, T, int8=True, norm=w, residual=r)
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    dy = _rows(T, cfg.d, seed=9)
    dw, dh = torch.empty(cfg.d, device="cuda"), torch.empty_like(share.X)

    def step():
        y = share.run()
        g = share.backward(dy, balance=0.1, mask=mask)
        share.backward_norm(g["dx"], dh_add=dy, dh=dh, dw=dw)
        return [y, dh, dw] + [g[k] for k in sorted(g)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                       # allocates its buffers
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = step()
    for n in range(4):
        share.X.copy_(_rows(T, cfg.d, seed=20 + n))
        r.copy_(_rows(T, cfg.d, seed=30 + n))
        dy.copy_(_rows(T, cfg.d, seed=40 + n))
        mask.copy_(torch.rand(T, generator=torch.Generator().manual_seed(n)) > 0.3)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        again = step()
        torch.cuda.synchronize()
        for a, b in zip(got, again):
            assert torch.equal(a, b), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("padding", [0.0, 0.3])
def test_gradient_of_a_layer_with_norm_and_balance_loss(dtype, renorm, padding):
    """One GPU with every expert: the gradients of <dy, y> + 0.2 times the balance loss, to the sum in
    front of the norm, the norm's weight and the router, with the experts' own gradient from
    elementary products, against autograd of the definition in float64 (the choice of experts as
    the share made it).  fp32: 1e-5 of the largest value, and 2e-5 past the norm, whose gradient
    subtracts two such.  bf16: six roundings of 2^-8 on the way (the normed rows, h, y_perm, dy_perm,
    dx_perm's and dx's), whose errors are independent over sums of hundreds of terms: 2^-6 of the
    largest value."""
    say("[norm layer grad]", dtype, renorm, padding)
    T = 200
    cfg = synth.custom_config(dtype=dtype, d=128, E=12, k=3, f=64, zipf=1.0)
    dt = cfg.torch_dtype
    w, r = _weight(cfg.d, dt), _rows(T, cfg.d, dt)
    i, share = _share(cfg, T, renorm=renorm, fuse_combine=False, norm=w, residual=r)
    share.run()
    dy = _rows(T, cfg.d, dt, seed=5)
    add = _rows(T, cfg.d, dt, seed=6)
    mask = torch.rand(T, generator=torch.Generator().manual_seed(1)) >= padding if padding else None
    weight = 0.2 * T
    g = share.backward(dy, balance=weight, mask=None if mask is None else mask.cuda())
    off = share.perm["group_offsets"].tolist()
    tok = share.perm["row_token"].long()
    dx_perm = torch.zeros_like(share.y_perm)
    for s in range(cfg.E):                           # the experts' gradient, by plain products
        if off[s] == off[s + 1]:
            continue
        x = share.rows[tok[off[s]:off[s + 1]]].float().requires_grad_()
        a, b = x @ i.w13[s][:cfg.f].float().t(), x @ i.w13[s][cfg.f:].float().t()
        ((torch.nn.functional.silu(a) * b) @ i.w2[s].float().t()).backward(g["dy_perm"][off[s]:off[s + 1]].float())
        dx_perm[off[s]:off[s + 1]] = x.grad.to(dt)
    drows = share.backward_rows(dx_perm)
    dh, dnorm = share.backward_norm(drows, dh_add=add)
    torch.cuda.synchronize()

    H = share.hidden.double().cpu().requires_grad_()
    N = w.double().cpu().requires_grad_()
    W = i.Wr.double().cpu().requires_grad_()
    bias = i.bias.double().cpu().requires_grad_()
    X = H / (H.square().mean(1, keepdim=True) + 1e-6).sqrt() * N
    logits = X @ W.t() + bias
    idx = share.topk_idx.long().cpu()
    gate = torch.softmax(logits.gather(1, idx), 1) if renorm else torch.softmax(logits, 1).gather(1, idx)
    y = torch.zeros(T, cfg.d, dtype=torch.float64)
    for e in range(cfg.E):
        h = torch.nn.functional.silu(X @ i.w13[e][:cfg.f].double().cpu().t()) * (X @ i.w13[e][cfg.f:].double().cpu().t())
        y = y + (h @ i.w2[e].double().cpu().t()) * (gate * (idx == e)).sum(1, keepdim=True)
    live = torch.ones(T, dtype=torch.bool) if mask is None else mask
    n = int(live.sum())
    counts = torch.bincount(idx[live].flatten(), minlength=cfg.E).double()
    balance = cfg.E * (counts / (cfg.k * n) * torch.softmax(logits, 1)[live].sum(0) / n).sum()
    ((y * dy.double().cpu()).sum() + (H * add.double().cpu()).sum() + weight * balance).backward()
    assert abs(float(g["balance_loss"]) - balance.item()) <= (1e-5 if dtype == "f32" else 2.0 ** -8) * balance.item()
    tol = 1e-5 if dtype == "f32" else 2.0 ** -6
    for name, got, want, t in (("dw", g["dw"], W.grad, tol), ("dbias", g["dbias"], bias.grad, tol),
                               ("dh", dh, H.grad, 2 * tol if dtype == "f32" else tol),
                               ("dnorm", dnorm, N.grad, 2 * tol if dtype == "f32" else tol)):
        err = float((got.double().cpu() - want).abs().max() / want.abs().max())
        say("  ", name, "%.2e" % err)
        assert err <= t, (name, err)


def test_balance_loss_is_its_calls():
    cfg = synth.custom_config(**CFG)
    _, share = _share(cfg, 90, int8=True)
    share.run()
    mask = torch.arange(90, device="cuda") < 70
    b = share.balance_loss(0.3, mask)
    loss, counts, sums, n = moe.moe_balance_loss(share.logits, share.topk_idx, mask=mask)
    dl = moe.moe_balance_loss_backward(share.logits, counts, n, cfg.k, scale=0.3, mask=mask)
    for a, c in zip((b["loss"], b["counts"], b["prob_sum"], b["n_tokens"], b["dlogits"]), (loss, counts, sums, n, dl)):
        assert torch.equal(a, c)
    dy = _rows(90, cfg.d)
    plain = {k: v.clone() for k, v in share.backward(dy).items()}
    assert "balance_loss" not in plain
    with_loss = share.backward(dy, balance=0.3, mask=mask)
    assert torch.equal(with_loss["dy_perm"], plain["dy_perm"]) and torch.equal(with_loss["dgate"], plain["dgate"])
    want = moe.moe_route_topk_backward(plain["dgate"], share.topk_gate, share.topk_idx, share.X, share.Wr,
                                       dlogits_add=dl)
    for k, w in zip(("dx", "dw", "dbias"), want[1:]):
        assert torch.equal(with_loss[k], w) and not torch.equal(with_loss[k], plain[k]), k


@pytest.mark.parametrize("T", [5, 400])
def test_two_layers_of_a_residual_stream(T):
    """Layer after layer as a program runs them: the second's rows are the norm of the stream that the
    first's sum and output make; backward through both, and the step's gradients clipped together;
    eager, and replayed from one graph."""
    say("[two layers]", T)
    cfg = dataclasses.replace(synth.custom_config(**CFG), G=1, replicas=0)
    X, r = _rows(T, cfg.d, seed=1), _rows(T, cfg.d, seed=2)
    first = synth.make_layer(cfg, T, seed=0, device="cuda")
    second = synth.make_layer(cfg, T, seed=1, device="cuda")
    mk = lambda i, X, r, s: LayerShare(X, i.Wr, i.bias, cfg.k, i.placement, 0, i.w13, i.w2, int8=True,
                                       norm=_weight(cfg.d, seed=s), residual=r)
    a = mk(first, X, r, 5)
    b = mk(second, a.y, a.hidden, 6)
    assert a.y.shape == X.shape
    dy = _rows(T, cfg.d, seed=3)
    grads = None
    out = {k: torch.empty(n, device="cuda") for k, n in (("na", cfg.d), ("nb", cfg.d))}

    def step():
        nonlocal grads
        a.run()
        b.run()
        gb = b.backward(dy, balance=0.01)
        # (through the scores alone: the experts are frozen, and their rows' gradient is zero here)
        dhb, _ = b.backward_norm(gb["dx"], dh_add=dy, dw=out["nb"])
        ga = a.backward(dhb, balance=0.01)
        dha, _ = a.backward_norm(ga["dx"], dh_add=dhb, dw=out["na"])
        grads = moe.GradTable([ga["dw"], ga["dbias"], gb["dw"], gb["dbias"], out["na"], out["nb"]])
        norm = moe.moe_grad_norm(grads)
        before = [t.clone() for t in grads.grads]
        moe.moe_clip_grads(grads, norm, 0.5)
        return [b.y, dha, norm] + grads.grads, before
    step()
    torch.cuda.synchronize()
    got, before = step()
    torch.cuda.synchronize()
    exact = float(torch.cat([t.double().flatten() for t in before]).norm())
    assert exact > 0.5 and abs(float(got[2]) - exact) <= 2.0 ** -23 * exact
    assert abs(float(torch.cat([t.double().flatten() for t in got[3:]]).norm()) - 0.5) <= 1e-6
    # the same by hand
    h, rows = moe.moe_rmsnorm(X, a.norm, residual=r)[:2]
    h2, rows2 = moe.moe_rmsnorm(a.y, b.norm, residual=h)[:2]
    assert torch.equal(a.rows, rows) and torch.equal(b.hidden, h2) and torch.equal(b.rows, rows2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held, _ = step()
    for n in range(4):
        X.copy_(_rows(T, cfg.d, seed=50 + n))
        dy.copy_(_rows(T, cfg.d, seed=60 + n))
        g.replay()
        torch.cuda.synchronize()
        seen = [t.clone() for t in held]
        for x, y in zip(seen, step()[0]):
            assert torch.equal(x, y), n


def test_placement_switch_quantizes_the_new_experts():
    cfg = synth.custom_config(**CFG)
    i, share = _share(cfg, 50, int8=True)
    other = synth.make_layer(cfg, 50, seed=9, device="cuda")
    old = share.weights
    g = torch.cuda.CUDAGraph()
    share.run()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        share.run()
    share.set_placement(i.placement, other.w13, other.w2)
    assert share.captured_tables == [old]
    y = share.run().clone()
    fresh = LayerShare(i.X, i.Wr, i.bias, cfg.k, i.placement, 0, other.w13, other.w2, int8=True)
    assert torch.equal(y, fresh.run())
    g.replay()                                       # goes on with the experts that it was captured with
    torch.cuda.synchronize()
    assert torch.equal(share.y, LayerShare(i.X, i.Wr, i.bias, cfg.k, i.placement, 0, i.w13, i.w2, int8=True).run())


def test_refusals():
    cfg = synth.custom_config(d=64, E=8, k=2, f=64)
    i = synth.make_layer(cfg, 8, device="cuda")
    mk = lambda **kw: LayerShare(i.X, i.Wr, i.bias, cfg.k, i.placement, 0, i.w13, i.w2, **kw)
    for kw in (dict(gather_in_ffn=False), dict(fuse_combine=True), dict(shared_in_ffn=True)):
        with pytest.raises(ValueError, match="int8"):
            mk(int8=True, **kw)
    with pytest.raises(ValueError, match="4 bits or in 8"):
        mk(int8=True, mxfp4=True)
    with pytest.raises(ValueError, match="bfloat16"):
        f = synth.make_layer(dataclasses.replace(cfg, dtype="f32"), 8, device="cuda")
        LayerShare(f.X, f.Wr, f.bias, cfg.k, f.placement, 0, f.w13, f.w2, int8=True)
    w, r = _weight(64), _rows(8, 64)
    for bad in (w.float(), w[:32]):
        with pytest.raises(ValueError, match="norm must be"):
            mk(norm=bad)
    with pytest.raises(ValueError, match="in front of the norm"):
        mk(residual=r)
    with pytest.raises(ValueError, match="residual must be"):
        mk(norm=w, residual=r[:7])
    share = mk(norm=w, int8=True, want_logits=False)
    with pytest.raises(ValueError, match="without a residual"):
        share.set_inputs(i.X, residual=r)
    with pytest.raises(ValueError, match="none was made"):
        share.backward_norm(r)
    with pytest.raises(ValueError, match="want_logits"):
        share.balance_loss()
    share.run()
    with pytest.raises(ValueError, match="want_logits"):
        share.backward(r, balance=0.1)
    with pytest.raises(ValueError, match="no norm"):
        mk().backward_norm(r)
    with pytest.raises(ValueError, match="none was made"):
        mk().balance_loss()
    with pytest.raises(ValueError, match="mxfp4 or int8"):
        GateTuner(i, i.Wr.float(), 1e-3, experts="int4")


def test_tuning_a_router_over_8_bit_experts_runs(capsys):
    args = ["--config", "qwen15_moe_a27b", "--tokens", "512", "--steps", "2", "--experts", "int8", "--balance", "0.01",
            "--max-norm", "0.05"]
    assert main(args) == 0 and main(args + ["--norm"]) == 0
    assert capsys.readouterr().out.count("held-out batch") == 2


def test_gradient_of_the_tuning_loss():
    """A step's gradient against the definition in float64: of the outputs' difference and the balance
    loss, by the router's weights and bias, with the rows y_perm of the 8-bit experts as they are;
    clipped to a tenth of its norm it is the same direction, that long.  bf16 rounds y (twice), dy
    and dlogits' operands on the way: 2^-6 of the largest value."""
    cfg = dataclasses.replace(synth.custom_config(d=128, E=12, k=3, f=64, zipf=1.0), G=1, replicas=0)
    i = synth.make_layer(cfg, 150, device="cuda")
    start = i.Wr.float() + 0.01 * torch.randn(i.Wr.shape, generator=torch.Generator().manual_seed(1)).cuda()
    tuner = GateTuner(i, start.clone(), 1e-3, experts="int8", balance=0.5)    # (it keeps what it is given)
    loss, g = tuner.loss_and_gradient(i.X)
    layer, want = tuner.layer, tuner.teacher.y.double().cpu()
    W = layer.Wr.double().cpu().requires_grad_()
    b = layer.bias.double().cpu().requires_grad_()
    logits = i.X.double().cpu() @ W.t() + b
    idx, row = layer.topk_idx.long().cpu(), layer.perm["token_row"].long().cpu()
    gate = torch.softmax(logits.gather(1, idx), 1)
    y = (gate[..., None] * layer.y_perm.double().cpu()[row]).sum(1)
    counts = torch.bincount(idx.flatten(), minlength=12).double()
    exact = (y - want).square().sum() / want.square().sum() + \
        0.5 * 12 * (counts / (3 * 150) * torch.softmax(logits, 1).sum(0) / 150).sum()
    exact.backward()
    assert abs(float(loss) - exact.item()) <= 2.0 ** -6 * exact.item()
    for got, ref in ((g["dw"], W.grad), (g["dbias"], b.grad)):
        err = float((got.double().cpu() - ref).abs().max() / ref.abs().max())
        say("  ", "%.2e" % err)
        assert err <= 2.0 ** -6
    whole = [g["dw"].clone(), g["dbias"].clone()]
    norm = float(torch.cat([t.double().flatten() for t in whole]).norm())
    tuner.max_norm = 0.1 * norm
    tuner.step(i.X)
    for t, ref in zip((layer._grads["dw"], layer._grads["dbias"]), whole):
        assert (t.double() - 0.1 * ref.double()).abs().max() <= 2.0 ** -22 * 0.1 * ref.abs().max()
    assert not torch.equal(tuner.router, start)
