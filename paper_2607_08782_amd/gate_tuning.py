"""Training the router of a layer whose experts are frozen in 4 or 8 bits.

A layer's experts take most of its weights and are cheap to hold in 4 bits; its
router is small and decides which of them answer.  Here a router is trained over
4-bit experts to reproduce the outputs of a layer with the original ones: over
batches of hidden states, the layer with 4-bit experts (`LayerShare(mxfp4=True)`)
is run beside the original, and its router, which starts away from the
original's, follows the gradient of the squared difference of their outputs, by
Adam on fp32 copies of its weights and bias.  The gradient is the layer's own
(`LayerShare.backward`): combine, gates, gate scores.

The experts are held in 4 bits or, with `--experts int8`, in 8-bit integers.  `--balance` adds a
balance loss over the routing to the loss, and `--max-norm` clips the gradient of the router's
weights and bias together (moe_grad_norm, moe_clip_grads); `--norm` trains over the residual
stream: the layer's rows are the norm of the batch and a residual, made in its own call.

One GPU holds every expert here (a layer that fits it in 4 bits); where experts
are spread, `backward` takes the reduction over GPUs of the gates' gradient.

    python -m paper_2607_08782_amd.gate_tuning --config deepseek_v2_lite --tokens 2048 --steps 60

On synthetic weights (60 batches of 2048 tokens) the held-out relative squared error goes
from 0.275 to 0.120 at the DeepSeek-V2-Lite shape and from 0.313 to 0.142 at
Qwen1.5-MoE's; 0.087 of it is the experts' rounding to 4 bits, the original router included.
"""
from __future__ import annotations

import argparse
import dataclasses
import os
import sys
from typing import List, Optional

import torch

if __package__ in (None, ""):
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    __package__ = "paper_2607_08782_amd"

from . import moe, synth  # noqa: E402
from .layer import LayerShare  # noqa: E402


class Adam:
    """Adam over fp32 tensors, in place."""

    def __init__(self, params: List[torch.Tensor], lr: float, beta1: float = 0.9, beta2: float = 0.99):
        self.params, self.lr, self.b1, self.b2, self.n = params, lr, beta1, beta2, 0
        self.m = [torch.zeros_like(p) for p in params]
        self.v = [torch.zeros_like(p) for p in params]

    def step(self, grads: List[torch.Tensor]):
        self.n += 1
        for p, g, m, v in zip(self.params, grads, self.m, self.v):
            m.lerp_(g, 1 - self.b1)
            v.lerp_(g * g, 1 - self.b2)
            scale = self.lr * (1 - self.b2 ** self.n) ** 0.5 / (1 - self.b1 ** self.n)
            p.addcdiv_(m, v.sqrt() + 1e-12, value=-scale)


class GateTuner:
    """A layer with 4-bit (or 8-bit) experts whose router is moved towards the original layer's
    outputs.  `inputs`: synth.LayerInputs with every expert on this GPU;  `router` [E, d]: where
    the layer's router starts;  `balance`: weight of the balance loss beside the outputs'
    difference;  `max_norm`: largest norm of a step's gradient (None: any);  `norm` [d]: weight of a
    norm in front of both layers, over the sum of a batch and `residual`."""

    def __init__(self, inputs: synth.LayerInputs, router: torch.Tensor, lr: float, renorm: bool = True,
                 experts: str = "mxfp4", balance: float = 0.0, max_norm: Optional[float] = None,
                 norm: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None):
        if experts not in ("mxfp4", "int8"):
            raise ValueError("experts are held as mxfp4 or int8")
        i, k = inputs, inputs.cfg.k
        front = dict(norm=norm, residual=residual)
        self.teacher = LayerShare(i.X, i.Wr, i.bias, k, i.placement, i.dev, i.w13, i.w2, renorm=renorm,
                                  fuse_combine=False, **front)
        self.router, self.bias = router.float(), i.bias.clone()        # the fp32 copies
        self.layer = LayerShare(i.X, self.router.to(i.Wr.dtype), self.bias, k, i.placement, i.dev, i.w13, i.w2,
                                renorm=renorm, **{experts: True}, **front)
        self.optimizer = Adam([self.router, self.bias], lr)
        self.balance, self.max_norm = balance, max_norm

    def loss_and_gradient(self, X: torch.Tensor, residual: Optional[torch.Tensor] = None):
        """Mean squared difference of the two layers' outputs over a batch, relative to the
        original's mean square (and `balance` times the balance loss), and its gradient
        ({"dw", "dbias", ...}; on the device)."""
        want = self.teacher
        want.set_inputs(X, residual=residual)
        self.layer.set_inputs(X, residual=residual)
        off = self.layer.run().float() - want.run().float()
        norm = want.y.float().square().sum()
        dy = (off * (2.0 / norm)).to(X.dtype)
        loss, g = off.square().sum() / norm, self.layer.backward(dy, balance=self.balance)
        return (loss + self.balance * g["balance_loss"][0] if self.balance else loss), g

    def step(self, X: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One step on a batch; returns its loss before the step (on the device)."""
        loss, g = self.loss_and_gradient(X, residual)
        if self.max_norm is not None:
            table = moe.GradTable([g["dw"], g["dbias"]])
            moe.moe_clip_grads(table, moe.moe_grad_norm(table), self.max_norm)
        self.optimizer.step([g["dw"], g["dbias"]])
        self.layer.Wr.copy_(self.router)
        return loss


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--config", default="deepseek_v2_lite", choices=sorted(c for c in synth.CONFIGS
                                                                         if synth.CONFIGS[c].dtype == "bf16"))
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=1e-3)
    ap.add_argument("--noise", type=float, default=0.5,
                    help="how far the router starts off: noise of this share of its weights' spread")
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--full-softmax", action="store_true",
                    help="gates from the softmax over all experts, not renormalised over the chosen ones")
    ap.add_argument("--experts", default="mxfp4", choices=("mxfp4", "int8"))
    ap.add_argument("--balance", type=float, default=0.0, help="weight of the balance loss")
    ap.add_argument("--max-norm", type=float, default=None, help="largest norm of a step's gradient")
    ap.add_argument("--norm", action="store_true", help="rows are the norm of a batch and a residual")
    a = ap.parse_args(argv)
    cfg = dataclasses.replace(synth.CONFIGS[a.config], G=1, replicas=0, shared_f=())
    inputs = synth.make_layer(cfg, a.tokens, seed=a.seed, device="cuda")
    noise = synth.normal(inputs.Wr.shape, a.seed, "noise", 0, a.noise * synth.WEIGHT_STD, "cuda")
    rows = lambda name, n: synth.normal((a.tokens, cfg.d), a.seed, name, n, 1.0, "cuda", cfg.torch_dtype)
    stream = (lambda n: rows("residual", n)) if a.norm else (lambda n: None)
    weight = (1 + synth.normal((cfg.d,), a.seed, "norm", 0, 0.2, "cuda")).to(cfg.torch_dtype) if a.norm else None
    tuner = GateTuner(inputs, inputs.Wr.float() + noise, a.lr, renorm=not a.full_softmax, experts=a.experts,
                      balance=a.balance, max_norm=a.max_norm, norm=weight, residual=stream(0))
    held_out = rows("X", 10 ** 6), stream(10 ** 6)
    before = float(tuner.loss_and_gradient(*held_out)[0])
    for n in range(a.steps):
        loss = tuner.step(rows("X", n + 1), stream(n + 1))
        if n % 10 == 0 or n + 1 == a.steps:
            print("step %3d: relative squared error %.6f" % (n, float(loss)), flush=True)
    after = float(tuner.loss_and_gradient(*held_out)[0])
    print("held-out batch: %.6f before, %.6f after" % (before, after), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
