"""Operators of a layer with 8-bit integer experts as cases that can be timed and compared:
the norm in front of it, its experts, and what its router's training adds.

* `int8_ffn`   the grouped SwiGLU FFN of experts whose weights are held in 8-bit integers:
               integer products of token rows and weights, a scale for each token and each
               output channel, the hidden rows to 8 bits between the two products
* `norm`       the residual's addition, the root-mean-square norm of the sum, and the normed
               rows in 8 bits with a scale for each
* `norm_grad`  its gradient: of the rows (on top of what reached them through the residual
               stream) and of the weight
* `balance`    the balance loss of a routing, its per-expert counts and mean scores, and the
               gradient of the gate scores
* `clip`       the norm over all gradients of a step, and their clipping to a largest one

8-bit rows here: scale = max |x| / 127 of the row (2^-126 at least), values rounded to
nearest, ties to even; rows are padded with zeros to a multiple of 128 columns.

Layer shapes and popularity are the repository's configurations, from one token to their
largest batch, and generic odd sizes beside them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

WEIGHT_STD = 0.02
EPS = 1e-6
# (hidden size, experts, experts per token, expert FFN size, GPUs, popularity exponent,
#  longest batch)
SHAPES = {
    "mixtral_8x7b": (4096, 8, 2, 14336, 4, 1.0, 4096),
    "deepseek_v2_lite": (2048, 64, 6, 1408, 8, 1.2, 8192),
    "qwen15_moe_a27b": (2048, 60, 4, 1408, 8, 1.2, 4096),
    "qwen3_30b_a3b": (2048, 128, 8, 768, 9, 1.5, 16384),
    # the small parity layer and an odd-sized one
    "tiny": (128, 8, 2, 256, 1, 0.0, 1024),
    "odd": (1000, 24, 3, 328, 2, 1.0, 4096),
}


def listed():
    return [
        # one sequence decoding alone, all experts here: the smallest step, launches and latency
        {"name": "ffn_single", "kind": "int8_ffn", "shape": "deepseek_v2_lite", "T": 1, "gpus": 1},
        # a decode step over 64 running sequences: bound by the weights it reads
        {"name": "ffn_decode", "kind": "int8_ffn", "shape": "mixtral_8x7b", "T": 64},
        # an odd-sized chunk of a prompt over many narrow experts: ragged groups of rows
        {"name": "ffn_chunk", "kind": "int8_ffn", "shape": "qwen15_moe_a27b", "T": 1111},
        # prompt processing over 2 of 8 wide experts: the largest products
        {"name": "ffn_prefill", "kind": "int8_ffn", "shape": "mixtral_8x7b", "T": 4096},
        # one decode step's rows in front of a layer: latency
        {"name": "norm_decode", "kind": "norm", "shape": "mixtral_8x7b", "T": 7, "dtype": "bf16",
         "residual": True},
        # the longest batch: the memory's rate
        {"name": "norm_large", "kind": "norm", "shape": "qwen3_30b_a3b", "T": 16384, "dtype": "bf16",
         "residual": True},
        # training over a long batch
        {"name": "norm_grad_large", "kind": "norm_grad", "shape": "deepseek_v2_lite", "T": 8192,
         "dtype": "bf16"},
        # a short odd batch in 32 bits
        {"name": "norm_grad_odd", "kind": "norm_grad", "shape": "odd", "T": 333, "dtype": "f32"},
        # 128 experts over the longest batch, every token counts
        {"name": "balance_large", "kind": "balance", "shape": "qwen3_30b_a3b", "T": 16384, "padding": 0.0},
        # a padded, odd-sized batch
        {"name": "balance_padded", "kind": "balance", "shape": "qwen15_moe_a27b", "T": 777, "padding": 0.3},
        # the routers, their biases and the norms in front of them, of a stack of layers: many
        # small tensors
        {"name": "clip_routers", "kind": "clip", "shape": "deepseek_v2_lite", "what": "routers",
         "layers": 27, "dtype": "f32", "norm": 0.5},
        # the experts of one layer that are on this GPU: long tensors
        {"name": "clip_experts", "kind": "clip", "shape": "deepseek_v2_lite", "what": "experts",
         "layers": 1, "dtype": "f32", "norm": 0.5},
    ]


def _size(rng, lo, hi):
    """Log-uniform in [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("int8_ffn", "int8_ffn", "norm", "norm_grad", "balance", "clip"))
    shape = rng.choice(sorted(SHAPES))
    if kind == "clip":
        what = rng.choice(("routers", "experts"))
        if what == "experts" and shape == "mixtral_8x7b":
            shape = "qwen15_moe_a27b"          # (their gradients alone are larger than any case)
        return {"kind": kind, "shape": shape, "what": what,
                "layers": _size(rng, 1, 48) if what == "routers" else 1,
                "dtype": rng.choice(("f32", "bf16")),
                # the largest norm, relative to the one expected: over 1 clips nothing
                "norm": round(rng.uniform(0.1, 1.5), 3)}
    case = {"kind": kind, "shape": shape, "T": _size(rng, 1, SHAPES[shape][6])}
    if kind == "int8_ffn" and shape == "deepseek_v2_lite" and case["T"] <= 1024:
        case["gpus"] = 1                       # 8-bit experts: a whole layer on one GPU
    if kind in ("norm", "norm_grad"):
        case["dtype"] = "f32" if shape == "tiny" else rng.choice(("bf16", "bf16", "f32"))
    if kind == "norm":
        case["residual"] = rng.random() < 0.7
    if kind == "balance":
        case["padding"] = rng.choice((0.0, round(rng.random(), 3)))
    return case


# ---------------------------------------------------------------------------
# inputs

def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _normal(g, shape, std=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


def _bias(shape):
    """Router bias of expert popularity ranks 1, 2, ...: selection roughly by Zipf's law."""
    d, E, _, _, _, zipf, _ = SHAPES[shape]
    p = np.arange(1, E + 1, dtype=np.float64) ** -zipf
    beta = WEIGHT_STD * math.sqrt(d) * math.sqrt(6.0) / math.pi
    return beta * np.log(p / p.sum()) if zipf else np.zeros(E)


def _local(case):
    """The experts on this GPU: every G-th by popularity."""
    _, E, _, _, G, _, _ = SHAPES[case["shape"]]
    return list(range(0, E, case.get("gpus", G)))


def _scores(case, g):
    """Gate scores of a batch and its choice of experts."""
    d, E, k, _, _, _, _ = SHAPES[case["shape"]]
    bias = torch.from_numpy(_bias(case["shape"])).float().cuda()
    logits = _normal(g, (case["T"], E), WEIGHT_STD * math.sqrt(d)) + bias
    return logits, torch.topk(logits, k, dim=1)[1]


def _row_maps(case, idx):
    """Rows of the experts here: grouped by expert, ascending tokens in a group."""
    _, E, k, _, _, _, _ = SHAPES[case["shape"]]
    T, here = case["T"], _local(case)
    slot = torch.full((E,), len(here), device="cuda")
    slot[torch.tensor(here, device="cuda")] = torch.arange(len(here), device="cuda")
    where = slot[idx].flatten()
    order = torch.argsort(where, stable=True)
    counts = torch.bincount(where, minlength=len(here) + 1)[:len(here)]
    offsets = torch.zeros(len(here) + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    n, cap = int(offsets[-1]), T * min(k, len(here))
    return {"offsets": offsets, "sizes": counts.tolist(), "rows": n, "cap": cap,
            "row_token": torch.nn.functional.pad((order[:n] // k).int(), (0, cap - n))}


def _int8_weights(g, rows, cols):
    # channels of unlike magnitudes, as the rows of a trained matrix are
    w = _normal(g, (rows, cols), WEIGHT_STD).mul_(torch.exp(_normal(g, (rows, 1), 0.3)))
    return _int8_encode(w.to(torch.bfloat16).float())


def _grad_shapes(case):
    """Shapes of the gradients of a step."""
    d, E, _, f, _, _, _ = SHAPES[case["shape"]]
    if case["what"] == "routers":
        return [(E, d), (E,), (d,)] * case["layers"]
    return [(2 * f, d), (d, f)] * len(_local(case))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"case": case}
    d, E, k, f, _, _, _ = SHAPES[case["shape"]]
    if case["kind"] == "clip":
        shapes, dt = _grad_shapes(case), _dtype(case)
        s["grads"] = [_normal(g, shape, math.exp(0.5 * (i % 3)) * 1e-3, dt) for i, shape in enumerate(shapes)]
        at, total = [], 0
        for shape in shapes:
            at.append(total)
            total += (math.prod(shape) + 63) // 64 * 64
        # a step's clipped gradients, one behind the other
        s["flat"] = torch.zeros(total, dtype=dt, device="cuda")
        s["out"] = [s["flat"][a:a + math.prod(shape)].view(shape) for a, shape in zip(at, shapes)]
        s["max_norm"] = case["norm"] * 1e-3 * math.sqrt(
            sum(math.exp(i % 3) * math.prod(shape) for i, shape in enumerate(shapes)))
        if own:
            # what a training program keeps: the table of its gradients, and the workspace
            from paper_2607_08782_amd import moe
            s["table"] = moe.GradTable(s["grads"], out=s["out"])
            s["ws"] = moe.workspace(moe.moe_grad_norm_ws_bytes(s["table"]), "cuda")
        return s
    T, dt = case["T"], _dtype(case)
    if case["kind"] == "norm":
        # hidden rows grow in magnitude over a model's layers
        s["x"] = _normal(g, (T, d)).mul_(torch.exp(_normal(g, (T, 1), 0.5))).to(dt)
        s["residual"] = _normal(g, (T, d), dtype=dt) if case["residual"] else None
        s["weight"] = (1.0 + _normal(g, (d,), 0.2)).to(dt)
        return s
    if case["kind"] == "norm_grad":
        s["h"] = _normal(g, (T, d)).mul_(torch.exp(_normal(g, (T, 1), 0.5))).to(dt)
        s["rstd"] = (s["h"].double().square().mean(1) + EPS).rsqrt().float()
        s["weight"] = (1.0 + _normal(g, (d,), 0.2)).to(dt)
        s["dy"] = _normal(g, (T, d), dtype=dt)
        s["dh_add"] = _normal(g, (T, d), dtype=dt)
        return s
    s["logits"], idx = _scores(case, g)
    s["idx"] = idx.int()
    if case["kind"] == "balance":
        # the sequences of a padded batch end anywhere
        keep = torch.rand(T, generator=g, device="cuda") >= case["padding"]
        s["mask"] = keep if case["padding"] > 0 else None
        return s
    s.update(_row_maps(case, idx))
    s["xq"], s["x_scale"] = _int8_encode(_normal(g, (T, d), dtype=torch.bfloat16).float())
    s["w13"] = [_int8_weights(g, 2 * f, d) for _ in s["sizes"]]
    s["w2"] = [_int8_weights(g, d, f) for _ in s["sizes"]]
    if own:
        # what a serving program keeps: the weight table and the workspace
        from paper_2607_08782_amd import moe
        s["table"] = moe.Int8WeightTable(s["w13"], s["w2"], d, f)
        s["ws"] = moe.workspace(moe.moe_grouped_ffn_int8_ws_bytes(s["cap"], d, f, len(s["sizes"])), "cuda")
    # the row buffer of a serving program, as long as a batch can need it
    s["y_perm"] = torch.zeros((s["cap"], d), dtype=torch.bfloat16, device="cuda")
    return s


# ---------------------------------------------------------------------------
# the plain forms

def _int8_encode(v):
    """Codes [rows][padded cols] int8 and scales [rows] of the rows of v (32 bits)."""
    scale = (v.abs().amax(1) / 127.0).clamp_(min=2.0 ** -126)
    code = torch.round(v / scale[:, None]).to(torch.int8)
    return torch.nn.functional.pad(code, (0, -v.shape[1] % 128)), scale


def _plain_ffn(s):
    d, _, _, f, _, _, _ = SHAPES[s["case"]["shape"]]
    n, sizes, dev = s["rows"], s["sizes"], s["xq"].device
    if n == 0:
        return s["y_perm"]
    w13 = torch.stack([q[:, :d] for q, _ in s["w13"]]).float()
    w2 = torch.stack([q[:, :f] for q, _ in s["w2"]]).float()
    s13, s2 = (torch.stack([t for _, t in s[w]])[:, None, :] for w in ("w13", "w2"))
    # every group padded to the longest one's rows: one product for all of them
    offsets = s["offsets"].long()
    row = torch.arange(n, device=dev)
    group = torch.searchsorted(offsets, row, right=True) - 1
    place = group * max(sizes) + row - offsets[group]
    token = s["row_token"][:n].long()
    codes = torch.zeros((len(sizes) * max(sizes), d), device=dev)
    codes[place] = s["xq"][token, :d].float()
    scale = torch.zeros(len(sizes) * max(sizes), device=dev)
    scale[place] = s["x_scale"][token]
    ab = torch.bmm(codes.view(len(sizes), -1, d), w13.transpose(1, 2))
    ab = ab * scale.view(len(sizes), -1, 1) * s13
    a, b = ab[..., :f], ab[..., f:]
    h = (a / (1.0 + torch.exp(-a)) * b).to(torch.bfloat16).float()
    codes, scale = _int8_encode(h.reshape(-1, f))
    y = torch.bmm(codes[:, :f].float().view(len(sizes), -1, f), w2.transpose(1, 2))
    y = y * scale.view(len(sizes), -1, 1) * s2
    s["y_perm"][:n] = y.view(-1, d)[place].to(torch.bfloat16)
    return s["y_perm"]


def _plain_norm(s):
    x, d = s["x"], s["x"].shape[1]
    h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    v = h.float()
    rstd = 1.0 / torch.sqrt(v.square().mean(1) + EPS)
    y = (v * rstd[:, None] * s["weight"].float()).to(x.dtype)
    code, scale = _int8_encode(y.float())
    # the 8-bit rows as the values they stand for
    return {"h": h, "y": y, "rstd": rstd, "q": (code[:, :d].float() * scale[:, None]).to(torch.bfloat16)}


def _plain_norm_grad(s):
    h, r = s["h"].float(), s["rstd"][:, None]
    n = h * r
    up = s["dy"].float()
    g = up * s["weight"].float()
    dh = r * (g - n * (g * n).mean(1, keepdim=True)) + s["dh_add"].float()
    dw = (up * n).sum(0, dtype=torch.float64)
    return {"dh": dh.to(s["h"].dtype), "dw": dw.float()}


def _plain_balance(s):
    l, mask = s["logits"], s["mask"]
    T, E = l.shape
    k = s["idx"].shape[1]
    live = torch.ones(T, device=l.device) if mask is None else mask.float()
    p = torch.exp(l - l.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True) * live[:, None]
    sent = torch.zeros(T, E, device=l.device).scatter(1, s["idx"].long(), 1.0) * live[:, None]
    counts = sent.sum(0, dtype=torch.float64)
    prob_sum = p.sum(0, dtype=torch.float64)
    n = live.sum(dtype=torch.float64).clamp(min=1.0)
    scale = E / (k * n * n)
    # the mean of the counts leaves the gradient as it is, and its rounding small
    c = counts - counts.mean()
    dlogits = p * (c - (p.double() * c).sum(1, keepdim=True)) * scale
    return {"loss": ((counts * prob_sum).sum() * scale).float().view(1), "counts": counts.int(),
            "prob_sum": prob_sum.float(), "dlogits": dlogits.float()}


def _plain_clip(s):
    sums = [g.float().square().sum(dtype=torch.float64) for g in s["grads"]]
    norm = torch.stack(sums).sum().sqrt().float().view(1)
    factor = torch.where(norm <= s["max_norm"], torch.ones_like(norm), s["max_norm"] / norm)
    for g, out in zip(s["grads"], s["out"]):
        out.copy_(g.float() * factor)
    return {"norm": norm, "grads": s["flat"]}


PLAIN = {"int8_ffn": _plain_ffn, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
         "balance": _plain_balance, "clip": _plain_clip}


# ---------------------------------------------------------------------------
# one pass

def _own(s):
    from paper_2607_08782_amd import moe

    kind = s["case"]["kind"]
    if kind == "int8_ffn":
        return moe.moe_grouped_ffn_int8(s["xq"], s["x_scale"], s["offsets"], s["table"],
                                        row_token=s["row_token"], cap_rows=s["cap"], y_perm=s["y_perm"],
                                        ws=s["ws"])
    if kind == "norm":
        h, y, rstd, q, scales = moe.moe_rmsnorm(s["x"], s["weight"], residual=s["residual"], eps=EPS,
                                                want_rstd=True, want_q=True)
        return {"h": h, "y": y, "rstd": rstd,
                "q": moe.moe_dequantize_int8(q, scales, s["x"].shape[1], dtype=torch.bfloat16)}
    if kind == "norm_grad":
        dh, dw = moe.moe_rmsnorm_backward(s["dy"], s["h"], s["weight"], s["rstd"], dh_add=s["dh_add"])
        return {"dh": dh, "dw": dw}
    if kind == "balance":
        loss, counts, prob_sum, n_tokens = moe.moe_balance_loss(s["logits"], s["idx"], mask=s["mask"])
        dlogits = moe.moe_balance_loss_backward(s["logits"], counts, n_tokens, s["idx"].shape[1],
                                                mask=s["mask"])
        return {"loss": loss, "counts": counts, "prob_sum": prob_sum, "dlogits": dlogits}
    norm = moe.moe_grad_norm(s["table"], ws=s["ws"])
    moe.moe_clip_grads(s["table"], norm, s["max_norm"])
    return {"norm": norm, "grads": s["flat"]}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["kind"]](state)


def _expected(case):
    """Rows that a batch brings to the experts here, and how many of these experts get any."""
    d, E, k, _, _, _, _ = SHAPES[case["shape"]]
    r = np.random.RandomState(1)
    score = r.standard_normal((4096, E)) * WEIGHT_STD * math.sqrt(d) + _bias(case["shape"])
    chosen = np.zeros((4096, E), bool)
    np.put_along_axis(chosen, np.argpartition(-score, k - 1, 1)[:, :k], True, 1)
    p = chosen.mean(0)[_local(case)]
    return case["T"] * p.sum(), (1 - (1 - p) ** case["T"]).sum()


def work(case):
    size = 4 if case.get("dtype") == "f32" else 2
    if case["kind"] == "clip":
        n = sum(math.prod(shape) for shape in _grad_shapes(case))
        return {"bytes": 2 * n * size, "flops": 3 * n}
    d, E, k, f, _, _, _ = SHAPES[case["shape"]]
    T = case["T"]
    if case["kind"] == "norm":
        # the rows (and the residual), their sum, the normed rows, their codes and the values
        return {"bytes": T * d * ((4 if case["residual"] else 2) * size + 3) + T * 8 + d * size,
                "flops": T * d * 6}
    if case["kind"] == "norm_grad":
        return {"bytes": 4 * T * d * size + T * 4 + d * (size + 4), "flops": T * d * 10}
    if case["kind"] == "balance":
        return {"bytes": 2 * T * E * 4 + T * k * 4 + E * 8, "flops": T * E * 10}
    rows, experts = _expected(case)
    return {"bytes": min(T, rows) * (d + 4) + experts * (3 * d * f + (2 * f + d) * 4) + rows * d * 2,
            "flops": rows * 6 * d * f}


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def _int8_round64(v):
    """Every row of v at the nearest of the 255 values that its scale gives."""
    step = (v.abs().max(1, keepdim=True).values / 127.0).clamp(min=2.0 ** -126)
    return (v / step).round() * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "clip":
        total = 0.0
        for g in s["grads"]:
            total += float((g.double() ** 2).sum())
        norm = math.sqrt(total)
        factor = min(1.0, s["max_norm"] / norm)
        flat, at = torch.zeros(s["flat"].shape, dtype=torch.float64, device="cuda"), 0
        for g in s["grads"]:
            flat[at:at + g.numel()] = g.double().flatten() * factor
            at += -(-g.numel() // 64) * 64
        return {"norm": torch.tensor([norm], dtype=torch.float64), "grads": flat}
    d, E, k, f, _, _, _ = SHAPES[case["shape"]]
    T = case["T"]
    if case["kind"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h = (h + s["residual"].double()).to(s["x"].dtype).double()
        rms = (h.pow(2).sum(1, keepdim=True) / d + EPS).sqrt()
        y = h / rms * s["weight"].double()
        stored = y.to(s["x"].dtype).double()
        return {"h": h, "y": y, "rstd": 1.0 / rms[:, 0], "q": _int8_round64(stored)}
    if case["kind"] == "norm_grad":
        # by the Jacobian: d n_i / d h_j = r ([i = j] - r^2 h_i h_j / d), n = r h
        h, up, w = s["h"].double(), s["dy"].double(), s["weight"].double()
        r = s["rstd"].double()
        through = up * w
        inner = torch.bmm(through[:, None, :].contiguous(), h[:, :, None].contiguous()).view(T)
        dh = through * r[:, None] - h * (r ** 3 * inner / d)[:, None] + s["dh_add"].double()
        return {"dh": dh, "dw": r @ (up * h)}
    if case["kind"] == "balance":
        live = [True] * T if s["mask"] is None else s["mask"].tolist()
        rows = torch.tensor([t for t in range(T) if live[t]], dtype=torch.long, device="cuda")
        p = torch.softmax(s["logits"][rows].double(), 1)
        counts = torch.bincount(s["idx"][rows].flatten().long(), minlength=E)
        n = max(len(rows), 1)
        share = counts.double() / (k * n)
        mean = p.sum(0) / n
        up = E * share / n                               # of the loss by every p[t][e]
        dlogits = torch.zeros((T, E), dtype=torch.float64, device="cuda")
        dlogits[rows] = p * up - p * (p @ up)[:, None]
        return {"loss": (E * (share * mean).sum()).view(1), "counts": None, "prob_sum": p.sum(0),
                "dlogits": dlogits}
    y = torch.zeros((s["cap"], d), dtype=torch.float64, device="cuda")
    at = 0
    for size, (q13, s13), (q2, s2) in zip(s["sizes"], s["w13"], s["w2"]):
        token = s["row_token"][at:at + size].long()
        x = s["xq"][token, :d].double() * s["x_scale"][token, None].double()
        if size:
            ab = x @ (q13[:, :d].double() * s13[:, None].double()).t()
            h = ab[:, :f] * torch.sigmoid(ab[:, :f]) * ab[:, f:]
            h = _int8_round64(h.to(torch.bfloat16).double())
            y[at:at + size] = h @ (q2[:, :f].double() * s2[:, None].double()).t()
        at += size
    return y
