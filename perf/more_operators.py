"""Cases and plain forms of the operators at the two ends of a training step, from token ids to clipped gradients.

Four operators:

  gated       the first half of a gated feed-forward block kept in 16 bits: both projections, the
              activation and their product, and its backward pass
  loss        log probabilities of given tokens straight from the output layer's input and weight
              (softmax cross entropy over the vocabulary in pieces, no logits kept), and the gradients
              with respect to both
  embedding   scaled lookup of token embeddings, and the table's gradient
  clip        the global norm of many gradient tensors, and clipping by it

``run`` with ``own`` false computes them with elementary torch operations in 32 bits; with ``own``
true it makes the calls of the package's public entry points.  ``exact`` computes the same outputs
from the definitions in 64 bits.
"""
import math

import torch

own = False

HIDDEN, INTER, VOCAB = 4096, 14336, 128256       # one Llama-3.1-8B layer and its vocabulary
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of a decoding step
        {"name": "gated_fwd_1tok", "op": "gated", "form": "fwd", "tokens": 1, "in_f": HIDDEN, "inter": INTER,
         "act": "silu", "keep": False},
        # a ragged batch of prompts
        {"name": "gated_fwd_333tok", "op": "gated", "form": "fwd", "tokens": 333, "in_f": HIDDEN, "inter": INTER,
         "act": "silu", "keep": False},
        # forward of a training step, which keeps both projections for the backward pass
        {"name": "gated_fwd_8192tok", "op": "gated", "form": "fwd", "tokens": 8192, "in_f": HIDDEN, "inter": INTER,
         "act": "silu", "keep": True},
        # backward of a smaller batch: the gradients of the input and of both weights
        {"name": "gated_bwd_4096tok", "op": "gated", "form": "bwd", "tokens": 4096, "in_f": HIDDEN, "inter": INTER,
         "act": "silu", "keep": True},
        # scoring a short text with a small model of an odd vocabulary
        {"name": "loss_fwd_333tok_odd", "op": "loss", "form": "fwd", "tokens": 333, "in_f": 2048, "vocab": 32001},
        # validation loss of a batch of sequences
        {"name": "loss_fwd_8192tok", "op": "loss", "form": "fwd", "tokens": 8192, "in_f": HIDDEN, "vocab": VOCAB},
        # the loss's gradients of a training step, with a term on the normaliser
        {"name": "loss_bwd_4096tok", "op": "loss", "form": "bwd", "tokens": 4096, "in_f": HIDDEN, "vocab": VOCAB},
        # lookup of a training step's tokens
        {"name": "embed_fwd_16384tok", "op": "embedding", "form": "fwd", "tokens": 16384, "width": HIDDEN, "vocab": VOCAB,
         "type": "bf16", "grad": "bf16"},
        # the gradient of the whole table for a short odd batch
        {"name": "embed_bwd_777tok_odd", "op": "embedding", "form": "bwd", "tokens": 777, "width": 2048, "vocab": 32001,
         "type": "bf16", "grad": "bf16"},
        # the same of a training step, in fp32 for the optimiser; a few tokens are most of the text
        {"name": "embed_bwd_16384tok", "op": "embedding", "form": "bwd", "tokens": 16384, "width": HIDDEN, "vocab": VOCAB,
         "type": "bf16", "grad": "fp32"},
        # many small tensors of odd sizes
        {"name": "clip_288_small", "op": "clip", "layers": 48, "hidden": 129, "inter": 345, "type": "bf16", "out": "bf16",
         "max_norm": 1.0},
        # the gradients of one large layer
        {"name": "clip_layer", "op": "clip", "layers": 1, "hidden": HIDDEN, "inter": INTER, "type": "bf16", "out": "bf16",
         "max_norm": 1.0},
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gated", "loss", "embedding", "clip"])
    form = rng.choice(["fwd", "bwd"])
    if op == "gated":
        in_f, inter = rng.choice([(HIDDEN, INTER), (8 * rng.randint(16, 512), 8 * rng.randint(16, 1792))])
        return {"op": op, "form": form, "tokens": _between(rng, 1, 8192), "in_f": in_f, "inter": inter,
                "act": rng.choice(["linear", "sigmoid", "silu", "gelu", "gelu_tanh", "relu"]), "keep": form == "bwd" or rng.random() < 0.5}
    if op == "loss":
        return {"op": op, "form": form, "tokens": _between(rng, 16, 4096),
                "in_f": rng.choice([HIDDEN, 2048, 8 * rng.randint(16, 512)]),
                "vocab": rng.choice([VOCAB, 32001, _between(rng, 1000, 100000)])}
    if op == "embedding":
        return {"op": op, "form": form, "tokens": _between(rng, 1, 16384), "width": rng.choice([HIDDEN, 2048, 8 * rng.randint(4, 512)]),
                "vocab": rng.choice([VOCAB, 32001, _between(rng, 1000, 100000)]), "type": rng.choice(["bf16", "fp32"]),
                "grad": rng.choice(["bf16", "fp32"])}
    hidden = _between(rng, 32, HIDDEN)
    return {"op": op, "layers": _between(rng, 1, max(1, min(60, (HIDDEN // hidden) ** 2))), "hidden": hidden,
            "inter": int(hidden * rng.uniform(2.0, 3.5)), "type": rng.choice(["bf16", "fp32"]),
            "out": rng.choice(["bf16", "fp32"]), "max_norm": rng.choice([1.0, 0.3, 1e6])}


# ------------------------------------------------------------------------------------- inputs
def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device="cuda") * std


def _activations(gen, rows, cols):
    """N(0,1) with eight outlier channels x 20."""
    x = _normal(gen, rows, cols)
    x[:, torch.randint(0, cols, (8,), generator=gen, device="cuda")] *= 20.0
    return x.bfloat16()


def _gradients(gen, *shape, scale=1e-3):
    """Heavy tails: a normal over the root of an independent mean square of three."""
    d = _normal(gen, 3, *shape).square_().mean(0)
    return _normal(gen, *shape) * torch.rsqrt(d + 1e-6) * scale


def _ids(gen, n, vocab):
    """Token ids as text has them (the r-th most frequent about 1 / r as often as the first), frequent ones
    anywhere in the vocabulary, one position in fifty without a token."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab)) - 1.0).long().clamp(max=vocab - 1)
    ids = torch.randperm(vocab, generator=gen, device="cuda")[rank]
    if n > 8:
        ids[torch.rand(n, generator=gen, device="cuda") < 0.02] = -1
    return ids


def _clip_shapes(case):
    h, i = case["hidden"], case["inter"]
    return [(h + h // 2, h), (h, h), (2 * i, h), (h, i), (h,), (h,)] * case["layers"]


def _flat_places(case):
    """Where each tensor starts in the flat buffer of its kind (matrices, vectors), and the buffers' sizes."""
    place, sizes = [], {1: 0, 2: 0}
    for shape in _clip_shapes(case):
        place.append(sizes[len(shape)])
        sizes[len(shape)] += -(-math.prod(shape) // 64) * 64
    return place, sizes


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    if case["op"] == "clip":
        # matrices in the gradients' type, the norms' vectors in fp32
        s["grads"] = [_gradients(gen, *shape).to(TYPES[case["type"]] if len(shape) == 2 else torch.float32)
                      for shape in _clip_shapes(case)]
        # the clipped gradients go into the optimiser's two flat buffers, each tensor at a multiple of 128 bytes there
        place, sizes = _flat_places(case)
        s["flat"] = {2: torch.zeros(sizes[2], dtype=TYPES[case["out"]], device="cuda"), 1: torch.zeros(sizes[1], device="cuda")}
        s["outs"] = [s["flat"][g.dim()][at: at + g.numel()].view(g.shape) for g, at in zip(s["grads"], place)]
        return s
    T = case["tokens"]
    if case["op"] == "embedding":
        s["ids"] = _ids(gen, T, case["vocab"])
        s["scale"] = math.sqrt(case["width"])
        if case["form"] == "fwd":
            s["table"] = _normal(gen, case["vocab"], case["width"], std=0.02).to(TYPES[case["type"]])
        else:
            s["d_out"] = _gradients(gen, T, case["width"]).to(TYPES[case["type"]])
        return s
    D = case["in_f"]
    if case["op"] == "gated":
        s["x"] = _activations(gen, T, D)
        s["w_gate"], s["w_up"] = (_normal(gen, case["inter"], D, std=0.02).bfloat16() for _ in range(2))
        if case["form"] == "bwd":
            # the projections as the forward pass kept them
            x = s["x"].float()
            s["gate"], s["up"] = (x @ s["w_gate"].float().t()).bfloat16(), (x @ s["w_up"].float().t()).bfloat16()
            s["dh"] = _gradients(gen, T, case["inter"]).bfloat16()
        return s
    s["x"] = _normal(gen, T, D).bfloat16()
    s["w"] = _normal(gen, case["vocab"], D, std=0.04).bfloat16()
    s["targets"] = _ids(gen, T, case["vocab"])
    if case["form"] == "bwd":
        s["lse"] = torch.logsumexp(s["x"].float() @ s["w"].float().t(), 1)
        s["d_logp"] = torch.where(s["targets"] >= 0, -1.0 / T, 0.0)
        s["d_lse"] = 2e-4 * s["lse"] / T
    return s


# ------------------------------------------------------------------------------------- plain forms
def _act(g, act):
    """The activation of the gate and its derivative."""
    if act == "linear":
        return g, torch.ones_like(g)
    if act == "relu":
        return g.clamp(min=0.0), (g > 0).float()
    if act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * g * g)
    sg = torch.sigmoid(g)
    if act == "sigmoid":
        return sg, sg * (1.0 - sg)
    return g * sg, sg * (1.0 + g * (1.0 - sg))


def _plain_gated(s):
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    if s["form"] == "fwd":
        g, u = x @ wg.t(), x @ wu.t()
        out = {"h": (_act(g, s["act"])[0] * u).bfloat16()}
        return {**out, "gate": g.bfloat16(), "up": u.bfloat16()} if s["keep"] else out
    g, u, dh = s["gate"].float(), s["up"].float(), s["dh"].float()
    a, da = _act(g, s["act"])
    dg, du = dh * u * da, dh * a
    return {"dx": (dg @ wg + du @ wu).bfloat16(), "dw_gate": (dg.t() @ x).bfloat16(), "dw_up": (du.t() @ x).bfloat16()}


def _plain_loss(s):
    x, w, t = s["x"].float(), s["w"].float(), s["targets"]
    z = x @ w.t()
    at = t.clamp(min=0)[:, None]
    if s["form"] == "fwd":
        m = z.amax(1, keepdim=True)
        lse = (m + torch.log(torch.exp(z - m).sum(1, keepdim=True)))[:, 0]
        return {"logp": torch.where(t >= 0, z.gather(1, at)[:, 0] - lse, 0.0), "lse": lse}
    gl = torch.where(t >= 0, s["d_logp"], 0.0)
    dz = torch.exp(z - s["lse"][:, None]) * (s["d_lse"] - gl)[:, None]
    dz.scatter_add_(1, at, gl[:, None])
    return {"dx": (dz @ w).bfloat16(), "dw": (dz.t() @ x).bfloat16()}


def _plain_embedding(s):
    ids, valid = s["ids"].clamp(min=0), (s["ids"] >= 0)[:, None]
    if s["form"] == "fwd":
        rows = s["table"][ids]
        return {"out": torch.where(valid, rows.float() * s["scale"], 0.0).to(rows.dtype)}
    grad = torch.zeros(s["vocab"], s["width"], device=ids.device)
    grad.index_add_(0, ids, torch.where(valid, s["d_out"].float() * s["scale"], 0.0))
    return {"d_table": grad.to(TYPES[s["grad"]])}


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt().float()
    factor = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    for g, o in zip(s["grads"], s["outs"]):
        o.copy_(g.float() * factor)
    return {"norm": norm, "matrices": s["flat"][2], "vectors": s["flat"][1]}


# ------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _run_own(state)
    return {"gated": _plain_gated, "loss": _plain_loss, "embedding": _plain_embedding, "clip": _plain_clip}[state["op"]](state)


def _run_own(s):
    from paper_2605_09825_b200 import api
    if s["op"] == "gated":
        act = {"linear": api.GATE_LINEAR, "sigmoid": api.GATE_SIGMOID, "silu": api.GATE_SILU, "gelu": api.GATE_GELU,
               "gelu_tanh": api.GATE_GELU_TANH, "relu": api.GATE_RELU}[s["act"]]
        if s["form"] == "fwd":
            h, kept = api.gated_linear_forward(s["x"], s["w_gate"], s["w_up"], act, keep=s["keep"])
            return {"h": h, "gate": kept[0], "up": kept[1]} if s["keep"] else {"h": h}
        dx, dw_gate, dw_up = api.gated_linear_backward(s["dh"], s["x"], s["w_gate"], s["w_up"], (s["gate"], s["up"]), act)
        return {"dx": dx, "dw_gate": dw_gate, "dw_up": dw_up}
    if s["op"] == "loss":
        if s["form"] == "fwd":
            logp, lse = api.linear_logprobs_forward(s["x"], s["w"], s["targets"])
            return {"logp": logp, "lse": lse}
        dx, dw = api.linear_logprobs_backward(s["x"], s["w"], s["targets"], s["lse"], s["d_logp"], s["d_lse"])
        return {"dx": dx, "dw": dw}
    if s["op"] == "embedding":
        if s["form"] == "fwd":
            return {"out": api.embedding_forward(s["ids"], s["table"], s["scale"])}
        out = api.OUT_BF16 if s["grad"] == "bf16" else api.OUT_FP32
        return {"d_table": api.embedding_backward(s["ids"], s["d_out"], s["vocab"], s["scale"], out)}
    norm = api.clip_grads(s["grads"], s["max_norm"], out=s["outs"])
    return {"norm": norm, "matrices": s["flat"][2], "vectors": s["flat"][1]}


# ------------------------------------------------------------------------------------- work
def work(case):
    if case["op"] == "clip":
        shapes = _clip_shapes(case)
        size = {"bf16": 2, "fp32": 4}
        matrices = sum(a[0] * a[1] for a in shapes if len(a) == 2)
        vectors = sum(a[0] for a in shapes if len(a) == 1)
        return {"bytes": (size[case["type"]] + size[case["out"]]) * matrices + 8 * vectors + 4, "flops": 3 * (matrices + vectors)}
    T = case["tokens"]
    if case["op"] == "embedding":
        size, n = (2 if case["type"] == "bf16" else 4), T * case["width"]
        if case["form"] == "fwd":
            return {"bytes": 2 * size * n + 8 * T, "flops": n}
        return {"bytes": size * n + 8 * T + (2 if case["grad"] == "bf16" else 4) * case["vocab"] * case["width"], "flops": 2 * n}
    D = case["in_f"]
    if case["op"] == "gated":
        F = case["inter"]
        if case["form"] == "fwd":
            return {"bytes": 2 * (T * D + 2 * F * D + T * F * (3 if case["keep"] else 1)), "flops": 4 * T * D * F}
        return {"bytes": 2 * (3 * T * F + 2 * T * D + 4 * F * D), "flops": 8 * T * D * F}
    V = case["vocab"]
    if case["form"] == "fwd":
        return {"bytes": 2 * (T * D + V * D) + 16 * T, "flops": 2 * T * D * V}
    return {"bytes": 4 * (T * D + V * D) + 20 * T, "flops": 6 * T * D * V}


# ------------------------------------------------------------------------------------- 64 bits
def _exact_act(g, act):
    if act == "linear":
        return g, 1.0
    if act == "relu":
        return torch.where(g > 0, g, 0.0), torch.where(g > 0, 1.0, 0.0).double()
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return g * cdf, cdf + g / math.sqrt(2.0 * math.pi) * torch.exp(-g * g / 2.0)
    if act == "gelu_tanh":
        inner = math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)
        slope = math.sqrt(2.0 / math.pi) * (1.0 + 0.134145 * g ** 2)
        share = 1.0 / (1.0 + torch.exp(-2.0 * inner))          # (1 + tanh) / 2
        return g * share, share + 2.0 * g * share * (1.0 - share) * slope
    share = 1.0 / (1.0 + torch.exp(-g))
    slope = share * (1.0 - share)
    return (share, slope) if act == "sigmoid" else (g * share, share + g * slope)


def _exact_gated(s):
    x, wg, wu = s["x"].double(), s["w_gate"].double(), s["w_up"].double()
    if s["form"] == "fwd":
        g, u = torch.matmul(x, wg.T), torch.matmul(x, wu.T)
        out = {"h": _exact_act(g, s["act"])[0] * u}
        if s["keep"]:
            out["gate"], out["up"] = g, u
        return out
    value, slope = _exact_act(s["gate"].double(), s["act"])
    du = s["dh"].double() * value
    dg = s["dh"].double() * s["up"].double() * slope
    return {"dx": torch.addmm(torch.matmul(dg, wg), du, wu), "dw_gate": torch.matmul(dg.T, x), "dw_up": torch.matmul(du.T, x)}


def _exact_loss(s):
    x, w, t = s["x"].double(), s["w"].double(), s["targets"]
    step = max(1, (1 << 28) // s["vocab"])
    logp, lse, dx, dw = [], [], [], torch.zeros_like(w) if s["form"] == "bwd" else None
    for r in range(0, s["tokens"], step):
        rows = slice(r, min(r + step, s["tokens"]))
        z, has = torch.matmul(x[rows], w.T), torch.nonzero(t[rows] >= 0)[:, 0]
        if s["form"] == "fwd":
            total = torch.logsumexp(z, 1)
            picked = torch.zeros_like(total)
            picked[has] = z[has, t[rows][has]] - total[has]
            logp.append(picked)
            lse.append(total)
        else:
            p = torch.exp(z - s["lse"][rows].double()[:, None])
            d = s["d_lse"][rows].double()[:, None] * p
            d[has] -= s["d_logp"][rows].double()[has][:, None] * p[has]
            d[has, t[rows][has]] += s["d_logp"][rows].double()[has]
            dx.append(torch.matmul(d, w))
            dw += torch.matmul(d.T, x[rows])
    return {"logp": torch.cat(logp), "lse": torch.cat(lse)} if s["form"] == "fwd" else {"dx": torch.cat(dx), "dw": dw}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "gated":
        return _exact_gated(s)
    if case["op"] == "loss":
        return _exact_loss(s)
    if case["op"] == "clip":
        total = sum(float((g.double() ** 2).sum()) for g in s["grads"])
        factor = min(1.0, case["max_norm"] / (math.sqrt(total) + 1e-6))
        place, sizes = _flat_places(case)
        flat = {kind: torch.zeros(n, dtype=torch.float64, device="cuda") for kind, n in sizes.items()}
        for g, at in zip(s["grads"], place):
            flat[g.dim()][at: at + g.numel()] = g.double().flatten() * factor
        return {"norm": torch.tensor(math.sqrt(total), dtype=torch.float64), "matrices": flat[2], "vectors": flat[1]}
    has = torch.nonzero(s["ids"] >= 0)[:, 0]
    if case["form"] == "fwd":
        out = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device="cuda")
        out[has] = s["scale"] * s["table"].double()[s["ids"][has]]
        return {"out": out}
    grad = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
    grad.index_put_((s["ids"][has],), s["scale"] * s["d_out"].double()[has], accumulate=True)
    return {"d_table": grad}
