"""Cases and plain forms of the operators around the quantized linear layers.

Three operators, each in both directions of use:

  block128       the 8-bit product with one fp32 scale per 128 elements along the reduction axis
                 (E4M3 codes; 1 x 128 blocks for activations and gradients, 128 x 128 for weights):
                 training passes that quantize both operands, and the serving form, where the
                 weights are kept as codes and only the activations are quantized in the call
  residual_norm  the end of one residual block and the start of the next: RMS norm of the branch,
                 gate, scaled residual addition, RMS norm of the stream
  logprobs       log probabilities of given tokens with the entropy and the top alternatives of
                 each row, and the gradient with respect to the logits

``run`` with ``own`` false computes them with elementary torch operations in 32 bits; with ``own``
true it makes the calls of the package's public entry points.  ``exact`` computes the same outputs
from the definitions in 64 bits.
"""
import math

import torch

own = False

# (out, in) of the four linears of one Llama-3.1-8B layer
LINEARS = {"qkv": (6144, 4096), "o": (4096, 4096), "gate_up": (28672, 4096), "down": (4096, 14336)}
VOCAB = 128256
FP8_MAX = 448.0
TINY = 2.0 ** -100           # smallest block maximum a scale is formed from
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of a decoding step through the widest reduction of a layer
        {"name": "block128_serve_down_1tok", "op": "block128", "form": "serve", "tokens": 1, "out_f": 4096,
         "in_f": 14336, "out": "bf16"},
        # a ragged batch of prompts through the largest weight
        {"name": "block128_serve_gate_up_333tok", "op": "block128", "form": "serve", "tokens": 333, "out_f": 28672,
         "in_f": 4096, "out": "bf16"},
        # backward of an attention output projection at a small batch
        {"name": "block128_dgrad_o_2048tok", "op": "block128", "form": "dgrad", "tokens": 2048, "out_f": 4096,
         "in_f": 4096, "out": "bf16"},
        # weight gradient of the largest linear, kept in fp32 for the optimiser
        {"name": "block128_wgrad_gate_up_8192tok", "op": "block128", "form": "wgrad", "tokens": 8192, "out_f": 28672,
         "in_f": 4096, "out": "fp32"},
        # one token of a decoding step: norm after the block, layer scale, norm before the next
        {"name": "norm_fwd_1tok", "op": "norm", "form": "fwd", "tokens": 1, "width": 4096, "stream": "bf16",
         "post": True, "pre": True, "gate": "channel", "act": "linear"},
        # forward of a training step, sigmoid gate computed per element
        {"name": "norm_fwd_16384tok", "op": "norm", "form": "fwd", "tokens": 16384, "width": 4096, "stream": "bf16",
         "post": True, "pre": True, "gate": "element", "act": "sigmoid"},
        # backward of the same place in a training step
        {"name": "norm_bwd_16384tok", "op": "norm", "form": "bwd", "tokens": 16384, "width": 4096, "stream": "bf16",
         "post": True, "pre": True, "gate": "element", "act": "silu"},
        # backward with an fp32 stream, an odd number of tokens and a wide row
        {"name": "norm_bwd_1003tok_wide", "op": "norm", "form": "bwd", "tokens": 1003, "width": 14336,
         "stream": "fp32", "post": True, "pre": True, "gate": "channel", "act": "linear"},
        # one sampled token with its alternatives, as a server returns them
        {"name": "logprobs_fwd_1tok_top20", "op": "logprobs", "form": "fwd", "tokens": 1, "vocab": VOCAB,
         "type": "bf16", "top": 20},
        # validation: a batch of sequences, some alternatives kept
        {"name": "logprobs_fwd_8192tok_top5", "op": "logprobs", "form": "fwd", "tokens": 8192, "vocab": VOCAB,
         "type": "bf16", "top": 5},
        # an odd vocabulary in fp32, no alternatives
        {"name": "logprobs_fwd_517tok_odd", "op": "logprobs", "form": "fwd", "tokens": 517, "vocab": 32001,
         "type": "fp32", "top": 0},
        # the loss's gradient of a training step, with an entropy term
        {"name": "logprobs_bwd_8192tok", "op": "logprobs", "form": "bwd", "tokens": 8192, "vocab": VOCAB,
         "type": "bf16", "top": 0},
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["block128", "norm", "logprobs"])
    if op == "block128":
        form = rng.choice(["serve", "fprop", "dgrad", "wgrad"])
        out_f, in_f = rng.choice(sorted(LINEARS.values()) + [(32 * rng.randint(4, 128), 32 * rng.randint(4, 128))])
        # the weight gradient sums over tokens, which come in multiples of 16 there
        tokens = {"serve": _between(rng, 1, 512), "wgrad": 16 * _between(rng, 8, 512)}.get(form) or _between(rng, 64, 8192)
        return {"op": op, "form": form, "tokens": tokens, "out_f": out_f, "in_f": in_f,
                "out": rng.choice(["bf16", "fp32"])}
    if op == "norm":
        width = rng.choice([2048, 4096, 8192, 14336, 8 * rng.randint(8, 1000)])
        tokens = _between(rng, 1, 16384 * 4096 // max(width, 4096))
        return {"op": op, "form": rng.choice(["fwd", "bwd"]), "tokens": tokens, "width": width,
                "stream": rng.choice(["bf16", "bf16", "fp32"]), "post": rng.random() < 0.8, "pre": rng.random() < 0.8,
                "gate": rng.choice(["none", "channel", "element"]),
                "act": rng.choice(["linear", "sigmoid", "silu"])}
    vocab = rng.choice([VOCAB, VOCAB, 32001, rng.randint(1000, 100000)])
    form = rng.choice(["fwd", "bwd"])
    return {"op": op, "form": form, "tokens": _between(rng, 1, 4096), "vocab": vocab,
            "type": rng.choice(["bf16", "bf16", "fp32"]), "top": rng.choice([0, 1, 5, 20]) if form == "fwd" else 0}


# ------------------------------------------------------------------------------------- inputs
def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device="cuda") * std


def _activations(gen, rows, cols):
    """N(0,1) with eight outlier channels x 20."""
    x = _normal(gen, rows, cols)
    x[:, torch.randint(0, cols, (8,), generator=gen, device="cuda")] *= 20.0
    return x.bfloat16()


def _gradients(gen, rows, cols, scale=1e-3):
    """Heavy tails: a normal over the root of an independent mean square of three."""
    t = _normal(gen, rows, cols)
    d = _normal(gen, rows, cols).square_()
    for _ in range(2):
        d += _normal(gen, rows, cols).square_()
    return (t * torch.rsqrt(d / 3.0 + 1e-6) * scale).bfloat16()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    T = case["tokens"]
    if case["op"] == "block128":
        out_f, in_f = case["out_f"], case["in_f"]
        form = case["form"]
        if form in ("serve", "fprop"):
            s["a"], s["b"] = _activations(gen, T, in_f), _normal(gen, out_f, in_f, std=0.02).bfloat16()
        elif form == "dgrad":
            s["a"], s["b"] = _gradients(gen, T, out_f), _normal(gen, out_f, in_f, std=0.02).bfloat16()
        else:
            s["a"], s["b"] = _gradients(gen, T, out_f), _activations(gen, T, in_f)
        if form == "serve":
            # a server keeps its weights as codes and scales: [out x in] E4M3, one fp32 scale per
            # 128 x 128 block, stored block column by block column (scale of rows o, columns of
            # block t at t * ceil(out / 128) + o / 128)
            codes, scales = _plain_quantize(s["b"], 128)
            s["b_codes"] = codes.to(torch.float8_e4m3fn).view(torch.uint8)
            s["b_scales"] = scales.t().contiguous()
            del s["b"]
        return s
    if case["op"] == "norm":
        d, stream = case["width"], TYPES[case["stream"]]
        s["branch"] = _activations(gen, T, d)
        x = _normal(gen, T, d, std=3.0).to(stream)
        s["w_post"] = 1.0 + _normal(gen, d, std=0.1) if case["post"] else None
        s["w_pre"] = 1.0 + _normal(gen, d, std=0.1) if case["pre"] else None
        s["gate_t"] = None
        if case["gate"] == "channel":
            s["gate_t"] = 0.5 + _normal(gen, d, std=0.1)
        elif case["gate"] == "element":
            s["gate_t"] = _normal(gen, T, d).bfloat16()
        s["skip_scale"], s["branch_scale"] = 1.0, 0.7071
        if case["form"] == "fwd":
            s["x"] = x
        else:
            s["y"] = x                       # the stream after the addition, as the forward stored it
            s["dh"] = _gradients(gen, T, d) if case["pre"] else None
            s["dy"] = _gradients(gen, T, d).to(stream)
        return s
    V = case["vocab"]
    x = _normal(gen, T, V, std=2.5)
    x[:, torch.randint(0, V, (64,), generator=gen, device="cuda")] += 8.0
    if V > 512:
        x[:, V - 200:] = -math.inf           # entries of a padded vocabulary
    s["logits"] = x.to(TYPES[case["type"]])
    s["targets"] = torch.randint(0, max(1, V - 200 if V > 512 else V), (T,), generator=gen, device="cuda")
    if T > 8:
        s["targets"][torch.rand(T, generator=gen, device="cuda") < 0.05] = -1      # positions that carry no loss
    if case["form"] == "bwd":
        _, s["entropy"], s["lse"], _, _ = _plain_logprobs(s["logits"], s["targets"], 0)
        s["d_logp"] = -torch.rand(T, generator=gen, device="cuda") / T
        s["d_entropy"] = _normal(gen, T, std=0.01) / T
    return s


# ------------------------------------------------------------------------------------- plain forms
def _blocks(x, rows_per_block):
    """[rows, cols] as [row blocks, rows_per_block, column blocks, 128], padded with zeros."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % rows_per_block))
    return x.view(x.shape[0] // rows_per_block, rows_per_block, x.shape[1] // 128, 128)


def _plain_quantize(x, rows_per_block):
    """E4M3 codes as the fp32 values they stand for, and fp32 scales [row blocks, column blocks]."""
    r, c = x.shape
    v = _blocks(x.float(), rows_per_block)
    a = v.abs().amax(dim=(1, 3), keepdim=True).clamp(min=TINY)
    top = torch.full_like(a, FP8_MAX)        # two tensors: torch turns a quotient with a number into a product
    q = (v * (top / a)).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).float()
    return q.reshape(q.shape[0] * q.shape[1], -1)[:r, :c], (a / top)[:, 0, :, 0]


def _plain_values(x, rows_per_block):
    """What the quantized operand stands for, in fp32."""
    q, scales = _plain_quantize(x, rows_per_block)
    return q * _spread(scales, rows_per_block, q.shape)


def _spread(scales, rows_per_block, shape):
    return scales.repeat_interleave(rows_per_block, 0).repeat_interleave(128, 1)[:shape[0], :shape[1]]


def _plain_block128(s):
    form, out = s["form"], TYPES[s["out"]]
    if form == "serve":
        w = s["b_codes"].view(torch.float8_e4m3fn).float()
        w = w * _spread(s["b_scales"].t(), 128, w.shape)
        return (_plain_values(s["a"], 1) @ w.t()).to(out)
    if form == "fprop":
        return (_plain_values(s["a"], 1) @ _plain_values(s["b"], 128).t()).to(out)
    if form == "dgrad":
        return (_plain_values(s["a"], 1) @ _plain_values(s["b"], 128)).to(out)
    return (_plain_values(s["a"].t(), 1) @ _plain_values(s["b"].t(), 1).t()).to(out)


def _act(gate, act):
    """The gate's value and its derivative."""
    if act == "linear":
        return gate, torch.ones_like(gate)
    sg = torch.sigmoid(gate)
    if act == "sigmoid":
        return sg, sg * (1.0 - sg)
    return gate * sg, sg * (1.0 + gate * (1.0 - sg))


def _rms(x):
    return torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def _plain_norm_fwd(s):
    b = s["branch"].float()
    if s["w_post"] is not None:
        b = b * _rms(b) * s["w_post"]
    if s["gate_t"] is not None:
        b = b * _act(s["gate_t"].float(), s["act"])[0]
    y = (s["skip_scale"] * s["x"].float() + s["branch_scale"] * b).to(s["x"].dtype)
    if s["w_pre"] is None:
        return {"y": y}
    yf = y.float()
    return {"y": y, "h": (yf * _rms(yf) * s["w_pre"]).bfloat16()}


def _plain_norm_bwd(s):
    out = {}
    u, y, d = s["branch"].float(), s["y"].float(), s["dy"].float()
    if s["w_pre"] is not None:
        r = _rms(y)
        yh, dh = y * r, s["dh"].float()
        out["dw_pre"] = (dh * yh).sum(0)
        g = dh * s["w_pre"]
        d = d + r * (g - yh * (g * yh).mean(-1, keepdim=True))
    out["dx"] = (s["skip_scale"] * d).to(s["y"].dtype)
    d = s["branch_scale"] * d
    n, b = u, u
    if s["w_post"] is not None:
        r = _rms(u)
        n = u * r
        b = n * s["w_post"]
    if s["gate_t"] is not None:
        v, dv = _act(s["gate_t"].float(), s["act"])
        dg = d * b * dv
        out["dgate"] = dg.sum(0) if s["gate"] == "channel" else dg.bfloat16()
        d = d * v
    if s["w_post"] is not None:
        out["dw_post"] = (d * n).sum(0)
        g = d * s["w_post"]
        d = r * (g - n * (g * n).mean(-1, keepdim=True))
    out["dbranch"] = d.bfloat16()
    return out


def _plain_logprobs(x, targets, top):
    z = x.float()
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = (m + torch.log(total))[:, 0]
    entropy = lse - (e * torch.where(e > 0, z, 0.0)).sum(1) / total[:, 0]
    valid = targets >= 0
    logp = torch.where(valid, z.gather(1, targets.clamp(min=0)[:, None])[:, 0] - lse, 0.0)
    if top == 0:
        return logp, entropy, lse, None, None
    # equal values in the order of their index: a key of the value's order and the index
    bits = z.view(torch.int32).long()
    order = torch.where(bits < 0, -1 - (bits & 0x7FFFFFFF), bits)
    key = order * (1 << 20) + ((1 << 20) - 1 - torch.arange(z.shape[1], device=z.device))
    index = (1 << 20) - 1 - (key.topk(top, 1).values & ((1 << 20) - 1))
    return logp, entropy, lse, z.gather(1, index) - lse[:, None], index


def _plain_logprobs_bwd(s):
    z = s["logits"].float()
    logp = z - s["lse"][:, None]
    p = torch.exp(logp)
    gl = torch.where(s["targets"] >= 0, s["d_logp"], 0.0)
    g = -p * (gl[:, None] + s["d_entropy"][:, None] * (torch.where(p > 0, logp, 0.0) + s["entropy"][:, None]))
    g.scatter_add_(1, s["targets"].clamp(min=0)[:, None], gl[:, None])
    return g.to(s["logits"].dtype)


# ------------------------------------------------------------------------------------- one pass
def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["op"] == "block128":
        return _plain_block128(s)
    if s["op"] == "norm":
        return _plain_norm_fwd(s) if s["form"] == "fwd" else _plain_norm_bwd(s)
    if s["form"] == "bwd":
        return {"dlogits": _plain_logprobs_bwd(s)}
    return _named(*_plain_logprobs(s["logits"], s["targets"], s["top"]))


def _named(logp, entropy, lse, top_logp, top_index):
    out = {"logp": logp, "entropy": entropy, "lse": lse}
    return out if top_index is None else {**out, "top_logp": top_logp, "top_index": top_index}


def _run_own(s):
    from paper_2605_09825_b200 import api
    if s["op"] == "block128":
        out = api.OUT_BF16 if s["out"] == "bf16" else api.OUT_FP32
        if s["form"] == "serve":
            a_codes, a_scales = api.quantize_block128(s["a"], api.AXIS_COLS, api.BLOCK_1X128)
            return api.gemm_block128(a_codes, a_scales, s["b_codes"], s["b_scales"], api.BLOCK_128X128, out)
        which = {"fprop": api.PASS_FPROP, "dgrad": api.PASS_DGRAD, "wgrad": api.PASS_WGRAD}[s["form"]]
        return api.linear_pass_block128(which, s["a"], s["b"], out)
    if s["op"] == "norm":
        act = {"linear": api.GATE_LINEAR, "sigmoid": api.GATE_SIGMOID, "silu": api.GATE_SILU}[s["act"]]
        if s["form"] == "fwd":
            y, h = api.residual_norm_forward(s["branch"], s["x"], s["w_post"], s["w_pre"], s["gate_t"], act,
                                             s["skip_scale"], s["branch_scale"], EPS)
            return {"y": y} if h is None else {"y": y, "h": h}
        dx, dbranch, dgate, dw_post, dw_pre = api.residual_norm_backward(
            s["dh"], s["dy"], s["branch"], s["y"], s["w_post"], s["w_pre"], s["gate_t"], act, s["skip_scale"],
            s["branch_scale"], EPS)
        out = {"dx": dx, "dbranch": dbranch, "dgate": dgate, "dw_post": dw_post, "dw_pre": dw_pre}
        return {k: v for k, v in out.items() if v is not None}
    if s["form"] == "bwd":
        return {"dlogits": api.logprobs_backward(s["logits"], s["targets"], s["lse"], s["entropy"], s["d_logp"],
                                                 s["d_entropy"])}
    return _named(*api.logprobs_forward(s["logits"], s["targets"], s["top"]))


# ------------------------------------------------------------------------------------- work
def work(case):
    T = case["tokens"]
    if case["op"] == "block128":
        o, i, size = case["out_f"], case["in_f"], 2 if case["out"] == "bf16" else 4
        a, b, c = {"serve": (T * i, o * i, T * o), "fprop": (T * i, o * i, T * o), "dgrad": (T * o, o * i, T * i),
                   "wgrad": (T * o, T * i, o * i)}[case["form"]]
        return {"bytes": 2 * a + (1 if case["form"] == "serve" else 2) * b + size * c, "flops": 2 * T * o * i}
    if case["op"] == "norm":
        n, st = T * case["width"], 2 if case["stream"] == "bf16" else 4
        gate = 2 if case["gate"] == "element" else 0
        if case["form"] == "fwd":
            per, ops = 2 + 2 * st + gate + (2 if case["pre"] else 0), 14
        else:
            per, ops = 4 + 3 * st + 2 * gate + (2 if case["pre"] else 0), 30
        vectors = 4 * case["width"] * (int(case["post"]) + int(case["pre"]) + int(case["gate"] == "channel"))
        return {"bytes": per * n + vectors * (1 if case["form"] == "fwd" else 2), "flops": ops * n}
    n, size = T * case["vocab"], 2 if case["type"] == "bf16" else 4
    if case["form"] == "fwd":
        return {"bytes": size * n + 8 * T + 12 * T + 12 * T * case["top"], "flops": 6 * n}
    return {"bytes": 2 * size * n + 24 * T, "flops": 8 * n}


# ------------------------------------------------------------------------------------- 64 bits
def _e4m3(v):
    """The nearest E4M3 value, ties to even, saturating, of 64-bit numbers."""
    e = torch.frexp(v.abs()).exponent.clamp(min=-5) - 4        # exponent of the last bit kept
    return torch.clamp(torch.ldexp(torch.round(torch.ldexp(v, -e)), e), -FP8_MAX, FP8_MAX)


def _exact_values(x, rows_per_block):
    """The definition forms 448 / a and its product with each element in 32 bits before rounding to
    E4M3; each is reached here by rounding the 64-bit result once."""
    r, c = x.shape
    v = _blocks(x.double(), rows_per_block)
    a = v.abs().amax(3, keepdim=True).amax(1, keepdim=True).clamp(min=TINY)
    inv, scale = (FP8_MAX / a).float().double(), (a / FP8_MAX).float().double()
    v = _e4m3((v * inv).float().double()) * scale
    return v.reshape(v.shape[0] * v.shape[1], -1)[:r, :c]


def _exact_gate(gate, act):
    sg = 1.0 / (1.0 + torch.exp(-gate))
    if act == "linear":
        return gate, torch.ones_like(gate)
    return (sg, sg * (1.0 - sg)) if act == "sigmoid" else (gate * sg, sg + gate * sg * (1.0 - sg))


def _exact_norm(s):
    u = s["branch"].double()
    d = u.shape[1]
    w_post = s["w_post"].double() if s["w_post"] is not None else None
    w_pre = s["w_pre"].double() if s["w_pre"] is not None else None
    ru = 1.0 / torch.sqrt((u * u).sum(1, keepdim=True) / d + EPS) if w_post is not None else 1.0
    b = u * ru * (w_post if w_post is not None else 1.0)
    g, dg = _exact_gate(s["gate_t"].double(), s["act"]) if s["gate_t"] is not None else (1.0, 0.0)
    if s["form"] == "fwd":
        y = s["skip_scale"] * s["x"].double() + s["branch_scale"] * g * b
        out = {"y": y}
        if w_pre is not None:
            y = y.to(s["x"].dtype).double()                    # the norm is of the stream as it is stored
            out["h"] = y / torch.sqrt((y * y).sum(1, keepdim=True) / d + EPS) * w_pre
        return out
    out, y, t = {}, s["y"].double(), s["dy"].double()
    if w_pre is not None:
        ry = 1.0 / torch.sqrt((y * y).sum(1, keepdim=True) / d + EPS)
        dh = s["dh"].double()
        out["dw_pre"] = (dh * y * ry).sum(0)
        t = t + ry * dh * w_pre - ry ** 3 * y * (dh * w_pre * y).sum(1, keepdim=True) / d
    out["dx"] = s["skip_scale"] * t
    t = s["branch_scale"] * t
    if s["gate_t"] is not None:
        q = t * b * dg
        out["dgate"] = q.sum(0) if s["gate"] == "channel" else q
    t = t * g
    if w_post is not None:
        out["dw_post"] = (t * u * ru).sum(0)
        t = ru * t * w_post - ru ** 3 * u * (t * w_post * u).sum(1, keepdim=True) / d
    out["dbranch"] = t
    return out


def _exact_logprobs_rows(s, rows):
    z, t = s["logits"][rows].double(), s["targets"][rows]
    at = t.clamp(min=0)[:, None]
    if s["form"] == "bwd":
        lse, H = s["lse"][rows].double()[:, None], s["entropy"][rows].double()[:, None]
        p = torch.exp(z - lse)
        gl = torch.where(t >= 0, s["d_logp"][rows].double(), 0.0)[:, None]
        dent = p * (torch.where(torch.isinf(z), 0.0, z) - lse + H)
        g = -gl * p - s["d_entropy"][rows].double()[:, None] * dent
        return {"dlogits": g.scatter_add_(1, at, gl).float()}
    m = z.max(1, keepdim=True).values
    lse = m + torch.log(torch.exp(z - m).sum(1, keepdim=True))
    logp = z - lse
    H = -(torch.exp(logp) * torch.where(torch.isinf(z), 0.0, logp)).sum(1)
    out = {"logp": torch.where(t >= 0, logp.gather(1, at)[:, 0], 0.0), "entropy": H, "lse": lse[:, 0]}
    if s["top"]:
        v, i = torch.sort(logp, dim=1, descending=True, stable=True)
        out["top_logp"], out["top_index"] = v[:, :s["top"]], i[:, :s["top"]]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "logprobs":
        step = max(1, (1 << 27) // case["vocab"])
        parts = [_exact_logprobs_rows(s, slice(r, min(r + step, case["tokens"])))
                 for r in range(0, case["tokens"], step)]
        return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    form = case["form"]
    if form == "serve":
        w = s["b_codes"].view(torch.float8_e4m3fn).double()
        return _exact_values(s["a"], 1) @ (w * _spread(s["b_scales"].t().double(), 128, w.shape)).t()
    if form == "wgrad":
        return _exact_values(s["a"].t(), 1) @ _exact_values(s["b"].t(), 1).t()
    b = _exact_values(s["b"], 128)
    return _exact_values(s["a"], 1) @ (b.t() if form == "fprop" else b)
