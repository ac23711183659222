"""A small language model's training step and decoding step on the 8-bit products with 128-element blocks, the
residual norm and the token log probabilities, used together the way a trainer and a server would.

    s0 = E[ids],                h0 = rms_norm(s0) * w_in
    u  = h0 W_up^T,  g = h0 W_gate^T,
    s1 = s0 + sigmoid(g) * rms_norm(u) * w_post,       h1 = rms_norm(s1) * w_out
    logits = h1 W_head^T,       loss = -mean(log p(target)) - entropy_weight * mean(entropy)

With ``inner`` a gated feed-forward block follows, whose projections stay in 16 bits, and the logits are never stored:

    h1 = rms_norm(s1) * w_mid,      f  = silu(h1 W_ffn_gate^T) * (h1 W_ffn_up^T)
    d  = f W_down^T,                s2 = s1 + rms_norm(d) * w_ffn_post,     h2 = rms_norm(s2) * w_out
    loss = -mean(log p(target)) + lse_weight * mean(lse^2)     of z = h2 W_head^T

``train_step`` (``train_step_gated`` with ``inner``) is the loss and the gradient of every weight, from the token ids to
clipped gradients in the latter; ``Decoder`` quantizes the weights once and answers one token per sequence and
call, replayed as a CUDA graph (a step is a dozen launches of a few microseconds, more to launch than to run).
PyTorch allocates, adds two gradients and sums up the loss.

    python -m paper_2605_09825_b200.block_step --tokens 8192 --hidden 4096 --vocab 128256 [--inner 14336]
"""
from __future__ import annotations

import argparse

import torch

from . import api

WEIGHTS = ("embedding", "w_in", "w_up", "w_gate", "w_post", "w_out", "w_head")
MATRICES = ("w_up", "w_gate", "w_head")
GATED = ("w_mid", "w_ffn_gate", "w_ffn_up", "w_down", "w_ffn_post")


def make_weights(hidden: int, vocab: int, seed: int = 0, device="cuda", inner: int = 0) -> dict:
    """Random weights: bf16 matrices, fp32 norm weights around one; with ``inner`` those of the feed-forward block too."""
    gen = torch.Generator(device=device).manual_seed(seed)
    matrix = lambda r, c, s: (torch.randn(r, c, device=device, generator=gen) * s).bfloat16()
    vector = lambda: 1 + 0.1 * torch.randn(hidden, device=device, generator=gen)
    w = {"embedding": matrix(vocab, hidden, 1.0), "w_in": vector(),
         "w_up": matrix(hidden, hidden, hidden ** -0.5), "w_gate": matrix(hidden, hidden, hidden ** -0.5),
         "w_post": vector(), "w_out": vector(), "w_head": matrix(vocab, hidden, hidden ** -0.5)}
    if inner:
        w |= {"w_mid": vector(), "w_ffn_gate": matrix(inner, hidden, hidden ** -0.5),
              "w_ffn_up": matrix(inner, hidden, hidden ** -0.5), "w_down": matrix(hidden, inner, inner ** -0.5),
              "w_ffn_post": vector()}
    return w


def train_step(w: dict, ids: torch.Tensor, targets: torch.Tensor, entropy_weight: float = 0.0):
    """``(loss, gradients)`` for ``ids`` and int64 ``targets`` [tokens] (negative targets count for nothing);
    tokens a multiple of 16, hidden and vocab of 16.  Matrix gradients are fp32 [out, in], the
    embedding's a bf16 [tokens, hidden] row per token, as a sparse update takes it."""
    linear = lambda x, m: api.linear_pass_block128(api.PASS_FPROP, x, m)
    grad_x = lambda dy, m: api.linear_pass_block128(api.PASS_DGRAD, dy, m)
    grad_w = lambda dy, x: api.linear_pass_block128(api.PASS_WGRAD, dy, x, api.OUT_FP32)
    act = api.GATE_SIGMOID
    ids = ids.long().contiguous()                           # of either integer type and any stride, as PyTorch's lookup
    # forward
    s0, h0 = api.residual_norm_forward(api.embedding_forward(ids, w["embedding"]), w_pre=w["w_in"])
    u, g = linear(h0, w["w_up"]), linear(h0, w["w_gate"])
    s1, h1 = api.residual_norm_forward(u, s0, w["w_post"], w["w_out"], g, act)
    logits = linear(h1, w["w_head"])
    logp, entropy, lse, _, _ = api.logprobs_forward(logits, targets)
    counted = (targets >= 0).float()
    share = counted / counted.sum().clamp(min=1)
    loss = -(logp * share).sum() - entropy_weight * (entropy * share).sum()
    # backward; the logits' memory takes their gradient
    dlogits = api.logprobs_backward(logits, targets, lse, entropy, -share,
                                    -entropy_weight * share if entropy_weight else None, dlogits=logits)
    grads = {"w_head": grad_w(dlogits, h1)}
    ds0, du, dg, grads["w_post"], grads["w_out"] = api.residual_norm_backward(
        grad_x(dlogits, w["w_head"]), None, u, s1, w["w_post"], w["w_out"], g, act)
    grads["w_up"], grads["w_gate"] = grad_w(du, h0), grad_w(dg, h0)
    dh0 = grad_x(du, w["w_up"]).add_(grad_x(dg, w["w_gate"]))
    _, grads["embedding"], _, _, grads["w_in"] = api.residual_norm_backward(dh0, ds0, s0, s0, w_pre=w["w_in"])
    return loss, grads


def train_step_gated(w: dict, ids: torch.Tensor, targets: torch.Tensor, lse_weight: float = 0.0, max_norm: float = float("inf")):
    """``(loss, gradients, norm)`` of a model with a feed-forward block, for ``ids`` and int64 ``targets`` [tokens] (negative
    ids: no token there; negative targets count for nothing); tokens a multiple of 16, the other sizes of 16.  The
    gradients of the table and of the 16-bit linears are bf16, the others fp32; all are scaled so that their norm, which
    is returned as it was, is at most ``max_norm``."""
    linear = lambda x, m: api.linear_pass_block128(api.PASS_FPROP, x, m)
    grad_x = lambda dy, m: api.linear_pass_block128(api.PASS_DGRAD, dy, m)
    grad_w = lambda dy, x: api.linear_pass_block128(api.PASS_WGRAD, dy, x, api.OUT_FP32)
    act = api.GATE_SIGMOID
    ids = ids.long().contiguous()                           # of either integer type and any stride, as PyTorch's lookup
    # forward
    s0, h0 = api.residual_norm_forward(api.embedding_forward(ids, w["embedding"]), w_pre=w["w_in"])
    u, g = linear(h0, w["w_up"]), linear(h0, w["w_gate"])
    s1, h1 = api.residual_norm_forward(u, s0, w["w_post"], w["w_mid"], g, act)
    f, kept = api.gated_linear_forward(h1, w["w_ffn_gate"], w["w_ffn_up"])
    d = linear(f, w["w_down"])
    s2, h2 = api.residual_norm_forward(d, s1, w["w_ffn_post"], w["w_out"])
    logp, lse = api.linear_logprobs_forward(h2, w["w_head"], targets)
    counted = (targets >= 0).float()
    share = counted / counted.sum().clamp(min=1)
    loss = (share * (lse_weight * lse.square() - logp)).sum()
    # backward
    dh2, d_head = api.linear_logprobs_backward(h2, w["w_head"], targets, lse, -share, 2 * lse_weight * share * lse)
    grads = {"w_head": d_head}
    ds1, dd, _, grads["w_ffn_post"], grads["w_out"] = api.residual_norm_backward(dh2, None, d, s2, w["w_ffn_post"], w["w_out"])
    grads["w_down"] = grad_w(dd, f)
    dh1, grads["w_ffn_gate"], grads["w_ffn_up"] = api.gated_linear_backward(grad_x(dd, w["w_down"]), h1, w["w_ffn_gate"],
                                                                            w["w_ffn_up"], kept)
    ds0, du, dg, grads["w_post"], grads["w_mid"] = api.residual_norm_backward(dh1, ds1, u, s1, w["w_post"], w["w_mid"], g, act)
    grads["w_up"], grads["w_gate"] = grad_w(du, h0), grad_w(dg, h0)
    dh0 = grad_x(du, w["w_up"]).add_(grad_x(dg, w["w_gate"]))
    _, d_rows, _, _, grads["w_in"] = api.residual_norm_backward(dh0, ds0, s0, s0, w_pre=w["w_in"])
    grads["embedding"] = api.embedding_backward(ids, d_rows, w["embedding"].shape[0], out_dtype=api.OUT_BF16)
    return loss, grads, api.clip_grads(grads.values(), max_norm)


class Decoder:
    """Decoding of ``batch`` sequences, one token each per call, from weights quantized once."""

    def __init__(self, w: dict, batch: int, top_k: int = 5, graph: bool = True):
        self.w, self.top_k = w, top_k
        self.matrices = {name: api.quantize_block128(w[name], api.AXIS_COLS, api.BLOCK_128X128)
                         for name in (*MATRICES, "w_down") if name in w}
        self.ids = torch.zeros(batch, dtype=torch.int64, device=w["embedding"].device)
        self.graph = None
        if graph:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):                   # first calls set the kernels up outside the capture
                self._run()
            torch.cuda.current_stream().wait_stream(side)
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.out = self._run()

    def _run(self):
        w = self.w
        s0, h0 = api.residual_norm_forward(api.embedding_forward(self.ids, w["embedding"]), w_pre=w["w_in"])
        linear = lambda x, name: api.gemm_block128(*x, *self.matrices[name])
        x = api.quantize_block128(h0)                       # once for both products
        u, g = linear(x, "w_up"), linear(x, "w_gate")
        gated = "w_down" in w
        s1, h1 = api.residual_norm_forward(u, s0, w["w_post"], w["w_mid" if gated else "w_out"], g, api.GATE_SIGMOID, y=s0)
        if gated:
            f, _ = api.gated_linear_forward(h1, w["w_ffn_gate"], w["w_ffn_up"], keep=False)
            _, h1 = api.residual_norm_forward(linear(api.quantize_block128(f), "w_down"), s1, w["w_ffn_post"], w["w_out"], y=s1)
        _, entropy, _, top_logp, top_index = api.logprobs_forward(linear(api.quantize_block128(h1), "w_head"), None, self.top_k)
        return top_logp, top_index, entropy

    def step(self, ids: torch.Tensor):
        """``(log probabilities, token ids, entropy)`` of the ``top_k`` best next tokens, [batch, top_k] and
        [batch]; with a graph they are overwritten by the next call."""
        self.ids.copy_(ids)
        if self.graph is None:
            return self._run()
        self.graph.replay()
        return self.out


def _milliseconds(fn, n: int) -> float:
    for _ in range(3):
        fn()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(n):
        fn()
    end.record()
    end.synchronize()
    return begin.elapsed_time(end) / n


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=8192)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=128256)
    ap.add_argument("--batch", type=int, default=1, help="sequences per decoding step")
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--inner", type=int, default=0, help="width of a gated feed-forward block (0: none)")
    ap.add_argument("--max-norm", type=float, default=float("inf"), help="limit of the gradients' norm, with --inner")
    a = ap.parse_args()
    w = make_weights(a.hidden, a.vocab, inner=a.inner)
    step_of = (lambda: train_step_gated(w, ids, targets, 1e-4, a.max_norm)) if a.inner else (lambda: train_step(w, ids, targets))
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids, targets = (torch.randint(0, a.vocab, (a.tokens,), device="cuda", generator=gen) for _ in range(2))
    for step in range(a.steps):
        loss, grads, *norm = step_of()
        api.check()
        print(f"step {step}: loss {loss.item():.4f}" + (f", gradient norm {norm[0].item():.4f}" if norm else ""))
        for name in MATRICES + (("w_ffn_gate", "w_ffn_up", "w_down") if a.inner else ()):
            w[name].add_(grads[name], alpha=-a.lr)
    print(f"training step, {a.tokens} tokens: {_milliseconds(step_of, 5):.3f} ms")
    for graph in (False, True):
        decoder = Decoder(w, a.batch, graph=graph)
        ms = _milliseconds(lambda: decoder.step(ids[:a.batch]), 50)
        api.check()
        print(f"decoding step, {a.batch} sequence(s), {'CUDA graph' if graph else 'eager'}: {1e3 * ms:.1f} us")


if __name__ == "__main__":
    main()
