"""A small language model's training step and decoding step on the 8-bit products with 128-element blocks, the
residual norm and the token log probabilities, used together the way a trainer and a server would.

    s0 = E[ids],                h0 = rms_norm(s0) * w_in
    u  = h0 W_up^T,  g = h0 W_gate^T,
    s1 = s0 + sigmoid(g) * rms_norm(u) * w_post,       h1 = rms_norm(s1) * w_out
    logits = h1 W_head^T,       loss = -mean(log p(target)) - entropy_weight * mean(entropy)

``train_step`` is the loss and the gradient of every weight; ``Decoder`` quantizes the weights once and
answers one token per sequence and call, replayed as a CUDA graph (a step is a dozen launches of a few
microseconds, more to launch than to run).  PyTorch looks up embeddings, allocates and adds two gradients.

    python -m paper_2605_09825_b200.block_step --tokens 8192 --hidden 4096 --vocab 128256
"""
from __future__ import annotations

import argparse

import torch

from . import api

WEIGHTS = ("embedding", "w_in", "w_up", "w_gate", "w_post", "w_out", "w_head")
MATRICES = ("w_up", "w_gate", "w_head")


def make_weights(hidden: int, vocab: int, seed: int = 0, device="cuda") -> dict:
    """Random weights: bf16 matrices, fp32 norm weights around one."""
    gen = torch.Generator(device=device).manual_seed(seed)
    matrix = lambda r, c, s: (torch.randn(r, c, device=device, generator=gen) * s).bfloat16()
    vector = lambda: 1 + 0.1 * torch.randn(hidden, device=device, generator=gen)
    return {"embedding": matrix(vocab, hidden, 1.0), "w_in": vector(),
            "w_up": matrix(hidden, hidden, hidden ** -0.5), "w_gate": matrix(hidden, hidden, hidden ** -0.5),
            "w_post": vector(), "w_out": vector(), "w_head": matrix(vocab, hidden, hidden ** -0.5)}


def train_step(w: dict, ids: torch.Tensor, targets: torch.Tensor, entropy_weight: float = 0.0):
    """``(loss, gradients)`` for int64 ``ids`` and ``targets`` [tokens] (negative targets count for nothing);
    tokens a multiple of 16, hidden and vocab of 16.  Matrix gradients are fp32 [out, in], the
    embedding's a bf16 [tokens, hidden] row per token, as a sparse update takes it."""
    linear = lambda x, m: api.linear_pass_block128(api.PASS_FPROP, x, m)
    grad_x = lambda dy, m: api.linear_pass_block128(api.PASS_DGRAD, dy, m)
    grad_w = lambda dy, x: api.linear_pass_block128(api.PASS_WGRAD, dy, x, api.OUT_FP32)
    act = api.GATE_SIGMOID
    # forward
    s0, h0 = api.residual_norm_forward(w["embedding"].index_select(0, ids), w_pre=w["w_in"])
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


class Decoder:
    """Decoding of ``batch`` sequences, one token each per call, from weights quantized once."""

    def __init__(self, w: dict, batch: int, top_k: int = 5, graph: bool = True):
        self.w, self.top_k = w, top_k
        self.matrices = {name: api.quantize_block128(w[name], api.AXIS_COLS, api.BLOCK_128X128) for name in MATRICES}
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
        s0, h0 = api.residual_norm_forward(w["embedding"].index_select(0, self.ids), w_pre=w["w_in"])
        linear = lambda x, name: api.gemm_block128(*x, *self.matrices[name])
        x = api.quantize_block128(h0)                       # once for both products
        u, g = linear(x, "w_up"), linear(x, "w_gate")
        _, h1 = api.residual_norm_forward(u, s0, w["w_post"], w["w_out"], g, api.GATE_SIGMOID, y=s0)
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
    a = ap.parse_args()
    w = make_weights(a.hidden, a.vocab)
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids, targets = (torch.randint(0, a.vocab, (a.tokens,), device="cuda", generator=gen) for _ in range(2))
    for step in range(a.steps):
        loss, grads = train_step(w, ids, targets)
        api.check()
        print(f"step {step}: loss {loss.item():.4f}")
        for name in MATRICES:
            w[name].add_(grads[name], alpha=-a.lr)
    print(f"training step, {a.tokens} tokens: {_milliseconds(lambda: train_step(w, ids, targets), 5):.3f} ms")
    for graph in (False, True):
        decoder = Decoder(w, a.batch, graph=graph)
        ms = _milliseconds(lambda: decoder.step(ids[:a.batch]), 50)
        api.check()
        print(f"decoding step, {a.batch} sequence(s), {'CUDA graph' if graph else 'eager'}: {1e3 * ms:.1f} us")


if __name__ == "__main__":
    main()
