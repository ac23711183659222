"""The training and decoding step with a gated feed-forward block, from token ids to clipped gradients, against the same
model in 64 bits without any rounding.

The bounds are those of the step without the block: a product of two E4M3 operands is off by 0.037 of its norm, the
longest path of a gradient goes through five of them (two forward, three backward), which gives 0.083, a gradient is
itself such a product, and twice the sum of the two is 0.24.  The 16-bit products of the block and of the head
add less than 0.004 each.  The logits are three quantized products deep (0.064 per logit), the decoder's four: a log
probability stays within 6 * 0.074 * 2 of its value, a mean over n of them within 0.89 / sqrt(n).
"""
import subprocess
import sys
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2605_09825_b200 import api, block_step

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def rms_norm(x, w):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * w


def logits_of(w, ids):
    s0 = torch.where(ids[:, None] >= 0, w["embedding"][ids.clamp(min=0)], 0.0)
    h0 = rms_norm(s0, w["w_in"])
    u, g = h0 @ w["w_up"].t(), h0 @ w["w_gate"].t()
    s1 = s0 + torch.sigmoid(g) * rms_norm(u, w["w_post"])
    h1 = rms_norm(s1, w["w_mid"])
    a = h1 @ w["w_ffn_gate"].t()
    d = (a * torch.sigmoid(a) * (h1 @ w["w_ffn_up"].t())) @ w["w_down"].t()
    return rms_norm(s1 + rms_norm(d, w["w_ffn_post"]), w["w_out"]) @ w["w_head"].t()


@pytest.mark.parametrize("tokens,hidden,vocab,inner,lse_weight,max_norm",
                         [(48, 128, 528, 272, 0.0, float("inf")), (272, 416, 1203, 1040, 0.01, 0.05)])
def test_train_step(tokens, hidden, vocab, inner, lse_weight, max_norm):
    w = block_step.make_weights(hidden, vocab, inner=inner)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    ids, targets = (torch.randint(0, vocab, (tokens,), device="cuda", generator=gen) for _ in range(2))
    targets[5:9] = -1
    loss, grads, norm = block_step.train_step_gated(w, ids, targets, lse_weight, max_norm)
    api.check()
    w64 = {k: v.double().requires_grad_() for k, v in w.items()}
    z = logits_of(w64, ids)
    lse, keep = torch.logsumexp(z, -1), targets >= 0
    logp = z.gather(1, targets.clamp(min=0)[:, None])[:, 0] - lse
    ref = (lse_weight * lse.square() - logp)[keep].mean()
    ref.backward()
    assert abs(loss.item() - ref.item()) <= 0.89 / int(keep.sum()) ** 0.5 * (1 + lse_weight * 2 * lse.abs().max().item())
    want_norm = sum(v.grad.square().sum() for v in w64.values()).sqrt().item()
    assert abs(norm.item() - want_norm) <= 0.24 * want_norm
    factor = min(1.0, max_norm / norm.item())
    assert set(grads) == set(block_step.WEIGHTS + block_step.GATED)
    for name, got in grads.items():
        want = w64[name].grad
        assert got.shape == want.shape
        got = got.double() / factor
        assert (got - want).norm() <= 0.24 * want.norm(), f"{name}: {((got - want).norm() / want.norm()).item()}"
    total = sum(g.double().square().sum() for g in grads.values()).sqrt().item()
    assert total <= max_norm * (1 + 2.0 ** -8)


def test_positions_without_tokens():
    w = block_step.make_weights(128, 528, inner=272)
    ids = torch.arange(48, device="cuda")
    ids[10:20] = -1
    loss, grads, norm = block_step.train_step_gated(w, ids, ids + 1)
    api.check()
    assert all(g.isfinite().all() for g in (loss, norm, *grads.values()))
    assert (grads["embedding"][48:] == 0).all() and (grads["embedding"][10:20] == 0).all()
    assert (grads["embedding"][:10] != 0).any(1).all()


@pytest.mark.parametrize("batch", [1, 5, 16, 40])
def test_decoder(batch):
    w = block_step.make_weights(416, 1200, inner=528)
    gen = torch.Generator(device="cuda").manual_seed(batch)
    eager, replayed = (block_step.Decoder(w, batch, 4, graph) for graph in (False, True))
    for _ in range(3):
        ids = torch.randint(0, 1200, (batch,), device="cuda", generator=gen)
        a, b = eager.step(ids), replayed.step(ids)
        api.check()
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        ref = torch.log_softmax(logits_of({k: v.double() for k, v in w.items()}, ids), -1)
        top_logp, top_index, entropy = a
        assert ((top_logp - ref.gather(1, top_index)).abs() <= 0.89).all()
        assert (top_logp[:, 0] >= ref.max(1).values - 0.89).all()
        assert ((entropy + (ref.exp() * ref).sum(1)).abs() <= 0.89).all()


def test_command():
    for extra in ([], ["--inner", "272", "--max-norm", "0.5"]):
        res = subprocess.run([sys.executable, "-m", "paper_2605_09825_b200.block_step", "--tokens", "64", "--hidden", "128",
                              "--vocab", "528", "--steps", "1", *extra], cwd=ROOT, capture_output=True, text=True, timeout=300)
        assert res.returncode == 0, res.stderr[-2000:]
        assert ("gradient norm" in res.stdout) == bool(extra) and "CUDA graph" in res.stdout
