"""The training and decoding steps that use the 8-bit products, the residual norm and the log probabilities together,
against the same model in 64 bits without any rounding.

An E4M3 code is off by at most 2^-4 of its value; over random values that is a relative error of
2^-4 / sqrt(3) * 0.7 = 0.026 in the norm, 0.037 for a product of two quantized operands.  The longest path of
a gradient here goes through five such products (two forward, three backward: 0.083, independent errors
adding in quadrature), and a gradient is itself a product of two quantized matrices; twice the sum of the two
is 0.24, the bound on the relative error in the norm.  The logits are two products deep (0.052 of their norm,
which is about sqrt(vocab) per row here, so 0.052 per logit): a log probability stays within 6 * 0.052 * 2 of its
value (six standard deviations, of the logit and of the normaliser), a mean over n of them within 0.62 / sqrt(n)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2605_09825_b200 import api, block_step


def rms_norm(x, w):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * w


def logits_of(w, ids):
    s0 = w["embedding"][ids]
    h0 = rms_norm(s0, w["w_in"])
    u, g = h0 @ w["w_up"].t(), h0 @ w["w_gate"].t()
    s1 = s0 + torch.sigmoid(g) * rms_norm(u, w["w_post"])
    return rms_norm(s1, w["w_out"]) @ w["w_head"].t()


@pytest.mark.parametrize("tokens,hidden,vocab,entropy_weight", [(48, 128, 528, 0.0), (272, 416, 1200, 0.3)])
def test_train_step(tokens, hidden, vocab, entropy_weight):
    w = block_step.make_weights(hidden, vocab)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    ids, targets = (torch.randint(0, vocab, (tokens,), device="cuda", generator=gen) for _ in range(2))
    targets[5:9] = -1
    loss, grads = block_step.train_step(w, ids, targets, entropy_weight)
    api.check()
    w64 = {k: v.double().requires_grad_() for k, v in w.items()}
    logp = torch.log_softmax(logits_of(w64, ids), -1)
    entropy = -(logp.exp() * logp).sum(-1)
    keep = targets >= 0
    ref = -logp.gather(1, targets.clamp(min=0)[:, None])[keep].mean() - entropy_weight * entropy[keep].mean()
    ref.backward()
    assert abs(loss.item() - ref.item()) <= 0.62 / int(keep.sum()) ** 0.5 * (1 + entropy_weight)
    for name in block_step.WEIGHTS:
        got, want = grads[name].double(), w64[name].grad
        if name == "embedding":                             # a row per token
            got = torch.zeros_like(want).index_add_(0, ids, got)
        assert got.shape == want.shape
        assert (got - want).norm() <= 0.24 * want.norm(), f"{name}: {((got - want).norm() / want.norm()).item()}"


@pytest.mark.parametrize("batch", [1, 5, 16, 40])
def test_decoder(batch):
    w = block_step.make_weights(416, 1200)
    gen = torch.Generator(device="cuda").manual_seed(batch)
    eager, replayed = (block_step.Decoder(w, batch, 4, graph) for graph in (False, True))
    for _ in range(3):
        ids = torch.randint(0, 1200, (batch,), device="cuda", generator=gen)
        a, b = eager.step(ids), replayed.step(ids)
        api.check()
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        ref = torch.log_softmax(logits_of({k: v.double() for k, v in w.items()}, ids), -1)
        top_logp, top_index, entropy = a
        assert ((top_logp - ref.gather(1, top_index)).abs() <= 0.62).all()
        assert (top_logp[:, 0] >= ref.max(1).values - 0.62).all()
        assert ((entropy + (ref.exp() * ref).sum(1)).abs() <= 0.62).all()


@pytest.mark.parametrize("batch", [2, 40])
def test_decoder_with_an_odd_vocabulary(batch):
    w = block_step.make_weights(128, 1203)
    ids = torch.arange(batch, device="cuda")
    top_logp, top_index, entropy = block_step.Decoder(w, batch, 4).step(ids)
    api.check()
    ref = torch.log_softmax(logits_of({k: v.double() for k, v in w.items()}, ids), -1)
    assert ((top_logp - ref.gather(1, top_index)).abs() <= 0.62).all()
    assert (top_logp[:, 0] >= ref.max(1).values - 0.62).all()
    assert ((entropy + (ref.exp() * ref).sum(1)).abs() <= 0.62).all()
