"""Targets past the vocabulary in the backward pass of the loss from the output layer's input: NaN where a gradient goes
through them, not looked at otherwise."""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu


def inputs(T, D, V, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return rand(T, D).bfloat16(), (2 * rand(V, D) * D ** -0.5).bfloat16(), torch.randint(0, V, (T,), generator=gen, device="cuda"), gen


@pytest.mark.parametrize("T,V", [(40, 300), (300, 2011)])
def test_targets_past_the_vocabulary_without_their_gradient(T, V):
    """d_logp NULL is zero: the targets count for nothing, wherever they point."""
    x, w, targets, gen = inputs(T, 72, V)
    targets[:4] = torch.tensor([V, V + 7, 1 << 40, -1], device="cuda")
    _, lse = api.linear_logprobs_forward(x, w)
    gn = torch.randn(T, generator=gen, device="cuda")
    got, want = (api.linear_logprobs_backward(x, w, t, lse, None, gn) for t in (targets, None))
    api.check()
    assert all(g.isfinite().all() for g in got)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("at_zero", [False, True])
def test_targets_past_the_vocabulary_with_their_gradient(at_zero):
    """Such a position's gradient is NaN, also where d_logp is 0 there; dw, a sum over the positions, is NaN with it."""
    x, w, targets, gen = inputs(40, 72, 300)
    targets[5] = 300
    _, lse = api.linear_logprobs_forward(x, w)
    gl = torch.randn(40, generator=gen, device="cuda")
    if at_zero:
        gl[5] = 0
    dx, dw = api.linear_logprobs_backward(x, w, targets, lse, gl)
    api.check()
    assert dx[5].isnan().all() and int(dx.isnan().any(1).sum()) == 1
    assert dw.isnan().all()
