"""A loss that is a mean has the same gradient at every position.  Rounded to bf16 it would be off by the same factor
everywhere (1/255 by 2^-8), and so would all of dx and dw: the factor that the positions have in common is applied to
the sums in fp32 instead.

Bounds.  What is rounded is then delta - p.  At a target it is 1 - p, off by 2^-9 at most, and where p is small always to the
same side: so much of the exact gradient's direction may be missing or too much; the other roundings are
independent and add 2^-12 at most to that.  The norm of the whole error stays below 2^-8 (2^-9 of this kind, 2^-8 / sqrt(3) of
a result's rounding).
"""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu


def exact(x, w, targets, lse, gl, gn, scale):
    X, W = x.double(), w.double()
    z = scale * (X @ W.t())
    has = (targets >= 0).nonzero()[:, 0]
    l = torch.where(targets >= 0, gl.double(), 0.0)
    n = gn.double() if gn is not None else torch.zeros_like(l)
    dz = (n - l)[:, None] * torch.exp(z - lse.double()[:, None])
    dz[has, targets[has]] += l[has]
    return scale * dz @ W, scale * dz.t() @ X


@pytest.mark.parametrize("T,D,V", [(255, 256, 1000), (257, 136, 4097), (16383, 64, 8192 + 40), (31, 264, 20000)])
@pytest.mark.parametrize("dw", [api.OUT_BF16, api.OUT_FP32])
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_mean_over_the_positions(T, D, V, dw, scale):
    gen = torch.Generator(device="cuda").manual_seed(T)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, w = rand(T, D).bfloat16(), (rand(V, D) * D ** -0.5).bfloat16()
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
    targets[::9] = -1
    count = float((targets >= 0).sum())
    # of all numbers of positions, the one whose share is off most
    share = torch.where(targets >= 0, -1 / 255 * 2.0 ** -round(torch.tensor(count).log2().item() - 8), float("nan"))
    _, lse = api.linear_logprobs_forward(x, w, None, scale)
    for gl, gn in ((share, None), (share, 1e-3 * share.nan_to_num(0))):
        got = api.linear_logprobs_backward(x, w, targets, lse, gl, gn, scale, dw)
        api.check()
        for g, ref in zip(got, exact(x, w, targets, lse, gl, gn, scale)):
            ratio = (g.double() * ref).sum() / ref.square().sum()
            assert abs(ratio - 1) <= 2.0 ** -9 + 2.0 ** -12, ratio
            assert (g.double() - ref).norm() <= 2.0 ** -8 * ref.norm()


def test_gradients_of_very_different_size():
    """Neither a gradient of the normaliser far above the target's, nor positions far below the largest, are lost."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, w = rand(64, 64).bfloat16(), (rand(500, 64) * 0.1).bfloat16()
    targets = torch.randint(0, 500, (64,), generator=gen, device="cuda")
    _, lse = api.linear_logprobs_forward(x, w)
    for small, large in ((1e-37, None), (1e-37, 10.0), (1e-3, 1e30), (1e30, 1e-3), (0.0, 1e-3)):
        gl = torch.full((64,), small, device="cuda")
        gl[::2] *= 1e-3
        gn = None if large is None else torch.full((64,), large, device="cuda")
        dx, dw = api.linear_logprobs_backward(x, w, targets, lse, gl, gn, dw_dtype=api.OUT_FP32)
        api.check()
        want = exact(x, w, targets, lse, gl, gn, 1.0)
        for g, ref in zip((dx, dw), want):
            assert ((g.double() - ref).norm(dim=1) <= 2.0 ** -7 * ref.norm(dim=1) + 1e-37).all()
