"""The loss from the output layer's input with its vocabulary split over devices: what each share is given, and that together they
give what the whole does."""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu


def inputs(T, D, V, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return rand(T, D).bfloat16(), (2 * rand(V, D) * D ** -0.5).bfloat16(), torch.randint(0, V, (T,), generator=gen, device="cuda"), gen


@pytest.mark.parametrize("T,D,V,cut", [(40, 64, 300, 113), (300, 136, 5001, 4097)])
def test_two_shares_of_a_vocabulary(T, D, V, cut):
    """Each share: its part of w, the targets that lie in it (counted from its first column, the others -1), the lse of the
    whole, and where the target lies elsewhere d_lse - d_logp for d_lse.  dw is the shares' own, dx their sum.

    Bounds: those of the whole vocabulary against 64 bits -- dz rounded to bf16, and the results -- once for each
    share; the shares' roundings are independent: 2^-8 of the norm, as for the whole."""
    x, w, targets, gen = inputs(T, D, V)
    targets[0], targets[1], targets[2], targets[3] = -1, cut - 1, cut, V - 1
    gl, gn = (torch.randn(T, generator=gen, device="cuda") / T for _ in range(2))
    shares = [(0, cut), (cut, V)]
    here = [(targets >= a) & (targets < b) for a, b in shares]
    local = [torch.where(h, targets - a, -1) for h, (a, b) in zip(here, shares)]
    parts = [w[a:b] for a, b in shares]
    forward = [api.linear_logprobs_forward(x, p, t) for p, t in zip(parts, local)]
    lse = torch.logaddexp(forward[0][1], forward[1][1])
    logp = sum(torch.where(h, f[0] + f[1] - lse, 0.0) for h, f in zip(here, forward))
    elsewhere = [(targets >= 0) & ~h for h in here]
    back = [api.linear_logprobs_backward(x, p, t, lse, gl, torch.where(e, gn - gl, gn), dw_dtype=api.OUT_FP32)
            for p, t, e in zip(parts, local, elsewhere)]
    api.check()
    X, W, has = x.double(), w.double(), (targets >= 0).nonzero()[:, 0]
    z = X @ W.t()
    total = torch.logsumexp(z, 1)
    want = torch.zeros_like(total)
    want[has] = z[has, targets[has]] - total[has]
    size = 1e-5 * (X.abs() @ W.abs().t()).amax(1) + 2e-5 + 2.0 ** -21 * total.abs()
    assert ((lse.double() - total).abs() <= size).all() and ((logp.double() - want).abs() <= 3 * size).all()
    p = torch.exp(z - total[:, None])
    l = torch.where(targets >= 0, gl.double(), 0.0)
    dz = (gn.double() - l)[:, None] * p
    dz[has, targets[has]] += l[has]
    dx, dw = sum(b[0].double() for b in back), torch.cat([b[1] for b in back])
    for got, ref in ((dx, dz @ W), (dw.double(), dz.t() @ X)):
        assert (got - ref).norm() <= 2.0 ** -8 * ref.norm()
