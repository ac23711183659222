"""The 16-bit product at the lengths and widths of real models: sums of more than 1024 products, which the loss adds up in
registers across the accumulators, and tiles in several bands along either axis, the last one narrower.

Bounds as in the operators' own tests: a sum is off by 1e-5 of its products' magnitudes, a rounding to bf16 by 2^-8; a
gradient's norm by 2^-8, where the errors are independent.
"""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def memory_returned():
    yield
    torch.cuda.empty_cache()


HALF, SUM = 2.0 ** -8, 1e-5


def rand(gen, *shape, std=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).bfloat16()


def within(got, ref, tol, what):
    bad = ~((got.double() - ref).abs() <= tol + 1e-30)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off"


# in_features: one chain, a chain and one step, a chain and 8 elements, two chains, two and a short one, four
@pytest.mark.parametrize("D", [1024, 1032, 1088, 2048, 2056, 4096])
@pytest.mark.parametrize("T,V", [(1, 4097), (130, 1000), (333, 32001), (600, 19001)])
def test_loss_of_long_sums(D, T, V):
    gen = torch.Generator(device="cuda").manual_seed(D + T)
    x, w = rand(gen, T, D), rand(gen, V, D, std=3 * D ** -0.5)
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
    targets[T // 2] = V - 1
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    api.check()
    z, e = x.double() @ w.double().t(), SUM * (x.double().abs() @ w.double().abs().t())
    want = torch.logsumexp(z, 1)
    tol = e.amax(1) + 2e-5 + 2.0 ** -22 * want.abs()
    assert ((lse.double() - want).abs() <= tol).all()
    picked = z.gather(1, targets[:, None])[:, 0] - want
    assert ((logp.double() - picked).abs() <= 2 * tol + 2.0 ** -22 * picked.abs()).all()


def test_normaliser_of_long_sums_of_one_sign():
    """Logits that are sums of products of one sign, where truncations add up: four chains of 1024 are off by what one
    is, relative to the sum (half as much again for its own spread), plus three additions in fp32 of sums of about
    25 (2^-24 * 26 * 3 = 4.7e-6) -- not by four times as much, as one sum of 4096 would be."""
    T, V, off = 333, 2011, {}
    for D in (1024, 2048, 4096):
        gen = torch.Generator(device="cuda").manual_seed(D)
        x, w = rand(gen, T, D).abs(), (rand(gen, V, D).abs().float() * 40 / D).bfloat16()
        _, lse = api.linear_logprobs_forward(x, w)
        api.check()
        z = x.double() @ w.double().t()
        error = (lse.double() - torch.logsumexp(z, 1)).abs()
        assert (error <= SUM * z.amax(1) + 2e-5 + 2.0 ** -22 * lse.abs()).all()
        off[D] = error.mean().item()
    for D in (2048, 4096):
        assert off[D] <= 1.5 * off[1024] + 5e-6, off


# K of 8192 leaves a panel of eight tiles: nine tiles are two bands
@pytest.mark.parametrize("F", [1160, 9000])
def test_gated_products_of_several_bands(F):
    """2100 tokens are nine rows of tiles, 1160 features 15 columns of them, two bands of columns; 9000 features 71, two bands
    of rows."""
    T, D = 2100, 8192
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, wg, wu = rand(gen, T, D), rand(gen, F, D, std=1.5 * D ** -0.5), rand(gen, F, D, std=D ** -0.5)
    h, (gate, up) = api.gated_linear_forward(x, wg, wu)
    api.check()
    X, G, U = x.double(), wg.double(), wu.double()
    g, u, eg, eu = X @ G.t(), X @ U.t(), SUM * (X.abs() @ G.abs().t()), SUM * (X.abs() @ U.abs().t())
    within(gate, g, HALF * g.abs() + eg, "gate")
    within(up, u, HALF * u.abs() + eu, "up")
    a = g * torch.sigmoid(g)
    within(h, a * u, (HALF + 2.0 ** -14) * (a * u).abs() + 1.2 * eg * u.abs() + a.abs() * eu + 1.2 * eg * eu, "h")


@pytest.mark.parametrize("T,D,F", [(2304, 2304, 4104), (2100, 5000, 4104), (5000, 2104, 4104), (8200, 2320, 2056)])
def test_gradients_of_several_bands(T, D, F):
    """dx: K of 2 F leaves a panel of eight tiles, two and three bands of columns, three of rows; dw of 8200 tokens: two bands
    of columns."""
    gen = torch.Generator(device="cuda").manual_seed(T)
    x, wg, wu = rand(gen, T, D), rand(gen, F, D, std=D ** -0.5), rand(gen, F, D, std=D ** -0.5)
    kept = rand(gen, T, F), rand(gen, T, F)
    dh = rand(gen, T, F, std=1e-3)
    dx, dwg, dwu = api.gated_linear_backward(dh, x, wg, wu, kept)
    api.check()
    g, u, d = kept[0].double(), kept[1].double(), dh.double()
    s = torch.sigmoid(g)
    dg, du = d * u * s * (1 + g * (1 - s)), d * g * s
    for got, ref in ((dx, dg @ wg.double() + du @ wu.double()), (dwg, dg.t() @ x.double()), (dwu, du.t() @ x.double())):
        assert (got.double() - ref).norm() <= 2.0 ** -8 * ref.norm()
        # no tile is missing or misplaced
        rows, cols = got.shape[0] // 8 * 8, got.shape[1] // 8 * 8
        block = lambda m: m[:rows, :cols].reshape(rows // 8, 8, cols // 8, 8).square().sum((1, 3)).sqrt()
        assert (block(got.double() - ref) <= 0.03 * block(ref)).all()


@pytest.mark.parametrize("T,D,V", [(2100, 8192, 5001), (5000, 8192, 2100), (2100, 8192, 20001)])
def test_loss_of_several_bands(T, D, V):
    """Bands of columns, of rows in the gradient's product, and of rows in both (nine rows of tiles by 79 columns)."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    x, w = rand(gen, T, D), rand(gen, V, D, std=2 * D ** -0.5)
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    gl = torch.randn(T, generator=gen, device="cuda") / T
    dx, dw = api.linear_logprobs_backward(x, w, targets, lse, gl)
    api.check()
    X, W = x.double(), w.double()
    z = X @ W.t()
    want = torch.logsumexp(z, 1)
    tol = SUM * (X.abs() @ W.abs().t()).amax(1) + 2e-5 + 2.0 ** -22 * want.abs()
    assert ((lse.double() - want).abs() <= tol).all()
    picked = z.gather(1, targets[:, None])[:, 0] - want
    assert ((logp.double() - picked).abs() <= 2 * tol + 2.0 ** -22 * picked.abs()).all()
    dz = -gl.double()[:, None] * torch.exp(z - lse.double()[:, None])
    dz[torch.arange(T, device="cuda"), targets] += gl.double()
    for got, ref in ((dx, dz @ W), (dw, dz.t() @ X)):
        assert (got.double() - ref).norm() <= 2.0 ** -8 * ref.norm()
