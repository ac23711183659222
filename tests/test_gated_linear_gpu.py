"""The gated projections against the formulas in 64 bits.

Bounds.  A sum of the tensor cores is off by at most 1e-5 of the sum of its products' magnitudes (fp32
accumulation over a few thousand terms), a rounding to bf16 by 2^-8 of the value.  The activations' values are off by
at most 2^-14 of themselves (an exponential of 2 + 1.17 |x| units in the last place, |x| <= 88, and the rounding of its
argument), their derivatives by 2^-14 in absolute terms; both are below 1.13 times max(1, |g|) and 1.13 in magnitude.
In the backward pass dg and du are rounded to bf16 before they are summed: 2^-8 of each product's magnitude, and for
the whole matrix, where errors are independent, 2^-8 of the norm (twice what a rounding of operand and result gives).
"""
import math

import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def memory_returned():
    """What the large cases had goes back to the device: the allocator would otherwise give it back in some later test,
    which waits for all of the device's work."""
    yield
    torch.cuda.empty_cache()


HALF, ACT, SUM = 2.0 ** -8, 2.0 ** -14, 1e-5
ACTS = [api.GATE_LINEAR, api.GATE_SIGMOID, api.GATE_SILU, api.GATE_GELU, api.GATE_GELU_TANH, api.GATE_RELU]


def act(g, which):
    """Value and derivative in 64 bits."""
    if which == api.GATE_LINEAR:
        return g, torch.ones_like(g)
    if which == api.GATE_RELU:
        return g.clamp(min=0), (g > 0).double()
    if which == api.GATE_GELU:
        cdf = torch.special.ndtr(g)
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if which == api.GATE_GELU_TANH:
        c = math.sqrt(2 / math.pi)
        s = torch.sigmoid(2 * c * (g + 0.044715 * g ** 3))
        return g * s, s + 2 * g * s * (1 - s) * c * (1 + 3 * 0.044715 * g * g)
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if which == api.GATE_SIGMOID else (g * s, s + g * s * (1 - s))


def rand(gen, *shape, std=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).bfloat16()


def inputs(T, D, F, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return rand(gen, T, D), rand(gen, F, D, std=1.5 * D ** -0.5), rand(gen, F, D, std=D ** -0.5), gen


def within(got, ref, tol, what):
    bad = ~((got.double() - ref).abs() <= tol + 1e-30)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {((got.double() - ref).abs() / tol).max()} of the bound"


def check_forward(x, wg, wu, which, h, kept):
    X, G, U = x.double(), wg.double(), wu.double()
    g, u = X @ G.t(), X @ U.t()
    eg, eu = SUM * (X.abs() @ G.abs().t()), SUM * (X.abs() @ U.abs().t())
    a, _ = act(g, which)
    within(h, a * u, (HALF + ACT) * (a * u).abs() + 1.2 * eg * u.abs() + a.abs() * eu + 1.2 * eg * eu, "h")
    if kept is not None:
        within(kept[0], g, HALF * g.abs() + eg, "gate")
        within(kept[1], u, HALF * u.abs() + eu, "up")


SIZES = [(1, 8, 8), (1, 4096, 264), (20, 2056, 1000), (300, 2048, 1304), (290, 64, 14336), (170, 1024, 1304), (400, 1536, 9608), (1100, 1024, 2056), (1100, 2048, 136), (333, 2056, 72), (200, 72, 9608), (9, 136, 328), (2, 64, 72), (17, 72, 128), (31, 200, 136), (129, 128, 520), (255, 1032, 264),
         (257, 96, 1000), (600, 520, 392), (1030, 64, 16), (5, 16, 20000)]


@pytest.mark.parametrize("T,D,F", SIZES)
@pytest.mark.parametrize("keep", [False, True])
def test_forward(T, D, F, keep):
    x, wg, wu, _ = inputs(T, D, F)
    h, kept = api.gated_linear_forward(x, wg, wu, keep=keep)
    api.check()
    assert (kept is not None) == keep
    check_forward(x, wg, wu, api.GATE_SILU, h, kept)


@pytest.mark.parametrize("which", ACTS)
@pytest.mark.parametrize("T", [3, 40, 300])
def test_activations(which, T):
    x, wg, wu, gen = inputs(T, 256, 264, 1)
    x[::3] *= 12                                        # gates far from zero too
    h, kept = api.gated_linear_forward(x, wg, wu, which)
    check_forward(x, wg, wu, which, h, kept)
    dh = rand(gen, T, 264)
    got = api.gated_linear_backward(dh, x, wg, wu, kept, which)
    api.check()
    check_backward(dh, x, wg, wu, kept, which, *got, whole=False)


def check_backward(dh, x, wg, wu, kept, which, dx, dwg, dwu, dw32=False, whole=True):
    X, G, U, D = x.double(), wg.double(), wu.double(), dh.double()
    g, u = kept[0].double(), kept[1].double()
    a, da = act(g, which)
    dg, du = D * u * da, D * a
    edg, edu = HALF * dg.abs() + ACT * (D * u).abs(), (HALF + ACT) * du.abs()
    for got, ref, tol, bits in (
            (dx, dg @ G + du @ U, (edg + SUM * dg.abs()) @ G.abs() + (edu + SUM * du.abs()) @ U.abs(), HALF),
            (dwg, dg.t() @ X, (edg + SUM * dg.abs()).t() @ X.abs(), 2.0 ** -24 if dw32 else HALF),
            (dwu, du.t() @ X, (edu + SUM * du.abs()).t() @ X.abs(), 2.0 ** -24 if dw32 else HALF)):
        if got is None:
            continue
        within(got, ref, tol + bits * ref.abs(), "gradient")
        if whole:
            assert (got.double() - ref).norm() <= 2.0 ** -8 * ref.norm()


@pytest.mark.parametrize("T,D,F", SIZES)
@pytest.mark.parametrize("dw", [api.OUT_BF16, api.OUT_FP32])
def test_backward(T, D, F, dw):
    x, wg, wu, gen = inputs(T, D, F)
    kept = rand(gen, T, F), rand(gen, T, F)
    dh = rand(gen, T, F, std=1e-3)
    got = api.gated_linear_backward(dh, x, wg, wu, kept, api.GATE_SILU, dw)
    api.check()
    assert got[1].dtype == got[2].dtype == (torch.float32 if dw == api.OUT_FP32 else torch.bfloat16)
    check_backward(dh, x, wg, wu, kept, api.GATE_SILU, *got, dw32=dw == api.OUT_FP32, whole=T * D * F > 1 << 16)


def test_gradient_against_differences():
    """Along a random direction of each input: (h(p + e d) - h(p - e d)) / 2 e in 64 bits, summed with dh, is the inner
    product of the direction and the gradient.  The gradient's error is within 2^-8 of its norm (above), its inner
    product with a direction of unit length within that; e^2 and the difference's own rounding are below 1e-7."""
    T, D, F = 40, 64, 72
    x, wg, wu, gen = inputs(T, D, F, 3)
    h, kept = api.gated_linear_forward(x, wg, wu)
    dh = rand(gen, T, F)
    grads = api.gated_linear_backward(dh, x, wg, wu, kept, dw_dtype=api.OUT_FP32)
    api.check()
    values = [t.double() for t in (x, wg, wu)]

    def loss(v):
        return ((v[0] @ v[1].t()) * torch.sigmoid(v[0] @ v[1].t()) * (v[0] @ v[2].t()) * dh.double()).sum()

    # the stored g and u are off by 2^-8 of themselves: as much again in dg and du
    for i in range(3):
        for seed in range(4):
            d = torch.randn(values[i].shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").double()
            d /= d.norm()
            e = 1e-4
            move = lambda s: [v + s * e * d if j == i else v for j, v in enumerate(values)]
            slope = (loss(move(1)) - loss(move(-1))) / (2 * e)
            assert abs(slope - (grads[i].double() * d).sum()) <= 3 * 2.0 ** -8 * grads[i].double().norm()


@pytest.mark.parametrize("T", [1, 7, 50, 300])
def test_strides_halves_of_one_weight_and_untouched_surroundings(T):
    D, F = 136, 200
    gen = torch.Generator(device="cuda").manual_seed(T)
    both = rand(gen, 2 * F, D + 24, std=0.1)[:, :D]
    wg, wu = both[:F], both[F:]
    x = rand(gen, T + 2, D + 8)[1:-1, 8:]
    room = torch.full((T + 2, F + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    h, kept = api.gated_linear_forward(x, wg, wu, h=room[1:-1, 8:-8])
    check_forward(x, wg, wu, api.GATE_SILU, h, kept)
    plain, _ = api.gated_linear_forward(x.contiguous(), wg.contiguous(), wu.contiguous())
    assert torch.equal(h, plain)
    assert (room[0] == 7).all() and (room[-1] == 7).all() and (room[:, :8] == 7).all() and (room[:, -8:] == 7).all()
    dh = rand(gen, T, F + 8)[:, :F]
    dx_room, dw_room = (torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in ((T + 2, D + 16), (2 * F + 2, D + 16)))
    dw = dw_room[1:-1, 8:-8]
    got = api.gated_linear_backward(dh, x, wg, wu, kept, dx=dx_room[1:-1, 8:-8], dw_gate=dw[:F], dw_up=dw[F:])
    api.check()
    check_backward(dh, x, wg, wu, kept, api.GATE_SILU, *got, whole=False)
    for room in (dx_room, dw_room):
        assert (room[0] == 7).all() and (room[-1] == 7).all() and (room[:, :8] == 7).all() and (room[:, -8:] == 7).all()


def test_more_than_2_to_the_31_elements():
    T, D, F = 150100, 16, 14400                      # 2.16e9 in h, and in each of its companions
    x, wg, wu, gen = inputs(T, D, F)
    h, kept = api.gated_linear_forward(x, wg, wu)
    api.check()
    for rows in (slice(0, 40), slice(149120, 149160), slice(T - 40, T)):
        check_forward(x[rows], wg, wu, api.GATE_SILU, h[rows], [t[rows] for t in kept])
    dh = torch.zeros_like(h)
    del h
    dh[-3:] = rand(gen, 3, F)
    dx, dwg, dwu = api.gated_linear_backward(dh, x, wg, wu, kept)
    api.check()
    assert (dx[:-3] == 0).all()
    check_backward(dh[-3:], x[-3:], wg, wu, [t[-3:] for t in kept], api.GATE_SILU, dx[-3:], dwg, dwu, whole=False)


def test_activations_far_from_the_origin():
    """Where exponentials and squares leave fp32's range: values and slopes are the limits."""
    x = torch.tensor([[1.0], [-1.0], [100.0], [-100.0]], device="cuda").bfloat16().expand(4, 8).contiguous()
    x[:, 1:] = 0
    wg = torch.zeros(8, 8, device="cuda").bfloat16()
    wg[:, 0] = torch.tensor([1.0, 30.0, 100.0, 1e4, 1e10, 1e18, 1e25, 0.0], device="cuda")
    one = torch.zeros(8, 8, device="cuda").bfloat16()
    one[:, 0] = 1.0
    for which in ACTS:
        h, kept = api.gated_linear_forward(x, wg, one, which)
        check_forward(x, wg, one, which, h, kept)
        dh = torch.ones_like(h)
        got = api.gated_linear_backward(dh, x, wg, one, kept, which)
        api.check()
        assert all(g.isfinite().all() for g in got), which


def test_unwanted_gradients():
    x, wg, wu, gen = inputs(70, 128, 136)
    _, kept = api.gated_linear_forward(x, wg, wu)
    dh = rand(gen, 70, 136)
    dx, dwg, dwu = api.gated_linear_backward(dh, x, wg, wu, kept)
    a = api.gated_linear_backward(dh, x, wg, wu, kept, want_dw=False)
    b = api.gated_linear_backward(dh, x, wg, wu, kept, want_dx=False)
    api.check()
    assert torch.equal(a[0], dx) and a[1] is None and a[2] is None
    assert b[0] is None and torch.equal(b[1], dwg) and torch.equal(b[2], dwu)


@pytest.mark.parametrize("T", [4, 40, 400])
def test_infinities_and_nans_stay_in_their_rows(T):
    x, wg, wu, _ = inputs(T, 64, 72)
    clean, _ = api.gated_linear_forward(x, wg, wu)
    x[1, 3], x[2, 5] = float("nan"), float("inf")
    h, _ = api.gated_linear_forward(x, wg, wu)
    api.check()
    assert h[1].isnan().all() and not h[2].isfinite().any()
    keep = [i for i in range(T) if i not in (1, 2)]
    assert torch.equal(h[keep], clean[keep])


def test_repeats_bit_for_bit_and_as_a_graph():
    x, wg, wu, gen = inputs(300, 264, 520)
    dh = rand(gen, 300, 520)

    def step():
        h, kept = api.gated_linear_forward(x, wg, wu)
        return (h, *kept, *api.gated_linear_backward(dh, x, wg, wu, kept))

    want = step()
    assert all(torch.equal(a, b) for a, b in zip(want, step()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for t in out:
        t.zero_()
    graph.replay()
    api.check()
    assert all(torch.equal(a, b) for a, b in zip(want, out))
