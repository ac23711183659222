"""Log probabilities from an output layer's input and weight against the formulas in 64 bits.

Bounds.  A logit is off by at most 1e-5 of the sum of its products' magnitudes (fp32 accumulation); the row's lse by the
largest such error, 2e-5 for the sum of exponentials (a sum of 128 fp32 terms: 128 * 2^-24, exponentials of 2^-22,
joins of the pieces) and its rounding.  In the backward pass p carries the logit's error, and dz is rounded to
bf16 before it is summed: 2^-8 of each product's magnitude, and for the whole matrix, where errors are
independent, 2^-8 of the norm (twice what a rounding of operand and result gives).
"""
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


HALF, SUM, EXP = 2.0 ** -8, 1e-5, 2e-5


def inputs(T, D, V, seed=0, std=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, w = rand(T, D).bfloat16(), (rand(V, D) * std * D ** -0.5).bfloat16()
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
    targets[::7] = -1
    targets[T // 2] = V - 1
    if T > 3:
        targets[3] = 0
    return x, w, targets, gen


def reference(x, w, targets, scale=1.0):
    X, W = x.double(), w.double()
    z, e = scale * (X @ W.t()), scale * SUM * (X.abs() @ W.abs().t())
    lse = torch.logsumexp(z, 1)
    logp = torch.where(targets >= 0, z.gather(1, targets.clamp(min=0)[:, None])[:, 0] - lse, 0.0)
    return z, e, lse, logp


def check_forward(x, w, targets, logp, lse, scale=1.0):
    z, e, want_lse, want = reference(x, w, targets, scale)
    tol = e.amax(1) + EXP + 2.0 ** -22 * want_lse.abs()
    assert ((lse.double() - want_lse).abs() <= tol).all()
    assert ((logp.double() - want).abs() <= 2 * tol + 2.0 ** -22 * want.abs()).all()
    assert (logp[targets < 0] == 0).all()


SIZES = [(1, 8, 1), (1, 64, 1000), (2, 72, 129), (31, 128, 8), (33, 264, 4097), (130, 64, 127), (257, 136, 2011), (300, 520, 32001), (400, 64, 14900)]


@pytest.mark.parametrize("T,D,V", SIZES)
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_forward(T, D, V, scale):
    x, w, targets, _ = inputs(T, D, V)
    logp, lse = api.linear_logprobs_forward(x, w, targets, scale)
    none, alone = api.linear_logprobs_forward(x, w, None, scale)
    api.check()
    check_forward(x, w, targets, logp, lse, scale)
    assert none is None and torch.equal(alone, lse)


def check_backward(x, w, targets, lse, gl, gn, dx, dw, scale=1.0, dw32=False, whole=True):
    X, W = x.double(), w.double()
    z, e, _, _ = reference(x, w, targets, scale)
    p = torch.exp(z - lse.double()[:, None])
    l = torch.where(targets >= 0, gl.double(), 0.0)[:, None] if gl is not None else torch.zeros_like(p[:, :1])
    n = gn.double()[:, None] if gn is not None else torch.zeros_like(l)
    one = torch.zeros_like(p)
    has = (targets >= 0).nonzero()[:, 0] if targets is not None else []
    if len(has):
        one[has, targets[has]] = 1
    dz = scale * (l * (one - p) + n * p)
    edz = HALF * dz.abs() + scale * (n - l).abs() * p * (e + 4e-6 + 2.0 ** -22 * (z.abs() + lse.double().abs()[:, None]))
    for got, ref, tol, bits in ((dx, dz @ W, (edz + SUM * dz.abs()) @ W.abs(), HALF),
                                (dw, dz.t() @ X, (edz + SUM * dz.abs()).t() @ X.abs(), 2.0 ** -24 if dw32 else HALF)):
        if got is None:
            continue
        bad = ~((got.double() - ref).abs() <= tol + bits * ref.abs() + 1e-30)
        assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off"
        if whole:
            assert (got.double() - ref).norm() <= 2.0 ** -8 * ref.norm()


@pytest.mark.parametrize("T,D,V", SIZES + [(40, 64, 9001), (20000, 16, 9000)])
@pytest.mark.parametrize("dw", [api.OUT_BF16, api.OUT_FP32])
def test_backward(T, D, V, dw):
    x, w, targets, gen = inputs(T, D, V)
    gl, gn = (torch.randn(T, generator=gen, device="cuda") / T for _ in range(2))
    gl[:: 5] = 0
    lse = reference(x, w, targets, 0.7)[2].float()
    got = api.linear_logprobs_backward(x, w, targets, lse, gl, gn, 0.7, dw)
    api.check()
    check_backward(x, w, targets, lse, gl, gn, *got, scale=0.7, dw32=dw == api.OUT_FP32, whole=T * D * V > 1 << 18)


def test_pieces_of_the_vocabulary():
    """16384 tokens are a piece of 8192 columns: three pieces, the last one short."""
    T, D, V = 16384, 64, 8192 * 2 + 77
    x, w, targets, gen = inputs(T, D, V)
    gl, gn = (torch.randn(T, generator=gen, device="cuda") / T for _ in range(2))
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    dx, dw = api.linear_logprobs_backward(x, w, targets, lse, gl, gn)
    api.check()
    check_forward(x, w, targets, logp, lse)
    check_backward(x, w, targets, lse, gl, gn, dx, dw)


def test_a_last_piece_shorter_than_its_splits():
    """2048 tokens of 64 features: pieces of 65536 columns, split along K; the last one has a single step for them."""
    T, D, V = 2048, 64, 65536 + 40
    x, w, targets, gen = inputs(T, D, V)
    targets[5] = V - 20
    gl = torch.randn(T, generator=gen, device="cuda") / T
    _, lse = api.linear_logprobs_forward(x, w, targets)
    dx, dw = api.linear_logprobs_backward(x, w, targets, lse, gl)
    api.check()
    check_backward(x, w, targets, lse, gl, None, dx, dw)


def test_more_rows_than_one_product_takes():
    x, w, targets, _ = inputs(16384 + 300, 16, 520)
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    api.check()
    check_forward(x, w, targets, logp, lse)


def test_one_gradient_only_and_unwanted_results():
    x, w, targets, gen = inputs(70, 64, 500)
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    g, zero = torch.randn(70, generator=gen, device="cuda"), torch.zeros(70, device="cuda")
    for a, b, t in ((g, None, targets), (None, g, targets), (None, g, None)):
        got = api.linear_logprobs_backward(x, w, t, lse, a, b)
        full = api.linear_logprobs_backward(x, w, targets, lse, a if a is not None else zero, b if b is not None else zero)
        assert torch.equal(got[0], full[0]) and torch.equal(got[1], full[1])
    dx, none = api.linear_logprobs_backward(x, w, targets, lse, g, want_dw=False)
    none2, dw = api.linear_logprobs_backward(x, w, targets, lse, g, want_dx=False)
    both = api.linear_logprobs_backward(x, w, targets, lse, g)
    api.check()
    assert none is None and none2 is None and torch.equal(dx, both[0]) and torch.equal(dw, both[1])


def test_targets_out_of_range_and_rows_that_are_not_finite():
    x, w, targets, gen = inputs(40, 64, 300)
    targets[:4] = torch.tensor([-1, 300, 1 << 40, -(1 << 40)], device="cuda")
    x[10, 3] = float("nan")
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    assert logp[0] == 0 and logp[1].isnan() and logp[2].isnan() and logp[3] == 0
    assert lse[10].isnan() and logp[10].isnan() and int(lse.isnan().sum()) == 1
    x[10, 3] = 1.0
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    g = torch.ones(40, device="cuda")
    dx, _ = api.linear_logprobs_backward(x, w, targets, lse, g)
    api.check()
    assert dx[1].isnan().all() and dx[2].isnan().all() and int(dx.isnan().any(1).sum()) == 2
    assert (dx[0] == 0).all() and (dx[3] == 0).all()


def test_rows_without_gradients_add_nothing_whatever_their_logits():
    x, w, targets, gen = inputs(40, 64, 300)
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    g = torch.randn(40, generator=gen, device="cuda")
    g[5:9] = 0
    want = api.linear_logprobs_backward(x, w, targets, lse, g)
    lse[5], lse[6] = float("nan"), float("inf")
    x[7] = 3e38                                       # its logits are infinite or NaN
    got = api.linear_logprobs_backward(x, w, targets, lse, g)
    api.check()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert (got[0][5:9] == 0).all()


def test_large_logits_and_a_common_offset():
    """Logits of some hundreds: exponentials are of differences to the row's maximum."""
    x, w, targets, _ = inputs(64, 128, 777, std=300.0)
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    api.check()
    check_forward(x, w, targets, logp, lse)
    assert lse.max() > 100 and lse.isfinite().all()


def test_strides_and_untouched_surroundings():
    T, D, V = 50, 136, 203
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()
    x, w = rand(T + 2, D + 16)[1:-1, 8:-8], rand(V + 2, D + 16)[1:-1, 8:-8]
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    again = api.linear_logprobs_forward(x.contiguous(), w.contiguous(), targets)
    assert torch.equal(logp, again[0]) and torch.equal(lse, again[1])
    rooms = [torch.full((n + 2, D + 16), 7.0, dtype=torch.bfloat16, device="cuda") for n in (T, V)]
    g = torch.ones(T, device="cuda")
    dx, dw = api.linear_logprobs_backward(x, w, targets, lse, g, dx=rooms[0][1:-1, 8:-8], dw=rooms[1][1:-1, 8:-8])
    api.check()
    check_backward(x, w, targets, lse, g, None, dx, dw, whole=False)
    for room in rooms:
        assert (room[0] == 7).all() and (room[-1] == 7).all() and (room[:, :8] == 7).all() and (room[:, -8:] == 7).all()


def test_agrees_with_the_log_probabilities_of_finished_logits():
    x, w, targets, _ = inputs(100, 128, 3001)
    logp, lse = api.linear_logprobs_forward(x, w, targets)
    z = (x.float() @ w.float().t()).contiguous()
    logp2, _, lse2, _, _ = api.logprobs_forward(z, targets)
    api.check()
    assert (logp - logp2).abs().max() <= 2e-4 and (lse - lse2).abs().max() <= 1e-4


def test_repeats_bit_for_bit_and_as_a_graph():
    x, w, targets, gen = inputs(300, 64, 5001)
    g = torch.randn(300, generator=gen, device="cuda")

    def step():
        logp, lse = api.linear_logprobs_forward(x, w, targets)
        return (logp, lse, *api.linear_logprobs_backward(x, w, targets, lse, g))

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
