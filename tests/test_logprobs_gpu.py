"""Token log probabilities, entropy, top alternatives and their gradient against 64-bit formulas."""
import math
import struct

import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu

INF = math.inf


def logits(tokens, vocab, dtype=torch.bfloat16, std=2.5, seed=0, shift=0, pad=0):
    """Random logits as a view with `pad` extra columns, starting `shift` elements into its buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = (torch.randn(tokens * (vocab + pad) + shift, generator=g, device="cuda") * std).to(dtype)
    return flat[shift:].view(tokens, vocab + pad)[:, :vocab]


def f32(v):
    """The scale as the library receives it."""
    return struct.unpack("f", struct.pack("f", v))[0]


def reference(x, targets, top, scale=1.0):
    """Rows in 64 bits.  Masked rows and rows with NaN or +infinity by the definition's own words."""
    z = x.double() * f32(scale)
    poisoned = torch.isnan(z).any(1) | (z == INF).any(1)
    empty = (z == -INF).all(1) & ~poisoned
    top_z = z.amax(1, keepdim=True)
    d = torch.where(torch.isinf(z), -1e4, z - top_z)     # relative to the largest: the lowest value of a type absorbs a logarithm
    log_sum = torch.logsumexp(d, 1, keepdim=True)
    lse = torch.where(poisoned, math.nan, torch.where(empty, -INF, (top_z + log_sum)[:, 0]))
    logp_all = torch.where(torch.isinf(z), -INF, z - lse[:, None])
    entropy = -(torch.exp(d - log_sum) * (d - log_sum)).sum(1)
    entropy = torch.where(poisoned, math.nan, torch.where(empty, 0.0, entropy))
    logp = None
    if targets is not None:
        t = targets.clamp(0, x.shape[1] - 1)
        logp = torch.where(targets < 0, 0.0, logp_all.gather(1, t[:, None])[:, 0])
        logp = torch.where(empty & (targets >= 0), -INF, logp)
        logp = torch.where((targets >= x.shape[1]) | (poisoned & (targets >= 0)), math.nan, logp)
    if not top:
        return logp, entropy, lse, None, None
    v, i = torch.sort(torch.where(torch.isnan(z), -INF, z), dim=1, descending=True, stable=True)
    v, i = v[:, :top], i[:, :top]
    if v.shape[1] < top:
        v, i = torch.nn.functional.pad(v, (0, top - v.shape[1]), value=-INF), torch.nn.functional.pad(i, (0, top - i.shape[1]))
    i = torch.where(v == -INF, -1, i)
    v = torch.where(v == -INF, v, v - lse[:, None])
    return logp, entropy, lse, torch.where(poisoned[:, None], math.nan, v), torch.where(poisoned[:, None], -1, i)


def near(got, want, size, what):
    """fp32 values: 2^-20 of the size of what they are formed from (eight units: the exponentials' error, the
    rounded differences they are taken of, the sums and the logarithm), the same infinities and NaN."""
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= 2.0 ** -20 * size))
    assert not bad.any(), f"{what}: {int(bad.sum())}, got {got[bad][:4].tolist()} want {want[bad][:4].tolist()}"


def check_forward(x, targets=None, top=0, scale=1.0):
    got = api.logprobs_forward(x, targets, top, scale)
    want = reference(x, targets, top, scale)
    z = x.double() * f32(scale)
    size = 1.0 + torch.where(torch.isfinite(z), z.abs(), 0.0).amax(1) + want[2].nan_to_num(0, 0, 0).abs()
    near(got[2], want[2], size, "lse")
    if targets is not None:
        near(got[0], want[0], size, "logp")
    # the entropy's terms are p * (z - max), over all of the row
    near(got[1], want[1], 8.0 + 4.0 * want[1].nan_to_num(0).abs(), "entropy")
    if top:
        assert torch.equal(got[4], want[4]), (got[4][:2], want[4][:2])
        near(got[3], want[3], size[:, None], "top")
    return got


def some_targets(tokens, vocab, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    if tokens > 2:
        t[1] = -1
    return t


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,vocab", [(1, 1), (1, 2), (3, 7), (2, 8), (5, 9), (4, 63), (17, 1000), (9, 4097), (700, 513), (1, 32001),
                                          (40, 32001), (1, 128256), (3, 128256), (320, 50001), (2, 1000003)])
def test_sizes(tokens, vocab, dtype):
    x = logits(tokens, vocab, dtype, seed=vocab)
    for top in (0, 1, 20, 32):
        check_forward(x, some_targets(tokens, vocab), top)
    check_forward(x, None, 5, 0.37)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift,pad", [(1, 0), (0, 1), (3, 5), (7, 2), (0, 8)])
def test_rows_at_any_offset(shift, pad, dtype):
    for tokens, vocab in ((13, 4001), (1, 40000), (600, 130)):
        x = logits(tokens, vocab, dtype, seed=shift, shift=shift, pad=pad)
        check_forward(x, some_targets(tokens, vocab), 7, 1.7)


@pytest.mark.parametrize("tokens", [6, 700])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masks_ties_and_values_at_the_ends_of_the_type(tokens, dtype):
    vocab = 9001
    low = torch.finfo(dtype).min
    x = logits(tokens, vocab, dtype, seed=2)
    x[0] = -INF                                  # nothing left
    x[1] = -INF
    x[1, 5000] = 1.5                             # one alternative left
    x[2] = low                                   # masked by the type's lowest value: uniform
    x[3] = low
    x[3, 17], x[3, 8000] = -3.0, 2.0             # two left, then ties of the lowest value
    x[4] = 0.0
    x[4, ::2] = -0.0                             # both zeros are one value
    x[5, 100:] = -INF
    t = some_targets(tokens, vocab)
    t[0], t[1], t[2], t[3], t[4], t[5] = 3, 5000, 8, 8000, 0, 200
    for top in (3, 20, 32):
        check_forward(x, t, top)
    g = check_forward(x, t, 32)
    assert g[0][0] == -INF and g[1][0] == 0 and g[0][1] == 0 and g[1][1] == 0
    assert g[4][2].tolist() == list(range(32)) and g[4][4].tolist() == list(range(32))


@pytest.mark.parametrize("tokens", [3, 700])
def test_nan_and_infinity_poison_their_row_alone(tokens):
    x = logits(tokens, 5000, seed=3)
    x[0, 4321], x[1, 77] = math.nan, INF
    x[2, :] = -INF
    x[2, 4000] = math.nan
    check_forward(x, some_targets(tokens, 5000), 4)


@pytest.mark.parametrize("tokens", [2, 400])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_logits_all_in_a_few_threads_columns(tokens, dtype):
    """A period that puts thousands of large logits into the same few threads: far more reach the bound
    than are ranked at once."""
    vocab = 60000
    x = logits(tokens, vocab, dtype, seed=4)
    n = 16 // x.element_size()
    col = torch.arange(vocab, device="cuda")
    x += torch.where((col // n) % 512 < 9, 100.0, 0.0).to(dtype)
    check_forward(x, some_targets(tokens, vocab), 20)


def test_rising_and_spiked_rows():
    """A reference that moves many times, and a spike far above a thread's first logits."""
    vocab = 70000
    x = torch.linspace(-500, 500, vocab, device="cuda").repeat(4, 1)
    x[1] = x[1].flip(0)
    x[2] = logits(1, vocab, torch.float32, seed=5)[0]
    x[2, 65000] = 60.0
    x[3] = 0.0
    x[3, 12345] = 25.0
    check_forward(x, some_targets(4, vocab), 20)
    check_forward(x, some_targets(4, vocab), 20, 30.0)
    check_forward(x.bfloat16(), some_targets(4, vocab), 20, 0.01)


@pytest.mark.parametrize("tokens", [4, 700])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [1e-28, 1e-6, 1e5, 1e9])
def test_scales_far_from_one(tokens, dtype, scale):
    x = logits(tokens, 3001, dtype, seed=11)
    x[0, 100:200] = -INF
    x[1] = -INF
    x[2] *= 1e20
    check_forward(x, some_targets(tokens, 3001), 5, scale)


@pytest.mark.parametrize("tokens", [3, 700])
def test_rows_at_the_ends_of_fp32(tokens):
    """Largest logits whose scaled value leaves fp32, of either sign, beside ordinary rows."""
    x = logits(tokens, 5003, torch.float32, seed=12)
    x[0] = -3e38
    x[0, 7::50] = -2.9e38
    x[1] = 0.0
    x[1, 4000:4003] = 3.3e38
    x[2] = -2e30
    x[2, 17] = -1.5e30
    got = check_forward(x, some_targets(tokens, 5003), 7, 0.5)
    assert abs(got[1][1].item() - math.log(3)) < 1e-5 and got[1][2] == 0


def test_out_of_range_target_is_nan():
    x = logits(4, 100, seed=6)
    t = torch.tensor([0, 100, 1 << 40, -5], device="cuda")
    logp, entropy, lse, _, _ = api.logprobs_forward(x, t)
    assert torch.isnan(logp).tolist() == [False, True, True, False] and logp[3] == 0
    d = api.logprobs_backward(x, t, lse, entropy, torch.ones(4, device="cuda"))
    assert torch.isnan(d).all(1).tolist() == [False, True, True, False] and (d[3] == 0).all()


def backward_reference(x, t, lse, entropy, gl, ge, scale):
    scale = f32(scale)
    z = x.double() * scale
    l = torch.where(torch.isinf(z), -1e4, z - lse.double()[:, None])
    p = torch.exp(l)
    g = torch.where(t >= 0, gl.double(), 0.0)[:, None] if gl is not None else torch.zeros_like(p[:, :1])
    e = ge.double()[:, None] if ge is not None else torch.zeros_like(p[:, :1])
    H = entropy.double()[:, None] if entropy is not None else 0.0
    d = -p * (g + e * (l + H))
    size = p * (g.abs() + e.abs() * (l.abs() + H)) * (1.0 + l.abs())
    d.scatter_add_(1, t.clamp(min=0)[:, None], g)
    size.scatter_add_(1, t.clamp(min=0)[:, None], g.abs())
    empty = torch.isinf(lse)[:, None]
    return torch.where(empty, 0.0, d * scale), torch.where(empty, 0.0, size * scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,vocab,shift,pad", [(1, 1, 0, 0), (3, 7, 0, 0), (5, 1000, 0, 0), (4, 4001, 3, 4), (2, 128256, 0, 0), (65, 32001, 0, 0),
                                                    (9, 33000, 1, 7)])
def test_backward(tokens, vocab, shift, pad, dtype):
    x = logits(tokens, vocab, dtype, seed=tokens, shift=shift, pad=pad)
    if vocab > 500:
        x[0, 100:] = -INF
        if tokens > 2:
            x[2] = -INF
    t = some_targets(tokens, vocab)
    t[0] = min(int(t[0]), 99)
    g = torch.Generator(device="cuda").manual_seed(3)
    gl, ge = (torch.randn(tokens, generator=g, device="cuda") for _ in range(2))
    for scale in (1.0, 0.6):
        _, entropy, lse, _, _ = api.logprobs_forward(x, t, 0, scale)
        for a, b in ((gl, None), (None, ge), (gl, ge)):
            got = api.logprobs_backward(x, t, lse, entropy, a, b, scale)
            want, size = backward_reference(x, t, lse, entropy, a, b, scale)
            # 2^-21 of the terms (with the error of an exponential growing with its argument), and the type's half step
            tol = 2.0 ** -21 * size + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0) + 1e-37
            bad = ~((got.double() - want).abs() <= tol)
            assert not bad.any(), (int(bad.sum()), ((got.double() - want).abs() / tol).max())
        for out in (x.clone(), logits(tokens, vocab, dtype, shift=1, pad=3)):    # in place, and at another offset
            src = out if out.data_ptr() % 16 == 0 and out.is_contiguous() else x
            assert torch.equal(api.logprobs_backward(src, t, lse, entropy, gl, ge, scale, out), got)


def test_rows_without_gradient_are_zero_and_their_logits_not_used():
    x = logits(3, 2000, seed=7)
    x[1, 5] = math.nan
    t = torch.tensor([4, -1, 9], device="cuda")
    _, entropy, lse, _, _ = api.logprobs_forward(x, t)
    d = api.logprobs_backward(x, t, lse, entropy, torch.ones(3, device="cuda"))
    assert (d[1] == 0).all() and torch.isfinite(d).all() and (d[0] != 0).any()


def test_backward_against_differences():
    x = logits(3, 200, torch.float32, seed=8)
    t = torch.tensor([3, 199, 60], device="cuda")
    gl, ge = torch.tensor([1.0, -0.5, 2.0], device="cuda"), torch.tensor([0.3, 1.0, -0.7], device="cuda")
    _, entropy, lse, _, _ = api.logprobs_forward(x, t, 0, 0.8)
    got = api.logprobs_backward(x, t, lse, entropy, gl, ge, 0.8).double()

    def loss(v):
        logp, ent, *_ = reference(v, t, 0, 0.8)
        return (logp * gl + ent * ge).sum().item()

    d = torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda", dtype=torch.float64)
    eps = 1e-5
    diff = (loss(x.double() + eps * d) - loss(x.double() - eps * d)) / (2 * eps)
    # the differences' own error is of order eps^2; the gradient's is fp32's
    assert abs((got * d).sum().item() - diff) <= 2e-6 * (got * d).abs().sum().item() + 1e-8


def test_calls_repeat_bit_for_bit_and_follow_their_stream():
    x, t = logits(5, 128256, seed=9), some_targets(5, 128256)
    want = api.logprobs_forward(x, t, 20)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [api.logprobs_forward(x, t, 20) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


@pytest.mark.parametrize("tokens", [2, 700])
def test_scaled_logits_below_the_range_keep_their_place(tokens):
    """Finite logits whose scaled value is below fp32's range have probability 0 but stay alternatives; a row of nothing
    else counts as masked entirely."""
    low = torch.finfo(torch.float32).min
    x = torch.full((tokens, 40), low, device="cuda")
    x[::2, 7], x[::2, 9], x[:, 3] = 1.0, 0.0, float("-inf")
    logp, entropy, lse, top_logp, top_index = api.logprobs_forward(x, None, 4, 2.0)
    api.check()
    assert (top_index[::2] == torch.tensor([7, 9, 0, 1], device="cuda")).all()
    assert torch.isinf(top_logp[::2, 2:]).all() and torch.isfinite(top_logp[::2, :2]).all()
    assert (top_index[1::2] == -1).all() and (lse[1::2] == float("-inf")).all() and (entropy[1::2] == 0).all()


@pytest.mark.parametrize("tokens", [2, 700])
def test_scaled_logits_above_the_range_poison_their_row_alone(tokens):
    x = torch.zeros((tokens, 40), device="cuda")
    x[::2, 5] = torch.finfo(torch.float32).max
    targets = torch.full((tokens,), 5, device="cuda")
    logp, entropy, lse, top_logp, top_index = api.logprobs_forward(x, targets, 3, 2.0)
    api.check()
    for v in (logp, entropy, lse, top_logp):
        assert torch.isnan(v[::2]).all() and torch.isfinite(v[1::2]).all()
    assert (top_index[::2] == -1).all() and (top_index[1::2] == torch.arange(3, device="cuda")).all()


def far_reference(x, targets, top, scale):
    """logp, entropy, top alternatives in 64 bits from differences to the row's largest logit, which stay exact
    whatever the rows' common offset; lse loses log n there in any precision."""
    z = x.double() * f32(scale)
    d = z - z.amax(1, keepdim=True)
    logp = d - torch.logsumexp(d, 1, keepdim=True)
    entropy = -(logp.exp() * torch.where(torch.isinf(logp), 0.0, logp)).sum(1)
    v, i = torch.sort(logp, dim=1, descending=True, stable=True)
    return torch.where(targets < 0, 0.0, logp.gather(1, targets.clamp(min=0)[:, None])[:, 0]), entropy, v[:, :top], i[:, :top]


@pytest.mark.parametrize("tokens,vocab", [(3, 1000), (3, 40001), (700, 1003)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [2.0 ** 12, -2.0 ** 20, 2.0 ** 24, -1e30, "lowest"])
def test_log_probabilities_do_not_depend_on_a_common_offset(tokens, vocab, dtype, offset):
    """Rows far from zero: the difference of two logits is what counts.  The tolerance is 2^-20 of the sizes of
    that difference and of the logarithm (a rounding of the difference, one of the sum, and the logarithm's eight
    units), not of the logits."""
    low = torch.finfo(dtype).min
    x = (logits(tokens, vocab, torch.float32, seed=21) + (low if offset == "lowest" else offset)).clamp(min=low).to(dtype)
    x[0] = x[0, 0]                               # uniform
    x[-1, : vocab // 3] = -INF
    t = some_targets(tokens, vocab)
    t[0], t[-1] = 5, vocab - 1
    for scale in (1.0, 0.5):
        logp, entropy, _, top_logp, top_index = api.logprobs_forward(x, t, 20, scale)
        api.check()
        w_logp, w_entropy, w_top, w_index = far_reference(x, t, 20, scale)
        near(logp, w_logp, 1.0 + w_logp.abs() + math.log(vocab), "logp")
        assert torch.equal(top_index, w_index)
        near(top_logp, w_top, 1.0 + w_top.abs() + math.log(vocab), "top")
        near(entropy, w_entropy, 8.0 + 4.0 * w_entropy.abs(), "entropy")
        assert abs(logp[0].item() + math.log(vocab)) < 1e-5


def test_out_of_range_target_is_nan_in_a_masked_row_too():
    x = logits(3, 100, seed=6)
    x[0], x[1] = -INF, -INF
    t = torch.tensor([100, 7, 3], device="cuda")
    logp, entropy, lse, _, _ = api.logprobs_forward(x, t)
    d = api.logprobs_backward(x, t, lse, entropy, torch.ones(3, device="cuda"))
    api.check()
    assert torch.isnan(logp).tolist() == [True, False, False]
    assert torch.isnan(d[0]).all() and (d[1] == 0).all() and torch.isfinite(d[2]).all()
