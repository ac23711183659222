"""Every call around the linears runs on the stream that is current when it is made: its inputs arrive there late,
behind a delay of some milliseconds, so a launch on any other stream would read what the buffers held before."""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu

DELAY_CYCLES = 20_000_000


def on_a_late_stream(call, real, old):
    """The call's results on a side stream that first waits, then copies `real` over `old`."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY_CYCLES)
        for buf, t in zip(old, real):
            buf.copy_(t)
        out = call(*old)
        assert not side.query(), "the delay was over before the call was made"
    side.synchronize()
    api.check()
    return out


def check(call, *real):
    old = [t.flip(0).mul(2).contiguous() if t.is_floating_point() else torch.zeros_like(t) for t in real]
    stale = call(*old)
    want = call(*real)
    got = on_a_late_stream(call, real, old)
    flat = lambda r: [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]
    assert any(not torch.equal(a, b) for a, b in zip(flat(stale), flat(want)))
    assert all(torch.equal(a, b) for a, b in zip(flat(got), flat(want)))


def rand(*shape, dtype=torch.bfloat16, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("shape", [api.BLOCK_1X128, api.BLOCK_128X128])
def test_quantizer(axis, shape):
    check(lambda x: api.quantize_block128(x, axis, shape), rand(272, 400))


@pytest.mark.parametrize("tokens", [2, 300, 40])
def test_product(tokens):
    n, k = (4096, 4096) if tokens == 40 else (520, 400)              # split along K: two kernels
    b = api.quantize_block128(rand(n, k, seed=1), api.AXIS_COLS, api.BLOCK_128X128)
    check(lambda c, s: api.gemm_block128(c, s, *b), *api.quantize_block128(rand(tokens, k)))


@pytest.mark.parametrize("pass_", [api.PASS_FPROP, api.PASS_DGRAD, api.PASS_WGRAD])
def test_linear_pass(pass_):
    T, i, o = 400, 272, 528
    a, b = {api.PASS_FPROP: ((T, i), (o, i)), api.PASS_DGRAD: ((T, o), (o, i)), api.PASS_WGRAD: ((T, o), (T, i))}[pass_]
    check(lambda x, y: api.linear_pass_block128(pass_, x, y), rand(*a), rand(*b, seed=1))


@pytest.mark.parametrize("tokens,width", [(1, 4096), (300, 1032), (5, 8192)])
def test_residual_norm(tokens, width):
    w = rand(width, dtype=torch.float32, seed=2)
    m = [rand(tokens, width, seed=s) for s in range(3, 7)]
    check(lambda u, x, g: api.residual_norm_forward(u, x, w, w, g, api.GATE_SILU), *m[:3])
    check(lambda dh, u, y: api.residual_norm_backward(dh, None, u, y, w, w), *m[1:])


@pytest.mark.parametrize("tokens,vocab", [(1, 128256), (700, 3001)])
def test_log_probabilities(tokens, vocab):
    x, t = rand(tokens, vocab), torch.full((tokens,), 9, device="cuda")
    check(lambda x: api.logprobs_forward(x, t, 5), x)
    _, entropy, lse, _, _ = api.logprobs_forward(x, t)
    d = torch.ones(tokens, device="cuda")
    check(lambda x: api.logprobs_backward(x, t, lse, entropy, d, d), x)
