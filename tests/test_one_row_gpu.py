"""A single row has no pitch: whatever stride a one-row view carries, the calls around the linears take it."""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu

WIDTH = 4096


def odd(dtype, seed, width=WIDTH):
    """A one-row view of a buffer whose rows are 4100 (odd multiples of 4) elements apart, and its compact copy."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    view = torch.randn(2, width + 4, generator=g, device="cuda").to(dtype)[:1, :width]
    assert view.stride(0) % 8 != 0
    return view, view.clone(memory_format=torch.contiguous_format)


def both(call, *pairs):
    """The call on the views and on the compact copies."""
    return call(*(p[0] for p in pairs)), call(*(p[1] for p in pairs))


def equal(a, b):
    return all((x is None and y is None) or torch.equal(x, y) for x, y in zip(a, b))


def test_quantizer():
    x = odd(torch.bfloat16, 1)
    assert equal(*both(api.quantize_block128, x))


@pytest.mark.parametrize("out_dtype", [api.OUT_BF16, api.OUT_FP32])
def test_product_into_a_view(out_dtype):
    x, w = odd(torch.bfloat16, 2)[1], torch.randn(515, WIDTH, device="cuda").bfloat16()
    ops = (*api.quantize_block128(x), *api.quantize_block128(w, api.AXIS_COLS, api.BLOCK_128X128))
    buf = torch.full((2, 519), 7.0, device="cuda").to(torch.bfloat16 if out_dtype == api.OUT_BF16 else torch.float32)
    api.gemm_block128(*ops, out_dtype=out_dtype, out=buf[:1, :515])
    api.check()
    want = torch.empty(1, 520, device="cuda", dtype=buf.dtype)
    api.gemm_block128(*ops, out_dtype=out_dtype, out=want[:, :515])
    assert torch.equal(buf[:1, :515], want[:, :515]) and (buf[0, 515:] == 7).all() and (buf[1] == 7).all()


@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
def test_residual_norm(stream):
    u, x, g = odd(torch.bfloat16, 3), odd(stream, 4), odd(torch.bfloat16, 5)
    w = torch.ones(WIDTH, device="cuda")
    assert equal(*both(lambda u, x, g: api.residual_norm_forward(u, x, w, w, g, api.GATE_SILU), u, x, g))
    dh, dy = odd(torch.bfloat16, 6), odd(stream, 7)
    assert equal(*both(lambda dh, dy, u, x, g: api.residual_norm_backward(dh, dy, u, x, w, w, g, api.GATE_SILU),
                       dh, dy, u, x, g))
    api.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_log_probabilities(dtype):
    x, t = odd(dtype, 8), torch.tensor([17], device="cuda")
    a, b = both(lambda x: api.logprobs_forward(x, t, 3), x)
    assert equal(a, b)
    d = torch.ones(1, device="cuda")
    assert equal(*both(lambda x: (api.logprobs_backward(x, t, a[2], a[1], d, d),), x))
    api.check()
