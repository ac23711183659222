"""Vectors and scales of another size than the operands have are refused, not read in part."""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu

vec = lambda n: torch.ones(n, device="cuda")


def refused(call, *args, **kw):
    with pytest.raises(ValueError):
        call(*args, **kw)


@pytest.mark.parametrize("n", [63, 65, 128])
def test_residual_norm_vectors(n):
    u = torch.ones(4, 64, device="cuda", dtype=torch.bfloat16)
    for kw in ({"w_post": vec(n)}, {"w_pre": vec(n)}, {"gate": vec(n)}):
        refused(api.residual_norm_forward, u, u, **kw)
        refused(api.residual_norm_backward, u if "w_pre" in kw else None, u, u, u, **kw)


@pytest.mark.parametrize("n", [3, 5, 8])
def test_log_probability_vectors(n):
    x, t = torch.zeros(4, 10, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    bad_t = torch.zeros(n, dtype=torch.int64, device="cuda")
    refused(api.logprobs_forward, x, bad_t)
    refused(api.logprobs_backward, x, bad_t, vec(4), vec(4), vec(4))
    for i in range(4):
        rows = [vec(n if i == j else 4) for j in range(4)]
        refused(api.logprobs_backward, x, t, *rows)


def test_product_operands():
    x, w = (torch.ones(n, 256, device="cuda", dtype=torch.bfloat16) for n in (300, 264))
    a = api.quantize_block128(x)
    row, square = (api.quantize_block128(w, api.AXIS_COLS, s) for s in (api.BLOCK_1X128, api.BLOCK_128X128))
    refused(api.gemm_block128, *a, *row, api.BLOCK_128X128)          # scales of the other block shape
    refused(api.gemm_block128, *a, *square, api.BLOCK_1X128)
    refused(api.gemm_block128, *a, square[0], api.quantize_block128(torch.cat([w, w]), api.AXIS_COLS, api.BLOCK_128X128)[1])
    refused(api.gemm_block128, a[0][:100], a[1], *square)            # the scales' pitch is of 300 rows
    out = api.gemm_block128(*a, *square)
    api.check()
    assert (out == 256).all()


def test_flat_scale_buffers_may_be_larger():
    x = torch.ones(40, 256, device="cuda", dtype=torch.bfloat16)
    flat = torch.full((5000,), float("nan"), device="cuda")
    codes, scales = api.quantize_block128(x, scales=flat)
    out = api.gemm_block128(codes, scales, *api.quantize_block128(x, api.AXIS_COLS, api.BLOCK_128X128))
    api.check()
    assert scales is flat and (out == 256).all()


def test_linear_pass_takes_matrices_only():
    x, w = (torch.ones(n, 32, device="cuda", dtype=torch.bfloat16) for n in (16, 48))
    refused(api.linear_pass_block128, api.PASS_FPROP, x.reshape(8, 32, 2), w)
    refused(api.linear_pass_block128, api.PASS_FPROP, x, w.reshape(24, 32, 2))
