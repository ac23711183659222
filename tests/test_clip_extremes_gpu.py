"""Clipping where the factor, or the norm with eps, leaves fp32's normal range: a result is still its exact value rounded, up to
the norm's error (5 * 2^-24) and the roundings of the factor (4 * 2^-24)."""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu

FACTOR = 9 * 2.0 ** -24


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value,max_norm,eps", [(2e37, 1e-2, 1e-6), (2e37, 1e-6, 1e-6), (1e37, 1.0, 1e-6), (3.2e37, 1e38, 3e38),
                                                (1.0, 1e-38, 1e-6), (1.0, 1e-44, 0.0), (1e-3, 1e-2, 1e38)])
def test_factors_below_the_normal_numbers(kind, value, max_norm, eps):
    gen = torch.Generator(device="cuda").manual_seed(0)
    t = (value * (0.5 + 0.5 * torch.rand(100, generator=gen, device="cuda"))).to(kind)
    limit, add = (torch.tensor(v).double().item() for v in (max_norm, eps))      # as fp32 arguments hold them
    want = t.double() * min(1.0, limit / (t.double().square().sum().sqrt().item() + add))
    for out_kind, step, least in ((torch.float32, 2.0 ** -24, 2.0 ** -150), (torch.bfloat16, 2.0 ** -8, 2.0 ** -134)):
        out = torch.empty(100, dtype=out_kind, device="cuda")
        api.clip_grads([t], max_norm, [out], eps)
        api.check()
        assert ((out.double() - want).abs() <= (step + FACTOR) * want.abs() + least * (1 + 2.0 ** -8)).all()
    copy = t.clone()
    api.clip_grads([copy], max_norm, eps=eps)
    api.check()
    step, least = (2.0 ** -24, 2.0 ** -150) if kind == torch.float32 else (2.0 ** -8, 2.0 ** -134)
    assert ((copy.double() - want).abs() <= (step + FACTOR) * want.abs() + least * (1 + 2.0 ** -8)).all()
