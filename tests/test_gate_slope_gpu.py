"""The slope of the sigmoid gate, element by element against 64 bits and relative to itself on both sides of the origin.

With h's gradient, the other projection and the gate's weight one (the identity, for the weight) the input's gradient is
dg = act'(g), rounded to bf16; the second rounding is of a value that is bf16 already.  Bound: half a step, and 2^-14 for an
exponential of up to 2 + 1.17 * 80 units in the last place, two products and a division.
"""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu

HALF, ACT = 2.0 ** -8, 2.0 ** -14


def test_slope_of_the_sigmoid_gate():
    """Relative to itself on both sides: s (1 - s) = e / (1 + e)^2 with e = exp(-|g|)."""
    g = torch.cat([torch.linspace(-80, 80, 160, device="cuda"), torch.linspace(8, 20, 96, device="cuda")]).bfloat16()
    gate = g[:, None].expand(256, 16).contiguous()
    eye, none = torch.eye(16, device="cuda").bfloat16(), torch.zeros(16, 16, dtype=torch.bfloat16, device="cuda")
    one = torch.ones_like(gate)
    dx, _, _ = api.gated_linear_backward(one, one, eye, none, (gate, one), api.GATE_SIGMOID)
    api.check()
    e = torch.exp(-g.double().abs())
    want = (e / (1 + e) ** 2)[:, None]
    bad = ~((dx.double() - want).abs() <= (HALF + ACT) * want)
    assert not bad.any(), [(v, r) for v, r in zip(g[bad.any(1)].tolist(), (dx.double() / want)[bad.any(1), 0].tolist())]
