"""Values of the gates where their exponentials are small, element by element against 64 bits.

With x's rows (g, 1, 0 ..), the gate's weight rows (1, 0, ..) and the other one's (0, 1, ..) every element of a row of h is
act(g).  Bounds: a rounding to bf16, 2^-14 of the value for an exponential of up to 2 + 1.17 * 103 units in the last
place, its argument and a division; below bf16's normal numbers half of its smallest step, 2^-134.
"""
import math

import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu

HALF, ACT, TINY = 2.0 ** -8, 2.0 ** -14, 2.0 ** -134


def values(T):
    g = torch.linspace(-100, 88, 3 * 300, device="cuda")
    g = torch.cat([g, torch.linspace(-13.5, 13.5, 300, device="cuda")]).bfloat16()
    return [g[i: i + T] for i in range(0, len(g) - T + 1, T)]


def sigmoid(g):
    return torch.where(g >= 0, 1 / (1 + torch.exp(-g.abs())), torch.exp(-g.abs()) / (1 + torch.exp(-g.abs())))


VALUES = {
    api.GATE_SIGMOID: sigmoid,
    api.GATE_SILU: lambda g: g * sigmoid(g),
    api.GATE_GELU_TANH: lambda g: g * sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)),
}


@pytest.mark.parametrize("which", VALUES)
@pytest.mark.parametrize("T", [8, 60, 300])              # a kernel each
def test_values(which, T):
    wg, wu = (torch.zeros(16, 16, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wg[:, 0], wu[:, 1] = 1, 1
    for g in values(T):
        x = torch.zeros(T, 16, dtype=torch.bfloat16, device="cuda")
        x[:, 0], x[:, 1] = g, 1
        h, (gate, up) = api.gated_linear_forward(x, wg, wu, which)
        api.check()
        assert torch.equal(gate, g[:, None].expand(T, 16)) and (up == 1).all()
        want = VALUES[which](g.double())[:, None]
        # the tanh form's exponent is a sum of rounded terms: 4 * 2^-24 of up to 103
        bad = ~((h.double() - want).abs() <= (HALF + ACT) * want.abs() + TINY * (1 + want.abs()))
        assert not bad.any(), g[bad.any(1)].tolist()
