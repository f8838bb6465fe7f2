"""fp32's activations relative to the result, on the negative side too, where little of the argument is left."""
import math

import pytest
import torch

from layer_util import F32, Plan, check
from paper_2503_22796_amd import binding as B

pytestmark = pytest.mark.gpu

SMALLEST = 2.0 ** -149                            # fp32's smallest step


def run(v, act):
    v = v.reshape(-1, 1).cuda()
    out = torch.full_like(v, float("nan"))
    with Plan(dtype=torch.float32) as plan:
        B.difa_linear(plan, v, torch.ones(1, 1, device="cuda"), out, activation=act)
    return out.cpu().view(-1)


def values():
    near = torch.cat([torch.linspace(-110, 40, 40_009), torch.linspace(-12, 12, 40_009), torch.linspace(-0.01, 0.01, 1001)])
    return torch.cat([near, torch.tensor([0.0, 1e-30, -1e-30, 1e4, -1e4, 1e20, -1e20, 3e38, -3e38])])


def below(v):
    """Where the exponential has lost its bits it is off by a smallest step, or two with a correction, times v; and so are four more."""
    return (2 * v.double().abs().clamp(max=110) + 4) * SMALLEST


def logistic(z):
    """1 / (1 + exp(-z)) in 64 bits, as exact for z far below zero."""
    e = torch.exp(-z.abs())
    return torch.where(z < 0, e, torch.ones_like(e)) / (1 + e)


def test_silu():
    v = values()
    ref = v.double() * logistic(v.double())
    # The exponential within two half steps (one unit), met in the numerator and, at most half of it, in the denominator: three;
    # the denominator's sum, the product and the quotient: three more.
    check(run(v, B.DIFA_ACT_SILU), ref, 6.1 * F32 * ref.abs() + below(v), "silu")


def test_gelu_tanh():
    v = values()
    y = v.double().clamp(-1e6, 1e6)               # 0.5 y (1 + tanh u) = y / (1 + exp(-2 u)); beyond: the limits
    ref = v.double() * logistic(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))
    # as above, and the exponential's correction by what rounding its argument left: one half step more, one in the denominator
    check(run(v, B.DIFA_ACT_GELU_TANH), ref, 8.1 * F32 * ref.abs() + below(v), "gelu_tanh")


@pytest.mark.parametrize("act", [B.DIFA_ACT_SILU, B.DIFA_ACT_GELU_TANH])
def test_what_is_not_finite(act):
    """The definitions' own values: v times 1 and v times 0."""
    got = run(torch.tensor([float("inf"), float("-inf"), float("nan")]), act)
    assert got[0] == float("inf") and torch.isnan(got[1:]).all()
