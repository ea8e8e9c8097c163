"""The activations far below zero, where little of z is left: relative to that little, not to z.

Tolerances.  The factor beside z is an exponential 2^-x (or 1 / (1 + 2^x)) times what changes slowly: 2^-19 for a polynomial of 2e-7, the exponential's and the
reciprocal's own error and a dozen roundings of 2^-24, and ln 2 x times the relative error of x: GELU's x = a^2 log2(e) / 2 has two roundings and half of one in its
constant, the tanh form's four and a half (the square, the product inside, its constants, the last product), SiLU's one and a half.  Values stay
above 1e-37, so that none is rounded to a step of the smallest numbers.
"""
import math

import pytest

import paper_2003_10735_amd as st

from test_gpu_linear import ACTS, C0, EPS

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LOG2E = 1.0 / math.log(2.0)
TAILS = {"gelu": (12.4, 2.5, lambda a: a * a / 2 * LOG2E), "gelu_tanh": (9.6, 4.5, lambda a: 2 * C0 * (a + 0.044715 * a ** 3) * LOG2E), "silu": (80.0, 1.5, lambda a: a * LOG2E)}


@pytest.mark.parametrize("act", list(TAILS))
def test_the_lower_tail_keeps_relative_accuracy(act):
    far, roundings, x_of = TAILS[act]
    z = -torch.linspace(0.01, far, 20001, device="cuda")[:, None]
    y = st.st_linear(z, torch.ones(1, 1, device="cuda"), activation=ACTS[act])[:, 0].double()
    a = -z[:, 0].double()
    # (the distribution function by its logarithm: 1 + erf would lose what is asked about)
    factor = torch.exp(torch.special.log_ndtr(-a)) if act == "gelu" else 1 / (1 + torch.exp(x_of(a) / LOG2E))
    want = -a * factor
    tolerance = 2.0 ** -19 + math.log(2.0) * roundings * EPS * x_of(a)
    assert float(want.abs().min()) > 1e-37 and ((y - want).abs() <= tolerance * want.abs()).all()
