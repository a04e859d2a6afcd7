"""The activation functions out to their tails on the GPU, against 64 bits and the stated bounds."""
import math

import pytest
import torch

from paper_2609_33496_amd import cham

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
C = math.sqrt(2.0 / math.pi)


def _f(x, act):
    """(f(x), the exponent's argument) in 64 bits."""
    if act == "silu":
        w = -x
    elif act == "gelu":
        return 0.5 * x * torch.special.erfc(-x / math.sqrt(2.0)), x.square()
    else:
        w = -2.0 * C * (x + 0.044715 * x ** 3)
    return x / (1.0 + torch.exp(w)), w.abs()


@pytest.mark.parametrize("act,lo,hi", [("silu", -87.3, -60.0), ("silu", -20.0, 20.0), ("silu", 60.0, 200.0),
                                       ("gelu_tanh", -9.9, -8.0), ("gelu_tanh", -3.0, 3.0), ("gelu_tanh", 8.0, 200.0),
                                       ("gelu", -12.9, -9.0), ("gelu", -3.0, 3.0), ("gelu", 9.0, 200.0)])
def test_functions_within_their_bounds(act, lo, hi):
    """One element a block, brought to the size of 1 by the second factor: its scale is |y| / 448 in
    full precision, two roundings behind the function."""
    n = 4096
    print(f"[case] tails {act} {lo}..{hi}", flush=True)
    x = torch.zeros(n, 128)
    x[:, 5] = torch.linspace(lo, hi, n)
    y, arg = _f(x[:, 5].double(), act)
    u = torch.zeros_like(x)
    u[:, 5] = torch.exp2(torch.round(-torch.log2(y.abs().clamp(min=2.0 ** -126)))).float()
    y = (y * u[:, 5].double()).abs()
    q = cham.gated_quantize(x.to(DEV), u.to(DEV), getattr(cham, "ACT_" + act.upper()))
    s = q.scale.cpu().double()[0] * 448.0
    bound = 1e-6 + 4e-7 * arg + (1.2e-6 if act == "gelu" else 0.0) + 2 * U
    err = (s - y).abs() / y
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("act,lo,hi", [("silu", -200.0, -87.0), ("gelu_tanh", -20.0, -9.9), ("gelu", -20.0, -12.8)])
def test_values_below_the_least_ones_are_small_or_right(act, lo, hi):
    """Past the stated 2^-119: zero, or the value within the bound."""
    n = 4096
    print(f"[case] far tails {act} {lo}..{hi}", flush=True)
    x = torch.zeros(n, 128)
    x[:, 5] = torch.linspace(lo, hi, n)
    y, arg = _f(x[:, 5].double(), act)
    u = torch.full_like(x, 2.0 ** 100)
    q = cham.gated_quantize(x.to(DEV), u.to(DEV), getattr(cham, "ACT_" + act.upper()))
    got = q.scale.cpu().double()[0] * 448.0 * 2.0 ** -100
    got[q.scale.cpu()[0] == 2.0 ** -126] = 0.0  # the scale's floor: a block of zeros, or of less than it
    y = torch.where(y.abs() < 448.0 * 2.0 ** -226, 0.0, y.abs())
    err = (got - y).abs()
    assert bool(((err <= (4e-6 + 4e-7 * arg) * y) | (y <= 2.0 ** -119)).all())
    assert bool((got <= 2.0 ** -119 * 1.001).logical_or(y > 2.0 ** -119).all())
