"""The oracle's activations where they are small, against sums with 60 digits (CPU only)."""
from decimal import Decimal, getcontext

import pytest
import torch

from oracle import feed_forward as ff

getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494")


def density(z):
    return (-z * z / 2).exp() / (2 * PI).sqrt()


def below(z):
    """The normal distribution function at z: 1/2 + density(z) (z + z^3 / 3 + z^5 / (3 5) + ...), which cancels 45 digits at most here."""
    total, term, k = Decimal(0), z, 1
    while abs(term) > Decimal(10) ** -58:
        total += term
        k += 2
        term = term * z * z / k
    return Decimal("0.5") + density(z) * total


def by_hand(name, z):
    """(value, slope)"""
    if name == "gelu":
        return z * below(z), below(z) + z * density(z)
    a, b = (Decimal(1), Decimal(0)) if name == "silu" else ((8 / PI).sqrt(), Decimal("0.044715"))
    p = 1 / (1 + (-a * (z + b * z ** 3)).exp())
    return z * p, p + z * p * (1 - p) * a * (1 + 3 * b * z * z)


@pytest.mark.parametrize("name", ["gelu", "gelu_tanh", "silu"])
def test_tails(name):
    """1e-13 of the value (2^-53 times the exponent, up to 100, and a few roundings); of the slope, which is a difference, of its larger term."""
    for z in (-9.0, -8.5, -7.0, -6.125, -5.0, -4.0, -3.0, -2.0, -1.0, -0.25, 0.5, 3.0, 9.0):
        value, slope = by_hand(name, Decimal(z))
        t = torch.tensor(z, dtype=torch.float64)
        assert abs(Decimal(float(ff.act(name, t))) - value) <= Decimal("1e-13") * abs(value), z
        assert abs(Decimal(float(ff.slope(name, t))) - slope) <= Decimal("1e-13") * max(abs(slope), abs(slope - value / Decimal(z))), z
