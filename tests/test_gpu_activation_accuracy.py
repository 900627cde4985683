"""Activations where they are small: every bf16 pre-activation of a range, each result held to the formula's own error as csrc/activation.h states it, and
one rounding to bf16 (half a step, 2^-8 of the value)."""
import pytest
import torch

from oracle import feed_forward as ff

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


def mate_module():
    from paper_2109_04312_amd import mate
    return mate


def every_value(top):
    """All bf16 values with 2^-100 <= |z| <= top, padded with ones: [1, rows, 64]."""
    bits = (torch.arange(65536, dtype=torch.int32, device="cuda") << 16).view(torch.float32)
    z = bits[(bits.abs() >= 2.0 ** -100) & (bits.abs() <= top)]
    return torch.cat([z, z.new_ones(-len(z) % 64)]).to(torch.bfloat16).view(1, -1, 64)


def hold(got, want, formula, what):
    err, bound = (got.double() - want).abs(), formula + HALF * (want.abs() + formula)
    worst = (err / bound).flatten()
    print(f"   {what}: {float(worst.max()):.3f} x bound, at {float(want.flatten()[worst.argmax()]):.3e}", flush=True)
    assert bool((err <= bound).all()), what


# Of the value, in fp32.  gelu: 2^-10 of itself below 0, and nowhere more than 2.8e-7 (and the rounding of a positive value).  The others: the argument u of
# the exponential has two (silu) or three roundings and a rounded constant each, 2^-24 |u| each, and so has its power, in natural
# logarithms less; the hardware's 2^x and 1 / x are off by 2^-23 each, the sum and the product by 2^-24 each: (k |u| + 6) 2^-24 with k = 2 and 4.
def gelu_error(z, y):
    return torch.where(z < 0, torch.minimum(2.0 ** -10 * y.abs(), torch.tensor(2.8e-7, dtype=torch.float64, device=z.device)), 2.8e-7 + 2.0 ** -24 * y.abs())


def silu_error(z, y):
    return (2 * 1.4427 * z.abs() + 6) * 2.0 ** -24 * y.abs()


def gelu_tanh_error(z, y):
    return (4 * 1.4427 * (1.5958 * z.abs() + 0.07136 * z.abs() ** 3) + 6) * 2.0 ** -24 * y.abs()


# tanh = 2 p - 1 from 1/16 on: p, at most 1, is off by the same as silu's with k = 2 and |u| = 2.89 |z|, of which only e^-2|z| counts in p; twice that
# and one rounding.  Below: the first term left out, 17/315 z^7, and four roundings.
def tanh_error(z, y):
    large = 2 * ((2 * 2.8854 * z.abs() * torch.exp(-2 * z.abs()) + 6) * 2.0 ** -24) + 2.0 ** -24
    return torch.where(z.abs() < 0.0625, 0.054 * z.abs() ** 7 + 4 * 2.0 ** -24 * y.abs(), large)


@pytest.mark.parametrize("name,top,error", [("gelu", 9.0, gelu_error), ("silu", 60.0, silu_error), ("gelu_tanh", 9.0, gelu_tanh_error),
                                            ("tanh", 40.0, tanh_error)])
def test_values(name, top, error):
    """Through a product with the identity, whose results are the tokens' own values."""
    mate = mate_module()
    x = every_value(top)
    w = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    y, z = mate.linear(x, w, act=getattr(mate, "MATE_ACT_" + name.upper()), keep_z=mate.MATE_KEEP_BF16)
    assert torch.equal(z, x)
    want = ff.act(name, x.double())
    hold(y, want, error(x.double(), want), name)


def test_slope_of_gelu():
    """Off by 4.4e-7 below 0 and 5e-7 above, in fp32, whichever way z is kept."""
    mate = mate_module()
    z = every_value(30.0)
    for kept in (z, mate.checkpoint_pack(z)):
        at = z.double() if kept is z else ff.values(kept.codes, kept.scales)
        dz = mate.activation_bwd(torch.ones_like(z), kept, mate.MATE_ACT_GELU)
        hold(dz, ff.slope("gelu", at), torch.where(at < 0, 4.4e-7, 5e-7), "slope of gelu")
