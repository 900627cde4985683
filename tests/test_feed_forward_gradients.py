"""Where the gradient that linear_bwd adds to dx comes in: against automatic differentiation of the layer, in 64 bits."""
import os
import re

import pytest
import torch
import torch.nn.functional as F

from oracle import feed_forward as ff
from paper_2109_04312_amd import mate

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ACT = dict(none=lambda z: z, relu=torch.relu, gelu=F.gelu, gelu_tanh=lambda z: F.gelu(z, approximate="tanh"), silu=F.silu, tanh=torch.tanh)
BF16, F32_STEP = 2.0 ** -8, 2.0 ** -24


def gradient_at_z(name, z, w, dy, r, reaches):
    """Of <dy, act(z) w^T> + <r, z> or <r, act(z)>, by torch."""
    z = z.double().detach().clone().requires_grad_()
    x = ACT[name](z)
    ((x @ w.double().T * dy.double()).sum() + ((z if reaches == "z" else x) * r.double()).sum()).backward()
    return z.grad


def draw(seed, device, dtype, B=2, N=37, E=40, width=24):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64).to(dtype).to(device)
    return normal(B, N, E) * 2, normal(width, E), normal(B, N, width), normal(B, N, E) * 2


@pytest.mark.parametrize("name", ff.ACTS)
def test_the_formula(name):
    """The added gradient is one that reached z; one that reached act(z) takes the activation's own backward first."""
    z, w, dy, r = draw(1, "cpu", torch.float64)
    x = ff.act(name, z)
    added = lambda r: ff.linear_backward(dy, x, w, None, z, name, r)[0]
    assert float((added(r) - gradient_at_z(name, z, w, dy, r, "z")).abs().max()) < 1e-12
    want = gradient_at_z(name, z, w, dy, r, "x")
    assert float((added(ff.activation_backward(r, z, name)) - want).abs().max()) < 1e-12
    assert name == "none" or float((added(r) - want).abs().max()) > 0.1   # they are not the same


def test_the_text_says_so():
    """Header and docstring name the gradient that the formula adds."""
    header = open(os.path.join(ROOT, "include", "mate.h")).read()
    of_backward = header[header.index(" * mate_linear_bwd:  with G = dy"):header.index(" * mate_activation_bwd:")]
    entry = re.search(r" \*   residual  (.*?)\n \*   \w", of_backward, re.S)[1]
    for text in (entry, mate.linear_bwd.__doc__):
        assert re.search(r"reached\s+z\s+on\s+another\s+way", text) and not re.search(r"reached\s+x\s+on", text), text
        assert "activation_bwd" in text


@pytest.mark.gpu
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("name", ff.ACTS)
def test_both_ways(name, eight):
    """A layer whose activation has a second reader, and one whose pre-activation has: the calls that the documentation names."""
    z, w, dy, r = draw(2, "cuda", torch.bfloat16, 3, 70, 136, 200)
    act = getattr(mate, "MATE_ACT_" + name.upper())
    kept, zv = (mate.checkpoint_pack(z), None) if eight else (z, z.double())
    if zv is None:
        zv = ff.values(kept.codes, kept.scales)
    x = ff.act(name, zv).to(torch.bfloat16)
    raw = dy.double().abs() @ w.double().abs()
    # fp32 sum of `width` products, twice their roundings; the slope's formula, 2^-20 (1 + |z|) of what it is multiplied with; one rounding
    # of the result, and of the gradient that activation_bwd gives
    slope_error = 0.0 if name == "none" else 2.0 ** -20 * (1 + zv.abs())
    slope = ff.slope(name, zv).abs()
    for reaches in ("z", "x"):
        other, extra = r, 0.0
        if reaches == "x" and name != "none":
            other = mate.activation_bwd(r, kept, act)
            extra = BF16 * slope * r.double().abs() + (1 + BF16) * slope_error * r.double().abs()
        dx, _, _ = mate.linear_bwd(dy, x, w, None, z=None if name == "none" else kept, act=act, residual=other)
        want = gradient_at_z(name, zv, w, dy, r, reaches)
        e = (slope + slope_error) * 2 * w.shape[0] * F32_STEP * raw + slope_error * raw + extra + F32_STEP * (want.abs() + extra)
        bound = e + BF16 * (want.abs() + e) + 1e-300
        err = (dx.double() - want).abs()
        print(f"   {name} {reaches}: {float((err / bound).max()):.2f} x bound", flush=True)
        assert bool((err <= bound).all())
