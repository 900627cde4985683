"""Float64 oracle of the feed-forward half: products with an epilogue, their gradients, 8-bit activations.

Elementary torch operations in 64 bits on whatever device the inputs are on; shares no code with the
library.  Token tensors are [B, N, width], flags [B, N] uint8 with 2 (or more) for padding, or None.
Pins: tests/test_oracle_feed_forward.py (loops, central differences, brute force over all codes).
"""
from __future__ import annotations

import math

import torch

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu", "tanh")
BLOCK, LARGEST = 32, 448.0
SCORE = math.sqrt(2 / math.pi)


def live(flags, like):
    """[B, N, 1]: is the token not padding?"""
    if flags is None:
        return torch.ones(*like.shape[:2], 1, dtype=torch.bool, device=like.device)
    return (flags < 2)[..., None]


def zero_pads(x, flags):
    return torch.where(live(flags, x), x, torch.zeros((), dtype=x.dtype, device=x.device))


def act(name, z):
    if name == "none":
        return z
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return z * torch.sigmoid(2 * SCORE * (z + 0.044715 * z ** 3))     # (1 + tanh u = 2 sigmoid(2 u), which does not cancel below 0)
    if name == "silu":
        return z * torch.sigmoid(z)
    assert name == "tanh"
    return torch.tanh(z)


def slope(name, z):
    """Derivative of act (0 at 0 for relu)."""
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        u = 2 * SCORE * (z + 0.044715 * z ** 3)
        return torch.sigmoid(u) + z * torch.sigmoid(u) * torch.sigmoid(-u) * 2 * SCORE * (1 + 3 * 0.044715 * z ** 2)
    if name == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * torch.sigmoid(-z))
    assert name == "tanh"
    return torch.cosh(z.clamp(-300, 300)) ** -2


def linear(x, w, bias=None, flags=None, name="none", residual=None):
    """(z, y), rows of padding zero in both."""
    z = x.double() @ w.double().T
    if bias is not None:
        z = z + bias.double()
    y = act(name, z)
    if residual is not None:
        y = y + residual.double()
    return zero_pads(z, flags), zero_pads(y, flags)


def linear_backward(dy, x, w, flags=None, z=None, name="none", residual=None):
    """(dx, dw, dbias) of sum(y dy) for y = x w^T + bias with x = act(z); dx is the gradient at z, plus `residual`."""
    g = zero_pads(dy.double(), flags)
    dx = g @ w.double()
    if z is not None:
        dx = dx * slope(name, z.double())
    if residual is not None:
        dx = dx + residual.double()
    flat = g.reshape(-1, g.shape[-1])
    dw = flat.T @ zero_pads(x.double(), flags).reshape(-1, x.shape[-1])
    return zero_pads(dx, flags), dw, flat.sum(0)


def activation_backward(dy, z, name, flags=None):
    return zero_pads(dy.double() * slope(name, z.double()), flags)


# ---- 8 bits -------------------------------------------------------------------------------------
def code_values(device="cpu"):
    """What the 256 e4m3 codes stand for at scale 1: sign, exponent - 7, three mantissa bits; the last of each sign is NaN."""
    half = [(1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6 for e in range(16) for m in range(8)]
    half[127] = math.nan
    return torch.tensor(half + [-v for v in half], dtype=torch.float64, device=device)


def power(e):
    """2^e in 64 bits (exp2 is exact on a GPU too, unlike torch.ldexp and powers of 2)."""
    return torch.exp2(e.double())


def blocks_of(x):
    pad = -x.shape[-1] % BLOCK
    return torch.cat([x, x.new_zeros(*x.shape[:-1], pad)], -1).unflatten(-1, (-1, BLOCK))


def kept(x, flags=None):
    """(codes, scales): scale s of a block is the smallest in 1 .. 254 with its largest finite magnitude <= 448 2^(s - 127);
    codes are the nearest, ties to the even one, but none for a magnitude of 2^128, which fp32 cannot hold; not finite -> NaN with
    the value's sign (infinities) or any (NaN)."""
    x = zero_pads(x.double(), flags)
    x = torch.where(torch.isfinite(x), x.clamp(-240 * 2.0 ** 120, 240 * 2.0 ** 120), x)
    blocks = blocks_of(x)
    finite = torch.isfinite(blocks)
    most = torch.where(finite, blocks, 0.0).abs().amax(-1)
    m, e = torch.frexp(most / LARGEST)                      # m in [0.5, 1): a power of two itself is m = 0.5
    s = torch.where(most > 0, e - (m == 0.5).int() + 127, 1).clamp(1, 254)
    u = torch.where(finite, blocks, 0.0) * power(127 - s)[..., None]
    step = power(torch.frexp(u.abs().clamp_min(2.0 ** -6))[1] - 1 - 3)
    r = torch.round(u / step) * step                        # (round: halves to even)
    order = torch.argsort(code_values(x.device)[:127])
    code = torch.searchsorted(code_values(x.device)[:127][order].contiguous(), r.abs().contiguous())
    code = order[code] + 128 * torch.signbit(blocks).long()
    code = torch.where(finite, code, 127 + 128 * torch.signbit(blocks).long())
    return code.flatten(-2)[..., :x.shape[-1]].to(torch.uint8), s.to(torch.uint8)


def values(codes, scales):
    v = code_values(codes.device)[codes.long()]
    s = torch.repeat_interleave(scales.long() - 127, BLOCK, -1)[..., :codes.shape[-1]]
    return v * power(s)
