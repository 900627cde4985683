"""Pins for the oracle of the feed-forward half (CPU only)."""
import math

import pytest
import torch

from oracle import feed_forward as ff


def _normal(*shape, seed=0):
    return torch.randn(*shape, dtype=torch.float64, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("name", ff.ACTS)
def test_slope_is_the_derivative(name):
    z = torch.cat([torch.linspace(-9, 9, 2001, dtype=torch.float64) + 1e-3, torch.tensor([1e-4, -1e-4, 40.0, -40.0], dtype=torch.float64)])
    h = 1e-5
    # central differences: h^2 / 6 times a third derivative below 10, and 2^-53 |act| / h of rounding
    want = (ff.act(name, z + h) - ff.act(name, z - h)) / (2 * h)
    assert bool(((ff.slope(name, z) - want).abs() <= 10 * h * h / 6 + 4e-11 * (1 + z.abs())).all())


def test_activations_at_known_points():
    one = torch.ones((), dtype=torch.float64)
    assert abs(float(ff.act("gelu", one)) - 0.8413447460685429) < 1e-14        # 1 standard deviation
    assert abs(float(ff.act("silu", one)) - 1 / (1 + math.exp(-1))) < 1e-15
    assert abs(float(ff.act("tanh", one)) - math.tanh(1)) < 1e-15
    assert abs(float(ff.act("gelu_tanh", one)) - 0.5 * (1 + math.tanh(math.sqrt(2 / math.pi) * 1.044715))) < 1e-15
    assert float(ff.act("relu", -one)) == 0 and float(ff.act("relu", one)) == 1


def test_linear_as_loops():
    B, N, E, F = 2, 3, 5, 4
    x, w, bias, res = _normal(B, N, E), _normal(F, E, seed=1), _normal(F, seed=2), _normal(B, N, F, seed=3)
    flags = torch.tensor([[0, 1, 2], [2, 0, 0]], dtype=torch.uint8)
    z, y = ff.linear(x, w, bias, flags, "tanh", res)
    for b in range(B):
        for n in range(N):
            for f in range(F):
                want = sum(float(w[f, e] * x[b, n, e]) for e in range(E)) + float(bias[f])
                pad = flags[b, n] == 2
                assert abs(float(z[b, n, f]) - (0 if pad else want)) < 1e-12
                assert abs(float(y[b, n, f]) - (0 if pad else math.tanh(want) + float(res[b, n, f]))) < 1e-12


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_gradients_against_differences(name):
    """y = act(z) w^T + b, z itself reached by a residual gradient: every gradient against central differences."""
    B, N, E, F = 2, 3, 4, 5
    z, w, b = _normal(B, N, E), _normal(F, E, seed=1), _normal(F, seed=2)
    dy, res = _normal(B, N, F, seed=3), _normal(B, N, E, seed=4)
    flags = torch.tensor([[0, 2, 1], [0, 0, 2]], dtype=torch.uint8)

    def loss(z, w, b):
        return float((ff.linear(ff.act(name, z), w, b, flags)[1] * dy).sum() + (ff.zero_pads(z, flags) * res).sum())

    got = ff.linear_backward(dy, ff.act(name, z), w, flags, z, name, res)
    for which, (v, g) in enumerate(zip((z, w, b), got)):
        for i in range(v.numel()):
            h = torch.zeros_like(v).view(-1)
            h[i] = 1e-5
            h = h.view(v.shape)
            args = [[z, w, b], [z, w, b]]
            args[0][which], args[1][which] = v + h, v - h
            assert abs((loss(*args[0]) - loss(*args[1])) / 2e-5 - float(g.reshape(-1)[i])) < 1e-8


def test_code_values_are_those_of_the_type():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    v = ff.code_values()
    assert torch.equal(torch.isnan(t), torch.isnan(v)) and torch.equal(t[~torch.isnan(t)], v[~torch.isnan(v)])


def test_kept_by_brute_force():
    """The smallest scale that does not saturate, and the nearest of all codes (ties: even mantissa)."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn(40, 1, 70, dtype=torch.float64, generator=g) * 2.0 ** torch.randint(-20, 20, (40, 1, 1), generator=g)
    x[0, 0, :32] = 0
    x[1, 0, 3] = 448.0                                                        # exactly representable ends of the range
    x[2, 0, 40:45] = torch.tensor([1.0, 1.0625, 1.1875, -1.3125, 448 * 2.0 ** -3])   # ties
    codes, scales = ff.kept(x)
    assert codes.shape == (40, 1, 70) and scales.shape == (40, 1, 3)
    table = ff.code_values()[:127]
    for t in range(40):
        for k in range(3):
            block, s = x[t, 0, 32 * k:32 * k + 32], int(scales[t, 0, k]) - 127
            most = float(block.abs().max())
            assert most <= 448 * 2.0 ** s and (s == -126 or most > 448 * 2.0 ** (s - 1))
            for v, c in zip(block.tolist(), codes[t, 0, 32 * k:32 * k + 32].tolist()):
                d = (table - abs(v) * 2.0 ** -s).abs()
                near = (d == d.min()).nonzero()[:, 0].tolist()
                assert c & 127 in near and (len(near) == 1 or c % 2 == 0) and (c >> 7 == int(math.copysign(1, v) < 0))
    back = ff.values(codes, scales)
    assert bool(((back - x).abs() <= torch.maximum(x.abs() / 16, torch.repeat_interleave(2.0 ** (scales.double() - 137), 32, -1)[..., :70])).all())


def test_kept_keeps_what_is_not_finite_apart():
    x = torch.tensor([[[1.0, math.inf, -math.inf, math.nan, -2.0, 0.0, 0.5, 3.0]]], dtype=torch.float64)
    codes, scales = ff.kept(x)
    back = ff.values(codes, scales)[0, 0]
    assert torch.isnan(back[1:4]).all() and torch.equal(back[[0, 4, 5, 6, 7]], x[0, 0, [0, 4, 5, 6, 7]])
    assert int(scales) == 127 - 7                                              # of 3.0: 448 / 2^7 = 3.5
    codes, scales = ff.kept(x, torch.tensor([[2]], dtype=torch.uint8))
    assert int(codes.sum()) == 0 and int(scales) == 1
