"""Tiles of padding only, which skip the products, beside tiles that do not: the tokens of the others have the bits that they have without any padding, in
every form (the sum of a token goes by the sizes alone; tests/test_feed_forward_forms.py holds each size to its form), and padding is zeros whatever it held."""
import math

import pytest
import torch

from tests.test_gpu_feed_forward import PAD, Inputs

pytestmark = pytest.mark.gpu


def mate_module():
    from paper_2109_04312_amd import mate
    return mate


def some_sequences_only(B, N):
    """Flags: every other sequence is padding, and of the rest one has a last tile of padding, and one a first."""
    flags = torch.zeros(B, N, dtype=torch.uint8, device="cuda")
    flags[1::2] = PAD
    if B > 2 and N > 512:
        flags[0, N - 300:] = PAD
        flags[2, :260] = PAD
    return flags


def check(got, want, flags, what):
    pad = flags == PAD
    assert torch.equal(got[~pad], want[~pad]) and not bool(got[pad].any()), what


# of two groups and one, two stages and three, one launch for both gradients and two, whole contractions and split ones
FORWARD = [(6, 256, 2048, 264, "split 2"), (4, 64, 4104, 776, "split 4"), (6, 256, 40, 56, "tiles 64"), (6, 192, 144, 40, "tiles 64x2"),
           (6, 768, 328, 136, "tiles 64x2"), (12, 768, 328, 136, "tiles 128x2"), (6, 512, 40, 1160, "tiles 128"), (6, 768, 72, 2696, "tiles 256")]
BACKWARD = [(6, 64, 40, 136, "one launches, dw 128 ranges 1, dx 128x2"), (6, 64, 40, 4048, "one launches, dw 128 ranges 1, dx 64x2 split 4"),
            (6, 64, 40, 856, "one launches, dw 128 ranges 1, dx 64x2"), (6, 64, 40, 40, "two launches, dw 128 ranges 1, dx 64"),
            (6, 128, 3360, 40, "two launches, dw 128 ranges 1, dx 128"), (6, 768, 424, 1032, "one launches, dw 128 ranges 4, dx 128x2"),
            (4, 512, 13992, 72, "two launches, dw 128 ranges 2, dx 128"), (12, 768, 40, 352, "two launches, dw 128 ranges 9, dx 64x2")]


@pytest.mark.parametrize("B,N,E,F,form", FORWARD)
def test_linear(B, N, E, F, form):
    mate = mate_module()
    print(form, flush=True)
    i = Inputs(N, B, N, E, F, None)
    flags = some_sequences_only(B, N)
    kw = dict(act=mate.MATE_ACT_GELU, keep_z=mate.MATE_KEEP_8BIT, keep_y=True)
    want = mate.linear(i.x, i.w, i.bias, None, residual=i.res_y, **kw)
    i.x[flags == PAD], i.res_y[flags == PAD] = math.nan, math.inf
    for _ in range(3):
        got = mate.linear(i.x, i.w, i.bias, flags, residual=i.res_y, **kw)
        check(got[0], want[0], flags, "y")
        for k in (1, 2):
            check(got[k].codes, want[k].codes, flags, "codes")
            assert torch.equal(got[k].scales[flags != PAD], want[k].scales[flags != PAD]) and bool((got[k].scales[flags == PAD] == 1).all())


@pytest.mark.parametrize("B,N,E,F,form", BACKWARD)
def test_linear_bwd(B, N, E, F, form):
    mate = mate_module()
    print(form, flush=True)
    i = Inputs(N, B, N, E, F, None)
    flags = some_sequences_only(B, N)
    zeroed = torch.where((flags == PAD)[..., None], 0, i.dy)
    want = mate.linear_bwd(i.dy, i.x, i.w, None, z=i.z, act=mate.MATE_ACT_SILU, residual=i.res_x)[0]
    for t in (i.dy, i.x, i.z, i.res_x):
        t[flags == PAD] = math.nan
    for want_dw in (True, False):
        got = mate.linear_bwd(i.dy, i.x, i.w, flags, z=i.z, act=mate.MATE_ACT_SILU, residual=i.res_x, want_dw=want_dw, want_dbias=want_dw)
        check(got[0], want, flags, "dx")
    assert bool(torch.isfinite(mate.linear_bwd(zeroed, i.x, i.w, flags, z=i.z, act=mate.MATE_ACT_SILU)[1]).all())


@pytest.mark.parametrize("B,N,H", [(2, 64, 4), (6, 256, 12), (6, 768, 4), (6, 768, 16), (4, 2048, 16)])
def test_projections(B, N, H):
    mate = mate_module()
    E = 64 * H
    i = Inputs(N, B, N, E, 3 * E, None)
    live, flags = torch.zeros(B, N, dtype=torch.uint8, device="cuda"), some_sequences_only(B, N)
    w_o, dy = i.normal(E, E, scale=E ** -0.5), i.normal(B, N, E)
    by_token = lambda t: t.transpose(1, 2)
    want = [mate.qkv_project(i.x, i.w, i.bias, live, H), mate.out_project(i.x.view(B, H, N, 64), w_o, None, live)]
    x = i.x.clone()
    x[flags == PAD] = math.nan
    o = i.x.view(B, H, N, 64).clone()
    by_token(o)[flags == PAD] = math.nan
    for t, u in zip(mate.qkv_project(x, i.w, i.bias, flags, H), want[0]):
        check(by_token(t), by_token(u), flags, "q, k, v")
    check(mate.out_project(o, w_o, None, flags), want[1], flags, "y")
    d = [i.normal(B, H, N, 64) for _ in range(3)]
    want = mate.qkv_project_bwd(i.x, i.w, live, *d)[0], mate.out_project_bwd(i.x.view(B, H, N, 64), w_o, live, dy)[0]
    dy[flags == PAD] = math.nan
    for t in d:
        by_token(t)[flags == PAD] = math.nan
    check(mate.qkv_project_bwd(x, i.w, flags, *d)[0], want[0], flags, "dx")
    check(by_token(mate.out_project_bwd(o, w_o, flags, dy)[0]), by_token(want[1]), flags, "d_o")
