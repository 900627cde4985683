"""GPU parity of the feed-forward half (products with an epilogue, their gradients, 8-bit activations) against the
float64 oracle, through the tensor-level calls."""
import math

import pytest
import torch

from oracle import feed_forward as ff

pytestmark = pytest.mark.gpu
BF16, F32_STEP = 2.0 ** -8, 2.0 ** -24      # half a step of each type, relative
PAD = 2


def mate_module():
    from paper_2109_04312_amd import mate
    return mate


def code_of(name):
    return getattr(mate_module(), "MATE_ACT_" + name.upper())


class Inputs:
    """Seeded tensors of one product; padding: none (None), a tail of each sequence, scattered, or everything."""

    def __init__(self, seed, B, N, E, F, padding="tail"):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.normal = lambda *shape, scale=1.0, dtype=torch.bfloat16: (torch.randn(shape, device="cuda", generator=gen) * scale).to(dtype)
        self.x, self.w = self.normal(B, N, E), self.normal(F, E, scale=E ** -0.5)
        self.bias = self.normal(F, dtype=torch.float32)
        self.dy, self.res_y, self.res_x = self.normal(B, N, F), self.normal(B, N, F), self.normal(B, N, E)
        self.z = self.normal(B, N, E, scale=2.0)
        flags = torch.randint(0, 2, (B, N), device="cuda", generator=gen).to(torch.uint8)
        if padding == "tail":
            for b in range(B):
                flags[b, N - (b * N) // (B + 1):] = PAD
        elif padding == "scattered":
            flags[torch.rand(B, N, device="cuda", generator=gen) < 0.3] = PAD
        elif padding == "all":
            flags[:] = PAD
        self.flags = None if padding is None else flags


def within(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, what
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    err = (got - want).abs()
    worst = float((err / bound).max()) if err.numel() else 0.0
    print(f"   {what}: max-abs {float(err.max()):.2e}, {worst:.2f} x bound", flush=True)
    assert worst <= 1.0, what


def sum_error(terms, absolute):
    """An fp32 sum of exact products of bf16 values, in any order: each of its `terms` additions rounds by at most 2^-24 of a partial
    sum, which sum |terms| bounds.  Twice that, as the matrix instructions' own additions are not documented to round to nearest."""
    return 2 * terms * F32_STEP * absolute


def pre_activation_error(i):
    """Of z = x w^T + bias in fp32."""
    return sum_error(i.x.shape[-1] + 1, i.x.double().abs() @ i.w.double().abs().T + i.bias.double().abs())


# An activation's slope is below 1.13, which the error of z is multiplied with; its own formula is off by 1.5e-7 (gelu) or a few
# roundings of the hardware's 2^x and 1 / x (2^-22 relative each), of a value of at most |z| + 1: 2^-20 (1 + |z|).
def activation_error(z, ez):
    return 1.13 * ez + 2.0 ** -20 * (1 + z.abs())


def close_8bit(checkpoint, want, error, what):
    """Codes off by half a step, 2^-4 of a value or 2^-10 of its scale, on top of the error of what was rounded; and scales that are the
    smallest without saturation, but for a largest value within that error of the border."""
    mate = mate_module()
    assert checkpoint.codes.dtype == checkpoint.scales.dtype == torch.uint8
    got = mate.checkpoint_unpack(checkpoint, torch.float32).double()
    scale = ff.power(checkpoint.scales.long() - 127)
    each = torch.repeat_interleave(scale, 32, -1)[..., :want.shape[-1]]
    within(got, want, error + torch.maximum((want.abs() + error) / 16, each / 1024) + 1e-300, what)
    most, slack = ff.blocks_of(want.abs()).amax(-1), ff.blocks_of(error.expand_as(want)).amax(-1)
    assert bool((most - slack <= 448 * scale).all()), what
    assert bool(((checkpoint.scales == 1) | (most + slack > 224 * scale)).all()), what


def check_forward(seed, B, N, E, F, act="gelu", padding="tail", bias=True, residual=True, keep_z=2, keep_y=True):
    mate = mate_module()
    print(f"linear B={B} N={N} E={E} F={F} {act} padding={padding} bias={bias} residual={residual} z={keep_z} y8={keep_y}", flush=True)
    i = Inputs(seed, B, N, E, F, padding)
    if not bias:
        i.bias.zero_()
    y0 = torch.full((B, N, F), float("nan"), dtype=torch.bfloat16, device="cuda")
    got = mate.linear(i.x, i.w, i.bias if bias else None, i.flags, act=code_of(act), residual=i.res_y if residual else None, keep_z=keep_z,
                      keep_y=keep_y, y=y0)
    torch.cuda.synchronize()
    assert got[0] is y0 or got[0].data_ptr() == y0.data_ptr()
    z, y = ff.linear(i.x, i.w, i.bias, i.flags, act, i.res_y if residual else None)
    ez = torch.where(ff.live(i.flags, z), pre_activation_error(i), 0.0)
    raw = i.x.double() @ i.w.double().T + i.bias.double()
    ey = torch.where(ff.live(i.flags, z), activation_error(raw, ez) + F32_STEP * y.abs(), 0.0)
    within(got[0], y, ey + BF16 * (y.abs() + ey) + 1e-300, "y")
    if keep_z == mate.MATE_KEEP_BF16:
        within(got[1], z, ez + BF16 * (z.abs() + ez) + 1e-300, "z")
    elif keep_z == mate.MATE_KEEP_8BIT:
        close_8bit(got[1], z, ez, "z in 8 bits")
    else:
        assert got[1] is None
    if keep_y:
        close_8bit(got[2], y, ey, "y in 8 bits")
    else:
        assert len(got) == 2
    return got


def check_backward(seed, B, N, E, F, act="gelu", padding="tail", residual=True, x8=True, z8=True):
    mate = mate_module()
    print(f"linear_bwd B={B} N={N} E={E} F={F} {act} padding={padding} residual={residual} x8={x8} z8={z8}", flush=True)
    i = Inputs(seed, B, N, E, F, padding)
    x = mate.checkpoint_pack(i.x) if x8 else i.x
    z = None if act == "none" else mate.checkpoint_pack(i.z) if z8 else i.z
    xv = ff.values(x.codes, x.scales) if x8 else i.x
    zv = None if z is None else ff.values(z.codes, z.scales) if z8 else i.z
    dx, dw, db = mate.linear_bwd(i.dy, x, i.w, i.flags, z=z, act=code_of(act), residual=i.res_x if residual else None)
    torch.cuda.synchronize()
    wx, ww, wb = ff.linear_backward(i.dy, xv, i.w, i.flags, zv, act, i.res_x if residual else None)
    g = ff.zero_pads(i.dy.double().abs(), i.flags)
    raw = g @ i.w.double().abs()                     # bounds |dy w|, which the slope's error (2^-20 (1 + |z|), as above) is multiplied with
    s = 1.0 if zv is None else ff.slope(act, zv.double()).abs()
    es = 0.0 if zv is None else 2.0 ** -20 * (1 + zv.double().abs())
    ex = torch.where(ff.live(i.flags, wx), (s + es) * sum_error(F, raw) + es * raw + F32_STEP * wx.abs(), 0.0)
    within(dx, wx, ex + BF16 * (wx.abs() + ex) + 1e-300, "dx")
    flat = g.reshape(-1, F)
    within(dw, ww, sum_error(B * N, flat.T @ ff.zero_pads(xv.double().abs(), i.flags).reshape(-1, E)) + 1e-300, "dw")
    within(db, wb, sum_error(B * N, flat.sum(0)) + 1e-300, "dbias")
    return dx, dw, db


# widths beside multiples of 8, 32 (a scale), 64 (a stage) and the tiles; tokens from one on
@pytest.mark.parametrize("E,F", [(8, 8), (64, 64), (72, 40), (120, 136), (200, 520), (1032, 24), (768, 768)])
@pytest.mark.parametrize("B,N", [(1, 1), (2, 7), (3, 65), (1, 200)])
def test_widths_and_lengths(B, N, E, F):
    check_forward(E + N, B, N, E, F)
    check_backward(E + N, B, N, E, F)


@pytest.mark.parametrize("act", ff.ACTS)
@pytest.mark.parametrize("keep_z", [0, 1, 2])
def test_activations(act, keep_z):
    check_forward(1, 3, 130, 136, 264, act, bias=keep_z != 1, residual=keep_z != 2, keep_z=keep_z, keep_y=keep_z != 0)
    check_backward(2, 3, 130, 136, 264, act, residual=keep_z != 2, x8=keep_z != 1, z8=keep_z == 2)


@pytest.mark.parametrize("padding", [None, "scattered", "all"])
def test_padding(padding):
    check_forward(3, 4, 150, 256, 320, padding=padding)
    check_backward(3, 4, 150, 256, 320, padding=padding)


# every workgroup shape of the products, both tile sizes of dw, in one range of token blocks and several
@pytest.mark.parametrize("B,N,E,F", [(1, 515, 768, 1032), (9, 500, 768, 2048), (2, 2100, 1024, 4096), (5, 1000, 4096, 1024), (1, 16384, 72, 64),
                                     (40, 400, 520, 776), (300, 230, 64, 8)])
def test_larger(B, N, E, F):
    check_forward(N, B, N, E, F, keep_y=False)
    check_backward(N, B, N, E, F)


@pytest.mark.parametrize("K", [8, 64, 72, 128, 136, 320])
def test_what_is_not_finite_stays_in_its_row(K):
    """NaN and infinities at a row's end, beside the first stage's columns that do not exist: the rows beside it, and the features of
    other weights, have finite results; in padding they reach nothing."""
    mate = mate_module()
    print(f"not finite, contraction of {K}", flush=True)
    i = Inputs(K, 2, 80, K, 96, "tail")
    i.flags[1, 5] = PAD
    want, _ = mate.linear(i.x, i.w, i.bias, i.flags, keep_z=mate.MATE_KEEP_8BIT)   # (the same call: the order of the sums goes by sizes and what is kept)
    x, w = i.x.clone(), i.w.clone()
    x[0, 3, -1], x[0, 70, 0], x[1, 5] = math.nan, math.inf, math.nan
    w[7, -1] = math.inf
    y, z = mate.linear(x, w, i.bias, i.flags, keep_z=mate.MATE_KEEP_8BIT)
    back = mate.checkpoint_unpack(z)
    sick = torch.zeros(2, 80, 96, dtype=torch.bool, device="cuda")
    sick[0, 3] = sick[0, 70] = True
    sick[..., 7] = True
    sick &= (i.flags < PAD)[..., None]
    assert torch.equal(torch.isfinite(y), ~sick) and torch.equal(y[~sick], want[~sick])
    assert torch.equal(torch.isnan(back), sick)
    # backward: dy's sick row, and padding of x, z and dy full of NaN
    j = Inputs(K, 2, 80, 96, K, "tail")
    dy, x, z = j.dy.clone(), j.x.clone(), j.z.clone()
    pad = j.flags == PAD
    dx0, dw0, db0 = mate.linear_bwd(dy, x, j.w, j.flags, z=z, act=mate.MATE_ACT_GELU)
    dy[pad], x[pad], z[pad] = math.nan, math.inf, math.nan
    dx1, dw1, db1 = mate.linear_bwd(dy, x, j.w, j.flags, z=z, act=mate.MATE_ACT_GELU)
    assert torch.equal(dx0, dx1) and torch.equal(dw0, dw1) and torch.equal(db0, db1)
    assert torch.equal(mate.activation_bwd(x, z, mate.MATE_ACT_SILU, j.flags)[pad], torch.zeros_like(x)[pad])
    dy[0, 4, -1], dy[0, 60, 0] = math.nan, math.inf
    dx1, dw1, db1 = mate.linear_bwd(dy, x, j.w, j.flags, z=z, act=mate.MATE_ACT_GELU)
    sick = torch.zeros(2, 80, dtype=torch.bool, device="cuda")
    sick[0, 4] = sick[0, 60] = True
    assert torch.equal(dx1[~sick], dx0[~sick]) and not bool(torch.isfinite(dx1[sick]).any())
    rows = torch.arange(1, K - 1)
    assert torch.equal(dw1[rows], dw0[rows]) and torch.equal(db1[rows], db0[rows]) and not bool(torch.isfinite(db1[[0, K - 1]]).any())


def test_exact_where_the_sums_are():
    """Small whole numbers: every product and sum is exact, so z, y and their 8 bits are the oracle's, bit for bit."""
    mate = mate_module()
    gen = torch.Generator(device="cuda").manual_seed(4)
    whole = lambda top, *shape: torch.randint(-top, top + 1, shape, device="cuda", generator=gen).to(torch.bfloat16)
    for B, N, E, F in ((2, 70, 200, 104), (3, 900, 1024, 520)):
        x, w, res = whole(3, B, N, E), whole(2, F, E), whole(50, B, N, F)
        bias = whole(9, F).float()
        flags = (torch.rand(B, N, device="cuda", generator=gen) < 0.2).to(torch.uint8) * PAD
        y, z, y8 = mate.linear(x, w, bias, flags, act=mate.MATE_ACT_RELU, residual=res, keep_z=mate.MATE_KEEP_8BIT, keep_y=True)
        wz, wy = ff.linear(x, w, bias, flags, "relu", res)
        assert torch.equal(y, wy.to(torch.bfloat16))
        for got, want in ((z, wz), (y8, wy)):
            codes, scales = ff.kept(want)
            assert torch.equal(got.scales, scales) and torch.equal(got.codes & 127, codes & 127)
            assert torch.equal(mate.checkpoint_unpack(got, torch.float32).double(), ff.values(codes, scales))
        dx, dw, db = mate.linear_bwd(res, x, w, flags, residual=x)
        wx, ww, wb = ff.linear_backward(res, x, w, flags, residual=x)
        assert torch.equal(dx, wx.to(torch.bfloat16)) and torch.equal(dw.double(), ww) and torch.equal(db.double(), wb)


# ---- 8 bits on their own ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_checkpoint_of_every_magnitude(dtype):
    """All bf16 values, each beside others of its size and of far larger ones; for fp32 also values between them."""
    mate = mate_module()
    bits = torch.arange(65536, dtype=torch.int32, device="cuda") << 16
    x = torch.cat([bits.view(64, 32, 32).flatten(1), bits.view(32, 64, 32).transpose(1, 2).reshape(64, 1024)]).view(torch.float32)
    if dtype == torch.float32:
        x = torch.cat([x, (x.view(torch.int32) + 0x7fff).view(torch.float32)])
    x = x[None].to(dtype)
    got = mate.checkpoint_pack(x)
    codes, scales = ff.kept(x)
    nan = torch.isnan(ff.values(codes, scales))
    assert torch.equal(got.scales, scales) and torch.equal(got.codes[~nan], codes[~nan]) and bool(((got.codes & 127) == 127)[nan].all())
    back = mate.checkpoint_unpack(got, dtype)
    want = ff.values(codes, scales)
    assert torch.equal(torch.isnan(back), nan)
    # (below the type's smallest normal number a value may have more bits than it holds)
    fine = ~nan & ((want.abs() >= 2.0 ** -120) | (want == 0))
    assert torch.equal(back.double()[fine], want[fine])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,N,W", [(1, 1, 8), (3, 5, 24), (2, 33, 40), (1, 700, 48), (7, 1, 1000), (2, 3, 65536), (5, 401, 768), (3, 4097, 136)])
def test_checkpoint_shapes(B, N, W, dtype):
    mate = mate_module()
    gen = torch.Generator(device="cuda").manual_seed(W)
    x = (torch.randn(B, N, W, device="cuda", generator=gen) * torch.exp2(4 * torch.randn(B, N, W, device="cuda", generator=gen))).to(dtype)
    flags = torch.randint(0, 4, (B, N), device="cuda", generator=gen).to(torch.uint8)     # 3: padding as well
    for fl in (None, flags):
        n_codes, n_scales = B * N * W, B * N * -(-W // 32)
        room = [torch.full((n + 64,), 0xa5, dtype=torch.uint8, device="cuda") for n in (n_codes, n_scales)]
        out = mate.Checkpoint(room[0][:n_codes].view(B, N, W), room[1][:n_scales].view(B, N, -1))
        got = mate.checkpoint_pack(x, fl, out)
        assert got is out
        codes, scales = ff.kept(x, fl)
        assert torch.equal(got.codes, codes) and torch.equal(got.scales, scales)
        assert bool((room[0][n_codes:] == 0xa5).all()) and bool((room[1][n_scales:] == 0xa5).all())
        room = torch.full((B * N * W + 64,), 7.0, dtype=dtype, device="cuda")
        back = mate.checkpoint_unpack(got, dtype, out=room[:B * N * W].view(B, N, W))
        assert torch.equal(back.double(), ff.values(codes, scales)) and bool((room[B * N * W:] == 7).all())


@pytest.mark.parametrize("act", ff.ACTS[1:])
def test_activation_gradient_at_every_value(act):
    """All finite bf16 pre-activations, in 16 and in 8 bits, every gradient 1 and random: one rounding and the slope's own error (see
    activation_error; below 2^-126 a product may be a denormal number, off by 2^-134)."""
    mate = mate_module()
    bits = (torch.arange(65536, dtype=torch.int32, device="cuda") << 16).view(torch.float32)
    z = torch.where(torch.isfinite(bits), bits, 1.0).to(torch.bfloat16).view(4, 16, 1024)
    gen = torch.Generator(device="cuda").manual_seed(3)
    flags = torch.randint(0, 3, (4, 16), device="cuda", generator=gen).to(torch.uint8)
    for dy in (torch.ones_like(z), torch.randn(4, 16, 1024, device="cuda", generator=gen).to(torch.bfloat16)):
        for kept, zv in ((z, z.double()), (mate.checkpoint_pack(z), None)):
            if zv is None:
                zv = ff.values(kept.codes, kept.scales)
            dz = mate.activation_bwd(dy, kept, code_of(act), flags)
            want = ff.activation_backward(dy, zv, act, flags)
            near = 2.0 ** -20 * (1 + zv.abs().clamp_max(64))     # (beyond, every slope is 0 or 1 to 2^-24)
            within(dz, want, BF16 * want.abs() + 1.01 * near * dy.double().abs() + 2.0 ** -133, f"{act} dz")
    same = dy.clone()
    mate.activation_bwd(same, z, code_of(act), flags, dz=same)
    assert torch.equal(same, mate.activation_bwd(dy, z, code_of(act), flags))


@pytest.mark.parametrize("act", ff.ACTS)
def test_activation_values_at_every_value(act):
    """A product with the identity: z is the token's own value, all bf16 ones up to 2^60; y holds to one rounding and the formula's error."""
    mate = mate_module()
    bits = (torch.arange(65536, dtype=torch.int32, device="cuda") << 16).view(torch.float32)
    x = torch.where(bits.abs() < 2.0 ** 60, bits, 0.5).to(torch.bfloat16).view(1, 1024, 64)
    w = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    y, z = mate.linear(x, w, act=code_of(act), keep_z=mate.MATE_KEEP_BF16)
    normal = x.abs() >= 2.0 ** -126                       # (the matrix cores may take denormal numbers for zero)
    assert torch.equal(z[normal], x[normal])
    want = ff.act(act, x.double())
    within(y, want, BF16 * want.abs() + 2.0 ** -20 * torch.minimum(x.double().abs(), torch.tensor(64.0, device="cuda")) + 2.0 ** -120, act)


# ---- together, as they are used ----------------------------------------------------------------------
def feed_forward_step(mate, x, w1, b1, w2, b2, flags, dy, eight, act, x8=None):
    """x -> act(x w1^T + b1) w2^T + b2 + x and all gradients; eight: what is kept is kept in 8 bits."""
    keep = mate.MATE_KEEP_8BIT if eight else mate.MATE_KEEP_BF16
    first = mate.linear(x, w1, b1, flags, act=act, keep_z=keep, keep_y=eight)
    h, z, h8 = first if eight else (*first, first[0])
    y, _ = mate.linear(h, w2, b2, flags, residual=x)
    x8 = mate.checkpoint_pack(x, flags) if eight else x
    dz, dw2, db2 = mate.linear_bwd(dy, h8, w2, flags, z=z, act=act)
    dx, dw1, db1 = mate.linear_bwd(dz, x8, w1, flags, residual=dy)
    return dict(h=h, z=z, h8=h8, x8=x8, y=y, dz=dz, dw2=dw2, db2=db2, dx=dx, dw1=dw1, db1=db1)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("B,N,E,F", [(2, 37, 64, 200), (3, 401, 768, 1536)])
def test_feed_forward_step(B, N, E, F, eight):
    """Each link of the chain against the oracle on what the link before it gave, the same bits from a second run and from a
    graph that is replayed between other work."""
    mate = mate_module()
    i = Inputs(N, B, N, E, F, "tail")
    w2, b2, dy = i.normal(E, F, scale=F ** -0.5), i.normal(E, dtype=torch.float32), i.normal(B, N, E)
    act, args = mate.MATE_ACT_GELU, (i.x, i.w, i.bias, w2, b2, i.flags, dy, eight, mate.MATE_ACT_GELU)
    got = feed_forward_step(mate, *args)
    value = lambda t: ff.values(t.codes, t.scales) if isinstance(t, mate.Checkpoint) else t.double()
    h, z, h8, x8 = (value(got[n]) for n in ("h", "z", "h8", "x8"))
    _, y = ff.linear(got["h"], w2, b2, i.flags, residual=i.x)
    ey = sum_error(F + 2, h.abs() @ w2.double().abs().T + b2.double().abs() + i.x.double().abs())
    within(got["y"], y, ey + BF16 * (y.abs() + ey) + 1e-300, "y")
    dz, dw2, db2 = ff.linear_backward(dy, h8, w2, i.flags, z, "gelu")
    raw = dy.double().abs() @ w2.double().abs()
    ez = 1.2 * sum_error(E, raw) + 2.0 ** -20 * (1 + z.abs()) * raw + F32_STEP * dz.abs()
    within(got["dz"], dz, ez + BF16 * (dz.abs() + ez) + 1e-300, "dz")
    g = ff.zero_pads(dy.double().abs(), i.flags).reshape(-1, E)
    within(got["dw2"], dw2, sum_error(B * N, g.T @ h8.abs().reshape(-1, F)) + 1e-300, "dw2")
    within(got["db2"], db2, sum_error(B * N, g.sum(0)) + 1e-300, "db2")
    dx, dw1, db1 = ff.linear_backward(got["dz"], x8, i.w, i.flags, residual=dy)
    g = got["dz"].double().abs().reshape(-1, F)
    ex = sum_error(F + 1, (g @ i.w.double().abs()).view_as(dx) + dy.double().abs())
    within(got["dx"], dx, ex + BF16 * (dx.abs() + ex) + 1e-300, "dx")
    within(got["dw1"], dw1, sum_error(B * N, g.T @ ff.zero_pads(x8.abs(), i.flags).reshape(-1, E)) + 1e-300, "dw1")
    within(got["db1"], db1, sum_error(B * N, g.sum(0)) + 1e-300, "db1")

    def tensors(r):
        return [u for t in r.values() for u in ((t.codes, t.scales) if isinstance(t, mate.Checkpoint) else (t,))]

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        captured = feed_forward_step(mate, *args)
    for replay in range(3):
        for t in tensors(captured):
            if t.data_ptr() != i.x.data_ptr():
                t.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        again = feed_forward_step(mate, *args)
        torch.cuda.synchronize()
        for a, b, c in zip(tensors(got), tensors(captured), tensors(again)):
            assert torch.equal(a, b) and torch.equal(a, c), replay


def test_layer_with_attention():
    """The whole layer: projections, attention, output projection, then the feed-forward half with its residual, forward and back, one
    stream that is not the default one; every gradient finite, padding zero."""
    from paper_2109_04312_amd import synth
    from tests import helpers as hp
    mate = mate_module()
    st = synth.make_config(2, tensors=False).structure
    B, N, H, E, F = st.B, st.N, 12, 768, 1536
    i = Inputs(1, B, N, E, F, None)
    r, c, f = hp.dev_structure(st)
    kinds, x = synth.half_row_half_col(H), i.x
    w_qkv, w_o, w2 = i.normal(3 * E, E, scale=E ** -0.5), i.normal(E, E, scale=E ** -0.5), i.normal(E, F, scale=F ** -0.5)
    dy = i.normal(B, N, E)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        seg = mate.build_segments(r, c, f)
        q, k, v = mate.qkv_project(x, w_qkv, None, f, H)
        o, lse = mate.attn_fwd(q, k, v, seg, kinds, 0.125)
        a = mate.out_project(o, w_o, None, f)
        got = feed_forward_step(mate, a, i.w, i.bias, w2, None, f, dy, True, mate.MATE_ACT_GELU)
        do, dwo, _ = mate.out_project_bwd(o, w_o, f, got["dx"])
        dq, dk, dv = mate.attn_bwd(q, k, v, o, lse, do, seg, kinds, 0.125)
        dx, dwq, _ = mate.qkv_project_bwd(x, w_qkv, f, dq, dk, dv)
    stream.synchronize()
    pad = f == PAD
    for name, t in dict(y=got["y"], dz=got["dz"], da=got["dx"], dx=dx).items():
        assert bool(torch.isfinite(t).all()) and not bool(t[pad].any()), name
    z, h = ff.linear(a, i.w, i.bias, f, "gelu")
    _, y = ff.linear(got["h"], w2, None, f, residual=a)
    err = (got["y"].double() - y).abs()
    assert bool((err <= 2e-2 + BF16 * y.abs()).all())
    assert all(bool(torch.isfinite(t).all()) for t in (dwo, dwq, got["dw1"], got["dw2"]))


def test_gradients_alone_are_the_same_and_may_be_left_out():
    mate = mate_module()
    for B, N, E, F in ((1, 130, 136, 72), (4, 600, 768, 1536), (2, 4100, 520, 264)):
        i = Inputs(N, B, N, E, F, "tail")
        x, z = mate.checkpoint_pack(i.x), mate.checkpoint_pack(i.z)
        kw = dict(z=z, act=mate.MATE_ACT_SILU, residual=i.res_x)
        ws = torch.full((mate.mate_linear_bwd_workspace_bytes(B, N, E, F, 1) + 1,), 255, dtype=torch.uint8, device="cuda")
        both = mate.linear_bwd(i.dy, x, i.w, i.flags, **kw)
        again = mate.linear_bwd(i.dy, x, i.w, i.flags, ws=ws[1:], **kw)         # a workspace at an odd address, full of NaN
        only_x = mate.linear_bwd(i.dy, None, i.w, i.flags, want_dw=False, want_dbias=False, **kw)
        only_w = mate.linear_bwd(i.dy, x, i.w, i.flags, want_dx=False, **kw)
        no_bias = mate.linear_bwd(i.dy, x, i.w, i.flags, want_dbias=False, **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(both, again))
        assert torch.equal(only_x[0], both[0]) and only_x[1] is None and only_x[2] is None
        assert only_w[0] is None and torch.equal(only_w[1], both[1]) and torch.equal(only_w[2], both[2])
        assert torch.equal(no_bias[1], both[1]) and no_bias[2] is None
        with pytest.raises(mate.MateError) as e:
            mate.linear_bwd(i.dy, x, i.w, i.flags, want_dw=False, **kw)           # a bias gradient without the weight gradient
        assert e.value.status == mate.MATE_ERR_NULL


def test_buffers_of_the_caller():
    """The residual's buffer as the result, results that end where other data begins, and rows read from the middle of a tensor."""
    mate = mate_module()
    i = Inputs(8, 3, 70, 136, 200, "scattered")
    want, _ = mate.linear(i.x, i.w, i.bias, i.flags, act=mate.MATE_ACT_TANH, residual=i.res_y)
    n = want.numel()
    room = torch.full((n + 256,), 3.0, dtype=torch.bfloat16, device="cuda")
    got, _ = mate.linear(i.x, i.w, i.bias, i.flags, act=mate.MATE_ACT_TANH, residual=i.res_y, y=room[:n].view_as(want))
    assert torch.equal(got, want) and bool((room[n:] == 3).all())
    same = i.res_y.clone()
    mate.linear(i.x, i.w, i.bias, i.flags, act=mate.MATE_ACT_TANH, residual=same, y=same)
    assert torch.equal(same, want)
    one, _ = mate.linear(i.x[1:2], i.w, i.bias, i.flags[1:2], act=mate.MATE_ACT_TANH, residual=i.res_y[1:2])
    assert torch.equal(one, want[1:2])
    with pytest.raises(ValueError):
        mate.linear(i.x.transpose(0, 1), i.w)
    with pytest.raises(ValueError):
        mate.linear(i.x, i.w, residual=i.res_x)
    with pytest.raises(TypeError):
        mate.linear(i.x.float(), i.w)
    with pytest.raises(mate.MateError):
        mate.linear(torch.zeros(1 + 2 * 8, dtype=torch.bfloat16, device="cuda")[1:].view(1, 2, 8), i.w[:8, :8].contiguous())   # address 2


def test_offsets_past_32_bits():
    """Results of more than 4 GB: the last tokens' rows against the oracle."""
    mate = mate_module()
    B, N, E, F = 40, 16384, 8, 4096
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(B, N, E, device="cuda", generator=gen).to(torch.bfloat16)
    w = torch.randn(F, E, device="cuda", generator=gen).to(torch.bfloat16)
    flags = torch.zeros(B, N, dtype=torch.uint8, device="cuda")
    flags[:, -3] = PAD
    y, z = mate.linear(x, w, None, flags, act=mate.MATE_ACT_RELU, keep_z=mate.MATE_KEEP_8BIT)
    for b in (0, 20, B - 1):
        at = slice(N - 300, N)
        wz, wy = ff.linear(x[b:b + 1, at], w, None, flags[b:b + 1, at], "relu")
        e = sum_error(E, x[b:b + 1, at].double().abs() @ w.double().abs().T)
        within(y[b:b + 1, at], wy, e + BF16 * (wy.abs() + e) + 1e-300, f"y of sequence {b}")
        last = mate.Checkpoint(z.codes[b:b + 1, at].contiguous(), z.scales[b:b + 1, at].contiguous())
        close_8bit(last, wz, torch.where(ff.live(flags[b:b + 1, at], wz), e, 0.0), f"z of sequence {b}")
    back = mate.checkpoint_unpack(z)
    assert torch.equal(back[-1, -2:].double(), ff.values(z.codes[-1, -2:], z.scales[-1, -2:]))
    dz = mate.activation_bwd(y, z, mate.MATE_ACT_RELU, flags)
    assert torch.equal(dz[-1, -300:], torch.where((back[-1, -300:] > 0) & (flags[-1, -300:] < PAD)[:, None], y[-1, -300:], 0))
    _, dw, db = mate.linear_bwd(y, x, w, flags, want_dx=False)
    wdw = torch.zeros(F, E, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(wdw)
    for b in range(B):
        g = ff.zero_pads(y[b:b + 1].double(), flags[b:b + 1])[0]
        wdw += g.T @ x[b].double()
        bound += g.abs().T @ x[b].double().abs()
    within(dw, wdw, sum_error(B * N, bound), "dw")
    dx, _, _ = mate.linear_bwd(y, None, w, flags, want_dw=False, want_dbias=False)
    g = y[-1:, -300:]
    wx = ff.linear_backward(g, x[-1:, -300:], w, flags[-1:, -300:])[0]
    e = sum_error(F, ff.zero_pads(g.double().abs(), flags[-1:, -300:]) @ w.double().abs())
    within(dx[-1:, -300:], wx, e + BF16 * (wx.abs() + e) + 1e-300, "dx")


# ---- each form that sizes choose -----------------------------------------------------------------------
# few tokens without 8 bits: 4, 8, 16 and 32 features by 16, 32 and 64 tokens a workgroup; contractions of less than a step, of whole
# steps, with a rest for one of the eight wavefronts, and as wide as there is; a last token tile and feature tile that are not full
@pytest.mark.parametrize("keep_z", [0, 1])
@pytest.mark.parametrize("B,N,E,F", [(1, 1, 8, 8), (1, 7, 72, 776), (1, 1, 8, 1032), (5, 103, 136, 40), (1, 17, 264, 2048), (5, 13, 264, 1288),
                                     (2, 20, 264, 4096), (7, 100, 72, 1032), (1, 515, 200, 776), (2, 512, 520, 136), (3, 1, 4104, 72),
                                     (1, 9, 65536, 8), (3, 1, 8, 65536), (3, 11, 4096, 1024), (8, 125, 8, 8)])
def test_few_tokens(B, N, E, F, keep_z):
    check_forward(E + N, B, N, E, F, "silu" if keep_z else "gelu_tanh", padding="scattered" if keep_z else "tail", bias=N != 7, residual=N != 13,
                  keep_z=keep_z, keep_y=False)


# tiles of each size, with 8 bits of both, odd widths; and results that are written past the caches
@pytest.mark.parametrize("B,N,E,F", [(9, 1000, 72, 1288), (3, 1500, 768, 776), (9, 1000, 8, 136), (3, 100, 264, 136), (2, 7, 1032, 264), (4, 4096, 64, 4096)])
def test_products(B, N, E, F):
    check_forward(N, B, N, E, F, "silu", padding="scattered", keep_z=1 if N > 3000 else 2)


# both gradients in one launch, dx by tiles of 64 and of 128 tokens, dw in one to eight ranges of token blocks; and in two launches, dw by
# tiles of 128 and of 256, in one range and several; from 16 bits, from 8 bits as they are and copied, with rows that end in half of 16 codes
BACKWARDS = [(5, 13, 72, 2048), (2, 65, 264, 136), (7, 100, 264, 520), (7, 100, 264, 1288), (4, 500, 520, 1032), (3, 1000, 520, 1032), (9, 500, 24, 4096),
             (4, 500, 520, 520), (1, 2000, 136, 2048), (6, 1500, 24, 4096), (6, 1000, 264, 1032), (5, 1200, 200, 1288), (9, 500, 72, 2048),
             (16, 1024, 136, 8), (4, 4096, 4096, 136), (9, 1000, 1032, 1288), (6, 1000, 264, 520), (3, 4000, 136, 776), (3, 1500, 4096, 520),
             (1, 3, 65536, 8), (1, 3, 8, 65536), (1, 515, 4096, 4096), (2, 650, 2048, 264)]


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("B,N,E,F", BACKWARDS)
def test_gradients(B, N, E, F, x8):
    check_backward(N, B, N, E, F, "silu", padding="scattered" if N % 2 else "tail", residual=N % 100 != 0, x8=x8, z8=not x8)


@pytest.mark.parametrize("padding", [None, "all"])
def test_gradients_without_and_of_nothing_but_padding(padding):
    for B, N, E, F in ((2, 65, 264, 136), (4, 500, 520, 520), (9, 500, 72, 2048), (6, 1000, 264, 520)):
        check_backward(N, B, N, E, F, "relu", padding=padding, x8=N == 500)


def one_sequence_only(i, b):
    """Every other sequence is padding: most ranges of token blocks have nothing."""
    i.flags[:] = PAD
    i.flags[b, 3:] = 0


@pytest.mark.parametrize("B,N,E,F", [(9, 500, 72, 2048), (4, 500, 520, 520), (6, 1000, 264, 520)])
def test_results_do_not_depend_on_what_else_is_wanted_or_running(B, N, E, F):
    """Merged ranges and added ones, x in 8 bits and 16: either gradient alone has the same bits, from a workspace full of NaN at an odd address, and
    while the same call runs on another stream with a workspace of its own."""
    mate = mate_module()
    i = Inputs(N, B, N, E, F, "scattered")
    for x in (mate.checkpoint_pack(i.x), i.x):
        kw = dict(z=i.z, act=mate.MATE_ACT_GELU, residual=i.res_x)
        size = mate.mate_linear_bwd_workspace_bytes(B, N, E, F, int(x is not i.x))
        want = mate.linear_bwd(i.dy, x, i.w, i.flags, **kw)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        spaces = [torch.full((size + 3,), 255, dtype=torch.uint8, device="cuda") for _ in streams]
        torch.cuda.synchronize()
        got = []
        for _ in range(5):
            for s, ws in zip(streams, spaces):
                with torch.cuda.stream(s):
                    got.append(mate.linear_bwd(i.dy, x, i.w, i.flags, ws=ws[3:], **kw))
        torch.cuda.synchronize()
        for g in got:
            assert all(torch.equal(u, v) for u, v in zip(g, want))
        only_x = mate.linear_bwd(i.dy, x, i.w, i.flags, want_dw=False, want_dbias=False, **kw)
        only_w = mate.linear_bwd(i.dy, x, i.w, i.flags, want_dx=False, **kw)
        assert torch.equal(only_x[0], want[0]) and torch.equal(only_w[1], want[1]) and torch.equal(only_w[2], want[2])
        one_sequence_only(i, 1)
        alone = mate.linear_bwd(i.dy[1:2].contiguous(), i.x[1:2].contiguous(), i.w, i.flags[1:2].contiguous(), z=i.z[1:2].contiguous(),
                                act=mate.MATE_ACT_GELU, residual=i.res_x[1:2].contiguous())
        among = mate.linear_bwd(i.dy, i.x, i.w, i.flags, **kw)
        one = sum_error(N, i.dy[1].double().abs().T @ i.x[1].double().abs())
        within(among[1], alone[1].double(), 2 * one + 1e-300, "dw of one sequence")


@pytest.mark.parametrize("B,N,E,F", [(9, 500, 72, 2048), (4, 500, 520, 520), (2, 65, 264, 136), (6, 1000, 264, 520)])
def test_two_graphs_of_one_workspace(B, N, E, F):
    """Two captured backward passes share a workspace and are replayed in turn, with a call of the caller's own between them."""
    mate = mate_module()
    inputs = [Inputs(N + k, B, N, E, F, "tail") for k in range(2)]
    kept = [mate.checkpoint_pack(i.x) for i in inputs]
    ws = mate.linear_bwd_workspace(B, N, E, F, True, "cuda")
    ws.fill_(255)

    def step(k, space):
        i = inputs[k]
        return mate.linear_bwd(i.dy, kept[k], i.w, i.flags, z=i.z, act=mate.MATE_ACT_TANH, ws=space)

    want = [step(k, None) for k in range(2)]
    graphs, captured = [], []
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            captured.append(step(k, ws))
        graphs.append(graph)
    for replay in range(3):
        for k in (0, 1, 1, 0):
            for t in captured[k]:
                t.fill_(77)
            graphs[k].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(captured[k], want[k])), (replay, k)
            again = step(1 - k, ws)
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(again, want[1 - k])), (replay, k)


def test_few_tokens_in_a_graph_and_beside_each_other():
    """Single tokens, as an answer's: replays in a graph, the same bits whichever tokens stand beside them in a call of the same sizes."""
    mate = mate_module()
    for B, N, E, F in ((1, 1, 768, 776), (3, 11, 264, 4096)):
        i = Inputs(N, B, N, E, F, None)
        kw = dict(act=mate.MATE_ACT_GELU, residual=i.res_y, keep_z=mate.MATE_KEEP_BF16)
        want = mate.linear(i.x, i.w, i.bias, None, **kw)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            got = mate.linear(i.x, i.w, i.bias, None, **kw)
        for _ in range(3):
            for t in got:
                t.fill_(77)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(got, want))
        same = i.res_y.clone()
        mate.linear(i.x, i.w, i.bias, None, act=mate.MATE_ACT_GELU, residual=same, y=same)
        assert torch.equal(same, want[0])
        x = i.x.clone()
        x[:, 1:] = math.nan
        y, z = mate.linear(x, i.w, i.bias, None, **kw)
        assert torch.equal(y[:, 0], want[0][:, 0]) and torch.equal(z[:, 0], want[1][:, 0])
        assert N == 1 or bool(torch.isnan(y[:, 1:]).all())


# a contraction shared by two, three and four ranges, with a rest for the last one, tiles that are not full, one that is padding
SPLITS = [(1, 300, 2048, 1024), (2, 500, 4096, 264), (3, 100, 4104, 776), (1, 515, 4032, 1032), (5, 400, 1992, 136), (1, 64, 4096, 8)]


@pytest.mark.parametrize("B,N,E,F", SPLITS)
def test_split_contractions(B, N, E, F):
    check_forward(N, B, N, E, F, "gelu", padding="scattered")
    check_forward(N + 1, B, N, E, F, "none", bias=False, residual=False, keep_z=1, keep_y=False)
    check_forward(N + 2, B, N, E, F, "silu", padding="all")


def test_split_contractions_again_together_and_in_graphs():
    """The same bits in every run: on two streams at once, and from two graphs that share a workspace, full of NaN at first and at an odd address."""
    mate = mate_module()
    B, N, E, F = 3, 100, 4104, 776
    inputs = [Inputs(k, B, N, E, F, "scattered") for k in range(2)]
    size = mate.mate_linear_workspace_bytes(B, N, E, F, 1)
    assert size > 0

    def step(k, ws=None):
        i = inputs[k]
        y, z = mate.linear(i.x, i.w, i.bias, i.flags, act=mate.MATE_ACT_GELU, residual=i.res_y, keep_z=mate.MATE_KEEP_8BIT, ws=ws)
        return y, z.codes, z.scales

    want = [step(k) for k in range(2)]
    room = [torch.full((size + 5,), 255, dtype=torch.uint8, device="cuda") for k in range(2)]
    ws = [t[5:] for t in room]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got.append((k, step(k, ws[k])))
    torch.cuda.synchronize()
    for k, g in got:
        assert all(torch.equal(u, v) for u, v in zip(g, want[k]))
    graphs, captured = [], []
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            captured.append(step(k, ws[0]))
        graphs.append(graph)
    for replay in range(3):
        for k in (0, 1, 1, 0):
            for t in captured[k]:
                t.fill_(77)
            graphs[k].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(u, v) for u, v in zip(captured[k], want[k])), (replay, k)
            assert all(torch.equal(u, v) for u, v in zip(step(1 - k, ws[0]), want[1 - k])), (replay, k)
    with pytest.raises(mate.MateError) as e:
        step(0, ws[0][:size - 1])
    assert e.value.status == mate.MATE_ERR_WORKSPACE
    i = inputs[0]
    x = i.x.clone()
    x[0, 3, -1] = math.nan                        # of the last range
    x[0, 5, 0] = math.inf                         # of the first
    y, z = mate.linear(x, i.w, i.bias, None, keep_z=mate.MATE_KEEP_8BIT)
    sick = torch.zeros(B, N, dtype=torch.bool, device="cuda")
    sick[0, 3] = sick[0, 5] = True
    assert torch.equal(torch.isfinite(y).all(-1), ~sick) and torch.equal(torch.isnan(mate.checkpoint_unpack(z)).any(-1), sick)


# results in 8 bits of few tokens: a last scale block of 8, 16, 24 features or all 32, one to more than one token tile of each height
@pytest.mark.parametrize("B,N,E,F", [(1, 1, 8, 8), (1, 1, 768, 776), (3, 4, 1656, 2360), (1, 16, 4096, 48), (1, 17, 72, 88), (5, 13, 264, 1288),
                                     (3, 101, 3344, 216), (7, 100, 360, 272), (2, 512, 520, 136), (1, 9, 65536, 40), (2, 1, 8, 65536)])
def test_few_tokens_in_8_bits(B, N, E, F):
    check_forward(E + N, B, N, E, F, "silu", padding="scattered")
    check_forward(E + N + 1, B, N, E, F, "gelu", padding="tail", bias=False, residual=False, keep_z=1, keep_y=True)
    check_forward(E + N + 2, B, N, E, F, "tanh", padding="all", keep_z=2, keep_y=False)


# dx of few tokens and a long contraction, shared by two and more ranges beside dw's tiles or alone; a rest for the last range, padding
@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("B,N,E,F", [(2, 16, 216, 3656), (1, 1, 8, 4096), (9, 26, 264, 2376), (4, 34, 320, 2720), (3, 100, 520, 4104)])
def test_split_dx(B, N, E, F, x8):
    mate = mate_module()
    assert mate.mate_linear_bwd_dx_workspace_bytes(B, N, E, F) > 0
    check_backward(N, B, N, E, F, "gelu", padding="scattered", residual=N != 16, x8=x8, z8=not x8)
    check_backward(N + 1, B, N, E, F, "none", padding="all" if x8 else None, x8=x8)
    i = Inputs(N, B, N, E, F, "scattered")
    x = mate.checkpoint_pack(i.x) if x8 else i.x
    kw = dict(z=i.z, act=mate.MATE_ACT_GELU, residual=i.res_x)
    both = mate.linear_bwd(i.dy, x, i.w, i.flags, **kw)
    size = mate.mate_linear_bwd_dx_workspace_bytes(B, N, E, F)
    room = torch.full((size + 7,), 255, dtype=torch.uint8, device="cuda")
    for ws in (None, room[7:]):
        alone = mate.linear_bwd(i.dy, None, i.w, i.flags, want_dw=False, want_dbias=False, ws=ws, **kw)
        assert torch.equal(alone[0], both[0]) and alone[1] is None
    assert all(torch.equal(u, v) for u, v in zip(mate.linear_bwd(i.dy, x, i.w, i.flags, want_dx=False, **kw)[1:], both[1:]))
    with pytest.raises(mate.MateError) as e:
        mate.linear_bwd(i.dy, None, i.w, i.flags, want_dw=False, want_dbias=False, ws=room[:size - 1], **kw)
    assert e.value.status == mate.MATE_ERR_WORKSPACE
    ws = torch.full((mate.mate_linear_bwd_workspace_bytes(B, N, E, F, int(x8)) + 9,), 255, dtype=torch.uint8, device="cuda")[9:]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        captured = mate.linear_bwd(i.dy, x, i.w, i.flags, ws=ws, **kw)
    for replay in range(3):
        for t in captured:
            t.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(captured, both)), replay
        again = mate.linear_bwd(i.dy, x, i.w, i.flags, ws=ws, **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(again, both)), replay
