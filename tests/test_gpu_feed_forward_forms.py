"""Every form that sizes choose in the feed-forward half (tests/test_feed_forward_forms.py holds each size to the form named here), with small whole
numbers: every product and every partial sum is exact in fp32 in any order (below 2^24), so that results are the oracle's bit for bit, and a
lost, doubled or misplaced term shows at any width and length."""
import math

import pytest
import torch

from oracle import feed_forward as ff

pytestmark = pytest.mark.gpu
PAD = 2

# B, N, E, F, results in 8 bits, form: features x tokens of few tokens' workgroups, ranges of a split contraction, or tiles.  Token counts and widths
# that no tile divides, up to the widest.
FORWARD = [
    (1, 23, 40, 48, 0, "few 4x16"), (3, 1, 65536, 8, 0, "few 4x16"), (3, 37, 40, 152, 0, "few 8x16"), (1, 178, 40, 176, 0, "few 16x16"),
    (2, 201, 40, 296, 0, "few 16x32"), (4, 6, 1024, 4096, 0, "few 16x32"), (7, 89, 40, 392, 0, "few 16x64"), (3, 65, 40, 312, 0, "few 32x16"),
    (9, 1, 8, 65536, 0, "few 32x16"), (4, 73, 40, 424, 0, "few 32x32"), (5, 109, 40, 456, 0, "few 32x64"),
    (1, 23, 40, 56, 1, "few 32x16"), (9, 1, 40, 65528, 1, "few 32x16"), (2, 201, 40, 296, 1, "few 32x32"), (5, 109, 40, 456, 1, "few 32x64"),
    (1, 128, 1024, 4096, 1, "few 32x64"), (5, 25, 1000, 4088, 1, "few 32x64"),
    (2, 557, 2000, 40, 0, "split 2"), (2, 515, 3808, 40, 1, "split 3"), (3, 349, 4168, 40, 0, "split 4"), (1, 27, 4080, 40, 1, "split 4"),
    (1, 1, 14904, 5464, 1, "split 5"), (7, 333, 9208, 40, 0, "split 6"), (2, 65, 8016, 240, 0, "split 7"), (3, 7, 7184, 56, 1, "split 7"),
    (2, 17, 8216, 728, 0, "split 8"), (1, 9, 65536, 8, 0, "split 8"), (1, 9, 65536, 40, 1, "split 8"), (2, 33, 65528, 136, 1, "split 8"),
    (2, 517, 40, 48, 1, "tiles 64"), (2, 518, 40, 48, 0, "tiles 64"), (3, 11, 136, 65536, 1, "tiles 64"), (1, 1037, 144, 40, 0, "tiles 64x2"),
    (3, 347, 144, 40, 1, "tiles 64x2"), (8, 207, 40, 1160, 0, "tiles 128"), (5, 16001, 72, 136, 1, "tiles 128"),
    (1, 8453, 328, 136, 1, "tiles 128x2"), (3, 2819, 328, 136, 0, "tiles 128x2"), (7, 643, 72, 2696, 0, "tiles 256"), (3, 1501, 72, 2696, 1, "tiles 256"),
]
# B, N, E, F, how dw (tile and ranges of token blocks; 9: nine or more) and dx (tiles, ranges of its contraction), and x in 8 bits, are read
BACKWARD = [
    (1, 23, 40, 136, "one launches, dw 128 ranges 1, dx 128x2", "direct"), (3, 129, 40, 144, "one launches, dw 128 ranges 1, dx 128x2", "copied"),
    (1, 23, 40, 392, "one launches, dw 128 ranges 1, dx 64x2", "direct"), (1, 433, 40, 856, "one launches, dw 128 ranges 1, dx 64x2", "copied"),
    (2, 11, 40, 1992, "one launches, dw 128 ranges 1, dx 64x2 split 2", "direct"), (3, 151, 40, 1992, "one launches, dw 128 ranges 1, dx 64x2 split 2", "copied"),
    (5, 5, 48, 3032, "one launches, dw 128 ranges 1, dx 64x2 split 3", "direct"), (3, 153, 40, 3016, "one launches, dw 128 ranges 1, dx 64x2 split 3", "copied"),
    (1, 29, 40, 4048, "one launches, dw 128 ranges 1, dx 64x2 split 4", "direct"), (1, 389, 40, 4064, "one launches, dw 128 ranges 1, dx 64x2 split 4", "copied"),
    (1, 23, 288, 10024, "one launches, dw 128 ranges 1, dx 64x2 split 5", "direct"), (2, 265, 136, 9832, "one launches, dw 128 ranges 1, dx 64x2 split 5", "copied"),
    (1, 23, 40, 6088, "one launches, dw 128 ranges 1, dx 64x2 split 6", "direct"), (3, 139, 40, 6288, "one launches, dw 128 ranges 1, dx 64x2 split 6", "copied"),
    (8, 3, 40, 7112, "one launches, dw 128 ranges 1, dx 64x2 split 7", "direct"), (1, 397, 40, 7320, "one launches, dw 128 ranges 1, dx 64x2 split 7", "copied"),
    (1, 23, 40, 8184, "one launches, dw 128 ranges 1, dx 64x2 split 8", "direct"), (1, 419, 40, 8392, "one launches, dw 128 ranges 1, dx 64x2 split 8", "copied"),
    (2, 701, 40, 144, "one launches, dw 128 ranges 2, dx 128x2", "copied"), (5, 281, 1712, 336, "one launches, dw 128 ranges 2, dx 128x2", "direct"),
    (5, 279, 40, 1656, "one launches, dw 128 ranges 2, dx 64x2", "copied"), (8, 187, 40, 2080, "one launches, dw 128 ranges 2, dx 64x2 split 2", "copied"),
    (2, 745, 40, 3248, "one launches, dw 128 ranges 2, dx 64x2 split 3", "copied"), (3, 540, 40, 4192, "one launches, dw 128 ranges 2, dx 64x2 split 4", "copied"),
    (3, 689, 528, 1048, "one launches, dw 128 ranges 3, dx 128x2", "copied"), (7, 348, 1400, 400, "one launches, dw 128 ranges 3, dx 128x2", "direct"),
    (2, 2449, 40, 4264, "one launches, dw 128 ranges 3, dx 64x2", "copied"), (5, 489, 40, 4632, "one launches, dw 128 ranges 3, dx 64x2 split 3", "copied"),
    (6, 331, 352, 528, "one launches, dw 128 ranges 4, dx 128x2", "direct"), (5, 415, 40, 680, "one launches, dw 128 ranges 4, dx 128x2", "copied"),
    (13, 157, 40, 2272, "one launches, dw 128 ranges 4, dx 64x2 split 2", "copied"), (2, 1157, 1432, 352, "one launches, dw 128 ranges 4, dx 64x2", "direct"),
    (3, 2647, 8, 3896, "one launches, dw 128 ranges 5, dx 128x2", "copied"), (5, 1054, 40, 3272, "one launches, dw 128 ranges 6, dx 64x2", "copied"),
    (2, 2002, 40, 1112, "one launches, dw 128 ranges 7, dx 128x2", "copied"), (2, 1997, 584, 520, "one launches, dw 128 ranges 7, dx 128x2", "direct"),
    (1, 4079, 168, 1080, "one launches, dw 128 ranges 8, dx 128x2", "direct"), (2, 2142, 40, 2592, "one launches, dw 128 ranges 8, dx 64x2", "copied"),
    (1, 23, 40, 40, "two launches, dw 128 ranges 1, dx 64", "direct"), (5, 77, 48, 40, "two launches, dw 128 ranges 1, dx 64", "copied"),
    (3, 7, 1848, 2208, "two launches, dw 128 ranges 1, dx 64x2", "direct"), (3, 67, 2712, 1416, "two launches, dw 128 ranges 1, dx 64x2", "copied"),
    (7, 85, 3360, 40, "two launches, dw 128 ranges 1, dx 128", "direct"), (3, 47, 11152, 360, "two launches, dw 128 ranges 1, dx 128x2", "direct"),
    (3, 313, 13992, 72, "two launches, dw 128 ranges 1, dx 256", "direct"), (9, 1, 65536, 8, "two launches, dw 128 ranges 1, dx 64", "direct"),
    (9, 1, 8, 65536, "two launches, dw 128 ranges 1, dx 64x2", "direct"), (3, 11, 136, 65536, "two launches, dw 128 ranges 1, dx 64x2", "direct"),
    (6, 228, 1424, 40, "two launches, dw 128 ranges 2, dx 128", "copied"), (11, 111, 1624, 40, "two launches, dw 128 ranges 2, dx 128", "direct"),
    (11, 89, 40, 40, "two launches, dw 128 ranges 2, dx 64", "copied"), (3, 333, 616, 40, "two launches, dw 128 ranges 2, dx 64", "direct"),
    (2, 8213, 40, 352, "two launches, dw 128 ranges 9, dx 128x2", "copied"), (5, 1678, 144, 344, "two launches, dw 128 ranges 9, dx 128x2", "direct"),
    (2, 2298, 144, 160, "two launches, dw 128 ranges 9, dx 64x2", "direct"), (5, 1091, 280, 40, "two launches, dw 128 ranges 9, dx 128", "direct"),
    (1, 20, 34872, 2120, "two launches, dw 256 ranges 1, dx 64", "direct"), (1, 1, 9480, 10272, "two launches, dw 256 ranges 1, dx 64x2", "copied"),
    (6, 309, 22344, 136, "two launches, dw 256 ranges 2, dx 256", "direct"), (3, 1937, 5464, 144, "two launches, dw 256 ranges 9, dx 256", "direct"),
    (2, 6343, 136, 3224, "two launches, dw 256 ranges 9, dx 128x2", "copied"), (7, 2557, 392, 2160, "two launches, dw 256 ranges 9, dx 256", "copied"),
    (5, 16001, 72, 136, "two launches, dw 128 ranges 9 listed apart, dx 128", "direct"), (5, 14001, 1032, 520, "two launches, dw 256 ranges 9 listed apart, dx 256", "direct"),
    (41, 16001, 8, 264, "two launches, dw 128 ranges 9 listed apart, dx 128", "copied"),
]


class Whole:
    """Whole numbers: |x| <= 3, |w| <= 2, |dy| <= 3, so a sum of 65536 products is below 2^19 and one of 656041 tokens below 2^23; flags as `padding`
    says, with every third sequence padding from its start to its end where there are several."""

    def __init__(self, seed, B, N, E, F):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        whole = lambda top, *shape: torch.randint(-top, top + 1, shape, device="cuda", generator=gen, dtype=torch.int8).to(torch.bfloat16)
        self.x, self.w, self.dy = whole(3, B, N, E), whole(2, F, E), whole(3, B, N, F)
        self.bias = whole(9, F).float()
        self.res_y, self.res_x, self.z = whole(50, B, N, F), whole(50, B, N, E), whole(2, B, N, E)
        self.flags = (torch.rand(B, N, device="cuda", generator=gen) < 0.2).to(torch.uint8) * PAD
        self.flags[1::3] = PAD


def mate_module():
    from paper_2109_04312_amd import mate
    return mate


def same_8_bits(got, want, what):
    codes, scales = ff.kept(want)
    assert torch.equal(got.scales, scales) and torch.equal(got.codes & 127, codes & 127), what
    assert torch.equal(mate_module().checkpoint_unpack(got, torch.float32).double(), ff.values(codes, scales)), what


@pytest.mark.parametrize("B,N,E,F,codes,form", FORWARD)
def test_forward(B, N, E, F, codes, form):
    mate = mate_module()
    print(f"{form}: {B} x {N}, {E} -> {F}", flush=True)
    i = Whole(N + E, B, N, E, F)
    keep = mate.MATE_KEEP_8BIT if codes else mate.MATE_KEEP_BF16
    got = mate.linear(i.x, i.w, i.bias, i.flags, act=mate.MATE_ACT_RELU, residual=i.res_y, keep_z=keep, keep_y=bool(codes))
    z, y = ff.linear(i.x, i.w, i.bias, i.flags, "relu", i.res_y)
    assert torch.equal(got[0], y.to(torch.bfloat16))
    if codes:
        same_8_bits(got[1], z, "z")
        same_8_bits(got[2], y, "y")
    else:
        assert torch.equal(got[1], z.to(torch.bfloat16))


def gradients(i):
    """The oracle's, one sequence at a time (the longest in 64 bits would not fit)."""
    dx, dw, db = [], 0, 0
    for b in range(len(i.x)):
        at = slice(b, b + 1)
        g = ff.linear_backward(i.dy[at], i.x[at], i.w, i.flags[at], i.z[at], "relu", i.res_x[at])
        dx.append(g[0].to(torch.bfloat16))
        dw, db = dw + g[1], db + g[2]
    return torch.cat(dx), dw.float(), db.float()


@pytest.mark.parametrize("B,N,E,F,form,how", BACKWARD)
def test_backward(B, N, E, F, form, how):
    """Both gradients together and each alone, x in 16 and in 8 bits (which whole numbers up to 3 are exact in)."""
    mate = mate_module()
    print(f"{form}, {how}: {B} x {N}, {E} <- {F}", flush=True)
    i = Whole(N + F, B, N, E, F)
    dx, dw, db = gradients(i)
    assert float(dw.abs().max()) < 2 ** 24
    for x, z in ((i.x, mate.checkpoint_pack(i.z)), (mate.checkpoint_pack(i.x), i.z)):
        kw = dict(z=z, act=mate.MATE_ACT_RELU, residual=i.res_x)
        both = mate.linear_bwd(i.dy, x, i.w, i.flags, **kw)
        only_x = mate.linear_bwd(i.dy, None, i.w, i.flags, want_dw=False, want_dbias=False, **kw)
        only_w = mate.linear_bwd(i.dy, x, i.w, i.flags, want_dx=False, **kw)
        for what, got in (("both", both), ("alone", (only_x[0], only_w[1], only_w[2]))):
            for name, u, v in zip(("dx", "dw", "dbias"), got, (dx, dw, db)):
                assert torch.equal(u, v), f"{name}, {what}"


def test_every_code_at_every_scale():
    """What a checkpoint stands for, at all scales that packing makes: exact in fp32, and in bf16 from scale 3 on; the nearest bf16 below."""
    mate = mate_module()
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(1, 247, 1)
    scales = torch.arange(1, 248, dtype=torch.uint8, device="cuda")[None, :, None].repeat(1, 1, 8)
    kept, want = mate.Checkpoint(codes.contiguous(), scales.contiguous()), ff.values(codes, scales)
    want = torch.where(want.abs() < 2.0 ** 128, want, math.nan)   # (the largest codes of the largest scales, which packing does not make)
    nan = torch.isnan(want)
    for dtype in (torch.float32, torch.bfloat16):
        got = mate.checkpoint_unpack(kept, dtype)
        assert torch.equal(got[~nan], want.to(dtype)[~nan])       # (below, want has at most four bits: one rounding, fp32 holds it)
    exact = ~nan & ((scales >= 3).repeat_interleave(32, -1) | (want.abs() >= 2.0 ** -130))
    assert torch.equal(got.double()[exact], want[exact]) and not torch.equal(got.double()[~nan], want[~nan])
