"""Elementwise passes over more rows than one dimension of a launch takes: the rows on either side of where the second begins, and the last."""
import pytest
import torch

from oracle import feed_forward as ff

pytestmark = pytest.mark.gpu
PAD = 2


def test_rows_past_the_first_dimension():
    from paper_2109_04312_amd import mate
    B, N, E = 513, 16384, 4104               # a row a workgroup, 2^23 of them in the first dimension: it ends with sequence 511
    need = B * N * E * 3.2
    if torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved() - torch.cuda.memory_allocated() < 1.1 * need:
        pytest.skip(f"needs {need / 1e9:.0f} GB")
    torch.cuda.empty_cache()
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.zeros(B, N, E, dtype=torch.bfloat16, device="cuda")
    flags = torch.zeros(B, N, dtype=torch.uint8, device="cuda")
    places = [(0, 0), (510, N - 40), (511, N - 40), (512, 0), (512, 7000), (512, N - 40)]
    for b, n in places:
        x[b, n:n + 40] = torch.randn(40, E, device="cuda", generator=gen).to(torch.bfloat16)
        flags[b, n + 3] = PAD
    kept = mate.checkpoint_pack(x, flags)
    for b, n in places:
        at = slice(n, n + 40)
        codes, scales = ff.kept(x[b:b + 1, at], flags[b:b + 1, at])
        assert torch.equal(kept.codes[b:b + 1, at], codes) and torch.equal(kept.scales[b:b + 1, at], scales), (b, n)
    want = [torch.where((flags[b, n:n + 40] < PAD)[:, None] & (ff.values(kept.codes[b, n:n + 40], kept.scales[b, n:n + 40]) > 0), x[b, n:n + 40], 0)
            for b, n in places]
    mate.activation_bwd(x, kept, mate.MATE_ACT_RELU, flags, dz=x)
    for (b, n), w in zip(places, want):
        assert torch.equal(x[b, n:n + 40], w), (b, n)
    mate.checkpoint_unpack(kept, torch.bfloat16, out=x)
    for b, n in places:
        assert torch.equal(x[b, n:n + 40].double(), ff.values(kept.codes[b, n:n + 40], kept.scales[b, n:n + 40])), (b, n)
    del x, kept, flags
    torch.cuda.empty_cache()
