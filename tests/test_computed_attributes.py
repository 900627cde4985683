"""Objects whose tensors are computed when they are asked for: nothing else holds them while a call looks at them (CPU only, nothing is launched)."""
import gc

import pytest
import torch

from paper_2109_04312_amd import mate


class Computed:
    """codes, scales and buf made anew at each access, from memory that others have just used."""
    B, N, W = 2, 5, 40

    def __init__(self, dims=3):
        self.dims, self.made = dims, 0

    def fresh(self, *shape):
        self.made += 1
        return torch.zeros(shape, dtype=torch.uint8)

    @property
    def codes(self):
        return self.fresh(*(self.B, self.N, self.W)[3 - self.dims:])

    @property
    def scales(self):
        return self.fresh(self.B, self.N, 2)

    @property
    def buf(self):
        return self.fresh(mate.mate_segments_bytes(self.B, self.N))


class ComputedCheckpoint(Computed, mate.Checkpoint):
    pass


@pytest.mark.parametrize("kind", [Computed, ComputedCheckpoint])
def test_checkpoint_unpack(kind):
    for _ in range(20):
        gc.collect()
        c = kind()
        with pytest.raises(ValueError, match="device tensors"):   # and not another shape or type, read from what was freed
            mate.checkpoint_unpack(c)
        assert c.made == 2                                        # each tensor is asked for once
        with pytest.raises(ValueError, match="B, N, width"):
            mate.checkpoint_unpack(kind(dims=2))


def test_checkpoint_of_no_tensors():
    with pytest.raises(TypeError, match="two tensors"):
        mate.checkpoint_unpack(mate.Checkpoint(None, torch.zeros(2, 5, 2, dtype=torch.uint8)))
    with pytest.raises(TypeError, match="two tensors"):
        mate.checkpoint_unpack(mate.Checkpoint(torch.zeros(2, 5, 40, dtype=torch.uint8), 3))
    with pytest.raises(AttributeError):
        mate.checkpoint_unpack(torch.zeros(2, 5, 40))


def test_segment_tables():
    x = torch.zeros(Computed.B, 4, Computed.N, 64, dtype=torch.bfloat16)
    lse = torch.zeros(Computed.B, 4, Computed.N)
    for _ in range(20):
        gc.collect()
        with pytest.raises(ValueError, match="q must be a contiguous device tensor"):   # the tables themselves are right
            mate.attn_fwd(x, x, x, Computed(), [0, 0, 1, 1], 0.125, out=x, lse=lse, ws=torch.zeros(16, dtype=torch.uint8))
        with pytest.raises(ValueError, match="q must be a contiguous device tensor"):
            mate.attn_bwd(x, x, x, x, lse, x, Computed(), [0, 0, 1, 1], 0.125, dq=x, dk=x, dv=x, ws=torch.zeros(16, dtype=torch.uint8))
    other = Computed()
    other.N = Computed.N + 1
    with pytest.raises(mate.MateError):
        mate.attn_fwd(x, x, x, other, [0, 0, 1, 1], 0.125)
