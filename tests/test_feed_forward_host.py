"""Refusals of the feed-forward half's entry points, before anything is launched (CPU only)."""
import pytest
import torch

from paper_2109_04312_amd import mate

FAKE = 0x1000  # never dereferenced


def refuses(f, ok, cases):
    for pos, val, want in cases:
        args = list(ok)
        args[pos] = val
        assert f(*args) == want, (pos, val)


def test_linear():
    #    x, w, bias, flags, residual, B, N, E, F, act, t, y, z, z_scales, y_codes, y_scales, ws, bytes, stream
    ok = [FAKE, FAKE, FAKE, FAKE, FAKE, 2, 100, 768, 1000, mate.MATE_ACT_GELU, mate.MATE_BF16, FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, None]
    refuses(mate.mate_linear, ok, [
        (0, None, mate.MATE_ERR_NULL), (1, None, mate.MATE_ERR_NULL), (11, None, mate.MATE_ERR_NULL), (12, None, mate.MATE_ERR_NULL),
        (14, None, mate.MATE_ERR_NULL), (15, None, mate.MATE_ERR_NULL),
        (5, 0, mate.MATE_ERR_SHAPE), (6, 0, mate.MATE_ERR_SHAPE), (6, mate.MATE_MAX_N + 1, mate.MATE_ERR_SHAPE), (5, 1 << 25, mate.MATE_ERR_SHAPE),
        (7, 0, mate.MATE_ERR_SHAPE), (8, -8, mate.MATE_ERR_SHAPE),
        (7, 764, mate.MATE_ERR_UNSUPPORTED), (8, 1001, mate.MATE_ERR_UNSUPPORTED), (7, mate.MATE_MAX_WIDTH + 8, mate.MATE_ERR_UNSUPPORTED),
        (9, 6, mate.MATE_ERR_UNSUPPORTED), (9, -1, mate.MATE_ERR_UNSUPPORTED), (10, mate.MATE_F32, mate.MATE_ERR_UNSUPPORTED),
        *((i, FAKE + 8, mate.MATE_ERR_UNSUPPORTED) for i in (0, 1, 2, 4, 11, 12, 14))])
    assert mate.mate_linear_workspace_bytes(2, 100, 768, 1000, 1) == 0       # none is needed
    assert mate.mate_linear_workspace_bytes(2, 0, 768, 1000, 1) == mate.mate_linear_workspace_bytes(2, 100, 764, 1000, 1) == 0
    need = mate.mate_linear_workspace_bytes(1, 300, 4096, 1000, 1)           # few tiles of a long contraction
    assert need > 0
    ok[5:9], ok[16:18] = [1, 300, 4096, 1000], [FAKE, need]
    refuses(mate.mate_linear, ok, [(16, None, mate.MATE_ERR_WORKSPACE), (17, need - 1, mate.MATE_ERR_WORKSPACE)])


def test_linear_bwd():
    #    dy, x, x_scales, w, flags, z, z_scales, residual, B, N, E, F, act, t, dx, dw, dbias, ws, bytes, stream
    ok = [FAKE] * 8 + [2, 100, 768, 1000, mate.MATE_ACT_GELU, mate.MATE_BF16, FAKE, FAKE, FAKE, FAKE, 1 << 40, None]
    refuses(mate.mate_linear_bwd, ok, [
        (0, None, mate.MATE_ERR_NULL), (1, None, mate.MATE_ERR_NULL), (3, None, mate.MATE_ERR_NULL), (5, None, mate.MATE_ERR_NULL),
        (15, None, mate.MATE_ERR_NULL), (8, 0, mate.MATE_ERR_SHAPE), (9, 0, mate.MATE_ERR_SHAPE), (10, 0, mate.MATE_ERR_SHAPE),
        (10, 12, mate.MATE_ERR_UNSUPPORTED), (11, 4, mate.MATE_ERR_UNSUPPORTED), (13, mate.MATE_F32, mate.MATE_ERR_UNSUPPORTED),
        (12, mate.MATE_ACT_NONE, mate.MATE_ERR_UNSUPPORTED), (12, 9, mate.MATE_ERR_UNSUPPORTED),
        *((i, FAKE + 8, mate.MATE_ERR_UNSUPPORTED) for i in (0, 1, 3, 5, 7, 14, 15, 16)),
        (17, None, mate.MATE_ERR_WORKSPACE), (18, 1, mate.MATE_ERR_WORKSPACE)])
    no_z = list(ok)
    no_z[5] = no_z[6] = None                                     # an activation without its pre-activation
    assert mate.mate_linear_bwd(*no_z) == mate.MATE_ERR_UNSUPPORTED
    need = mate.mate_linear_bwd_workspace_bytes(2, 100, 768, 1000, 1)
    assert need > 0
    refuses(mate.mate_linear_bwd, ok, [(18, need - 1, mate.MATE_ERR_WORKSPACE)])
    alone = list(ok)                                             # dx alone, at sizes where it needs a workspace
    alone[8:12], alone[15], alone[16] = [1, 32, 216, 4096], None, None
    need = mate.mate_linear_bwd_dx_workspace_bytes(1, 32, 216, 4096)
    assert 0 < need < mate.mate_linear_bwd_workspace_bytes(1, 32, 216, 4096, 1)
    refuses(mate.mate_linear_bwd, alone, [(17, None, mate.MATE_ERR_WORKSPACE), (18, need - 1, mate.MATE_ERR_WORKSPACE)])
    assert mate.mate_linear_bwd_dx_workspace_bytes(2, 100, 768, 1000) == mate.mate_linear_bwd_dx_workspace_bytes(1, 32, 212, 4096) == 0
    assert mate.mate_linear_bwd_workspace_bytes(2, 100, 765, 1000, 0) == 0
    assert mate.mate_linear_bwd_workspace_bytes(0, 100, 768, 1000, 0) == 0
    with pytest.raises(mate.MateError):
        mate.linear_bwd_workspace(2, 100, 765, 1000, False, "cpu")


def test_elementwise():
    ok = [FAKE, FAKE, FAKE, FAKE, 2, 100, 768, mate.MATE_ACT_SILU, mate.MATE_BF16, FAKE, None]   # dy, z, z_scales, flags, B, N, E, act, t, dz
    refuses(mate.mate_activation_bwd, ok, [
        (0, None, mate.MATE_ERR_NULL), (1, None, mate.MATE_ERR_NULL), (9, None, mate.MATE_ERR_NULL), (4, 0, mate.MATE_ERR_SHAPE),
        (6, 770, mate.MATE_ERR_UNSUPPORTED), (7, 0, mate.MATE_ERR_UNSUPPORTED), (7, 6, mate.MATE_ERR_UNSUPPORTED),
        (8, mate.MATE_F32, mate.MATE_ERR_UNSUPPORTED), (0, FAKE + 2, mate.MATE_ERR_UNSUPPORTED), (9, FAKE + 8, mate.MATE_ERR_UNSUPPORTED)])
    ok = [FAKE, FAKE, 2, 100, 768, mate.MATE_F32, FAKE, FAKE, None]      # x, flags, B, N, E, t, codes, scales
    refuses(mate.mate_checkpoint_pack, ok, [
        (0, None, mate.MATE_ERR_NULL), (6, None, mate.MATE_ERR_NULL), (7, None, mate.MATE_ERR_NULL), (3, 0, mate.MATE_ERR_SHAPE),
        (4, 4, mate.MATE_ERR_UNSUPPORTED), (5, 2, mate.MATE_ERR_UNSUPPORTED), (6, FAKE + 8, mate.MATE_ERR_UNSUPPORTED)])
    ok = [FAKE, FAKE, 2, 100, 768, mate.MATE_F32, FAKE, None]            # codes, scales, B, N, E, t, x
    refuses(mate.mate_checkpoint_unpack, ok, [
        (0, None, mate.MATE_ERR_NULL), (1, None, mate.MATE_ERR_NULL), (6, None, mate.MATE_ERR_NULL), (2, -1, mate.MATE_ERR_SHAPE),
        (4, 20, mate.MATE_ERR_UNSUPPORTED), (5, 7, mate.MATE_ERR_UNSUPPORTED), (0, FAKE + 8, mate.MATE_ERR_UNSUPPORTED)])


def test_tensors_of_other_types_shapes_and_places():
    """Every tensor is looked at before its memory is; host tensors are refused last, so no kernel is launched."""
    B, N, E, F = 2, 5, 16, 24
    x, w, dy = torch.zeros(B, N, E, dtype=torch.bfloat16), torch.zeros(F, E, dtype=torch.bfloat16), torch.zeros(B, N, F, dtype=torch.bfloat16)
    for call in (lambda: mate.linear(x, w), lambda: mate.linear_bwd(dy, x, w), lambda: mate.activation_bwd(x, x, mate.MATE_ACT_RELU),
                 lambda: mate.checkpoint_pack(x),
                 lambda: mate.checkpoint_unpack(mate.Checkpoint(torch.zeros(B, N, E, dtype=torch.uint8), torch.zeros(B, N, 1, dtype=torch.uint8)))):
        with pytest.raises(ValueError, match="device tensors"):
            call()
    with pytest.raises(ValueError, match="B, N, width"):
        mate.linear(x[0], w)
    with pytest.raises(TypeError):
        mate.linear(None, w)
    with pytest.raises(ValueError, match="keep_z"):
        mate.linear(x, w, keep_z=3)
    with pytest.raises(TypeError, match="dtype"):
        mate.checkpoint_unpack(mate.Checkpoint(x, x), torch.float16)
    with pytest.raises(TypeError, match="dtype"):
        mate.checkpoint_pack(x.to(torch.float16))
    with pytest.raises(AttributeError):
        mate.checkpoint_unpack(x)
