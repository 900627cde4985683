"""A whole layer's training step through the public calls: projections, attention, output projection, feed-forward half, and all gradients back.  Every
product is held to 64 bits on what the call before it gave (the attention between them has tests of its own), and the attention to the oracle."""
import numpy as np
import pytest
import torch

from oracle import feed_forward as ff
from oracle import mate_oracle as orc
from paper_2109_04312_amd import synth
from tests.test_gpu_feed_forward import BF16, PAD, Inputs, close_8bit, feed_forward_step, pre_activation_error, sum_error, within

pytestmark = pytest.mark.gpu


def product(got, x, w, bias, flags, residual, what):
    """y = x w^T + bias + residual in bf16."""
    _, y = ff.linear(x, w, bias, flags, residual=residual)
    absolute = x.double().abs() @ w.double().abs().T
    for t in (bias, residual):
        if t is not None:
            absolute = absolute + t.double().abs()
    e = sum_error(x.shape[-1] + 2, absolute)
    within(got, y, e + BF16 * (y.abs() + e) + 1e-300, what)


def gradients(dx, dw, db, dy, x, w, flags, residual, what):
    wx, ww, wb = ff.linear_backward(dy, x, w, flags, residual=residual)
    g = ff.zero_pads(dy.double().abs(), flags)
    absolute = g @ w.double().abs() + (0.0 if residual is None else residual.double().abs())
    e = sum_error(w.shape[0] + 1, absolute)
    within(dx, wx, e + BF16 * (wx.abs() + e) + 1e-300, "dx of " + what)
    rows, flat = g.shape[0] * g.shape[1], g.reshape(-1, g.shape[-1])
    within(dw, ww, sum_error(rows, flat.T @ ff.zero_pads(x.double().abs(), flags).reshape(-1, x.shape[-1])) + 1e-300, "dw of " + what)
    if db is not None:
        within(db, wb, sum_error(rows, flat.sum(0)) + 1e-300, "dbias of " + what)


def tokens(t):   # [B, H, N, 64] -> [B, N, 64 H]
    return t.transpose(1, 2).flatten(2)


@pytest.mark.parametrize("eight", [False, True])
def test_training_step(eight):
    from paper_2109_04312_amd import mate
    B, N, H, F = 2, 300, 4, 1000
    E = 64 * H
    rng = np.random.default_rng(3)
    st = synth.random_structure(rng, B, N, max_rows=10, max_cols=5, max_global=12, max_cell=4)
    r, c, f = (torch.from_numpy(t).cuda() for t in (st.row_ids, st.col_ids, st.flags))
    kinds = synth.half_row_half_col(H)
    i = Inputs(5, B, N, E, F, None)
    x = i.x
    w_qkv, w_o, w2 = i.normal(3 * E, E, scale=E ** -0.5), i.normal(E, E, scale=E ** -0.5), i.normal(E, F, scale=F ** -0.5)
    b_qkv, b_o, b2 = (i.normal(n, dtype=torch.float32) for n in (3 * E, E, E))
    dy = i.normal(B, N, E)
    seg = mate.build_segments(r, c, f)
    q, k, v = mate.qkv_project(x, w_qkv, b_qkv, f, H)
    o, lse = mate.attn_fwd(q, k, v, seg, kinds, 0.125)
    a = mate.out_project(o, w_o, b_o, f)
    got = feed_forward_step(mate, a, i.w, i.bias, w2, b2, f, dy, eight, mate.MATE_ACT_GELU)
    d_o, dw_o, db_o = mate.out_project_bwd(o, w_o, f, got["dx"])
    dq, dk, dv = mate.attn_bwd(q, k, v, o, lse, d_o, seg, kinds, 0.125)
    dx, dw_qkv, db_qkv = mate.qkv_project_bwd(x, w_qkv, f, dq, dk, dv)
    torch.cuda.synchronize()

    product(torch.cat([tokens(t) for t in (q, k, v)], -1), x, w_qkv, b_qkv, f, None, "q, k, v")
    host = lambda t: t.float().cpu().numpy()
    want = orc.attn_forward(host(q), host(k), host(v), st.row_ids, st.col_ids, st.flags, kinds, 0.125)[0]
    assert float(np.abs(host(o) - want).max()) <= 2e-2
    product(a, tokens(o), w_o, b_o, f, None, "the attention's output")
    # the feed-forward half: h, z, y and every gradient of its two products
    value = lambda t: ff.values(t.codes, t.scales) if isinstance(t, mate.Checkpoint) else t.double()
    z, _ = ff.linear(a, i.w, i.bias, f, "gelu")
    i.x = a
    ez = torch.where(ff.live(f, z), pre_activation_error(i), 0.0)
    if eight:
        close_8bit(got["z"], z, ez, "z")
    else:
        within(got["z"], z, ez + BF16 * (z.abs() + ez) + 1e-300, "z")
    product(got["y"], got["h"], w2, b2, f, a, "y")
    z, h8 = value(got["z"]), value(got["h8"])
    dz, dw2, db2 = ff.linear_backward(dy, h8, w2, f, z, "gelu")
    raw = dy.double().abs() @ w2.double().abs()
    e = (1.2 + 2.0 ** -20) * sum_error(E, raw) + 2.0 ** -20 * (1 + z.abs()) * raw + 2.0 ** -24 * dz.abs()
    within(got["dz"], dz, e + BF16 * (dz.abs() + e) + 1e-300, "dz")
    g = ff.zero_pads(dy.double().abs(), f).reshape(-1, E)
    within(got["dw2"], dw2, sum_error(B * N, g.T @ h8.abs().reshape(-1, F)) + 1e-300, "dw2")
    within(got["db2"], db2, sum_error(B * N, g.sum(0)) + 1e-300, "db2")
    gradients(got["dx"], got["dw1"], got["db1"], got["dz"], value(got["x8"]), i.w, f, dy, "the first product")
    # and on through the attention
    gradients(tokens(d_o), dw_o, db_o, got["dx"], tokens(o), w_o, f, None, "the attention's output")
    gradients(dx, dw_qkv, db_qkv, torch.cat([tokens(t) for t in (dq, dk, dv)], -1), x, w_qkv, f, None, "q, k, v")
    pad = f == PAD
    assert bool(pad.any()) and not any(bool(t[pad].any()) for t in (a, got["y"], got["dz"], got["dx"], dx))
