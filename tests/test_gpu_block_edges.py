"""Norms and joins around a block at the edges of what is asked of them (needs a B200)."""
import ctypes

import pytest
import torch

from paper_2508_12594_b200 import flare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["sigmoid", "linear"])
def test_items_without_rows(kind):
    """A gate row an item, and no rows: nothing comes out, and the sums over rows, the gate's gradient among them, are zeros."""
    x = torch.empty(3, 0, 64, device="cuda", dtype=torch.bfloat16)
    gate = torch.randn(3, 64, device="cuda").bfloat16()
    w, s = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    norm = flare.Norm("rms", w)
    y, h, stats = flare.block_join(x, x, post=norm, pre=norm, gate=gate, gate_kind=kind, scale=s)
    assert y.shape == h.shape == x.shape and stats.shape == (0, 4)
    for out in (None, torch.full((3, 80), 7.0, device="cuda", dtype=torch.bfloat16)):
        r = flare.block_join_backward(x, y, stats, None, h, post=norm, pre=norm, gate=gate, gate_kind=kind, scale=s,
                                      out=None if out is None else (None, None, out[:, :64]) + (None,) * 5)
        assert r.dgate.shape == gate.shape and (r.dgate == 0).all()
        assert all((g == 0).all() for g in (r.dscale, r.dpost_weight, r.dpre_weight))
        assert out is None or (out[:, 64:] == 7).all()


def test_norm_backward_with_the_workspace_of_a_gated_descriptor():
    """The gate of a descriptor is not looked at by the norm, so the size that the descriptor is told has to do for it too."""
    lib = flare.load()
    rows, width = 131072, 128
    desc = flare.FlareBlockDesc(rows=rows, width=width, dtype=flare.DTYPE_BF16, residual_dtype=flare.DTYPE_BF16, pre_norm=flare.NORM_RMS,
                                post_norm=flare.NORM_NONE, gate=flare.GATE_SIGMOID, gate_rows=1024, pre_eps=1e-5, post_eps=0.0, residual_scale=1.0)
    x = torch.randn(rows, width, device="cuda").bfloat16()
    dh = torch.randn(rows, width, device="cuda").bfloat16()
    w = torch.rand(width, device="cuda") + 0.5
    norm = flare.Norm("rms", w)
    _, stats = flare.block_norm(x, norm)
    want = flare.block_norm_backward(x, stats, dh, norm)
    need = lib.flare_block_workspace_bytes(ctypes.byref(desc))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    p = [ctypes.c_void_p(t.data_ptr()) for t in (x, w, stats, dh, dx, dw, ws)]
    rc = lib.flare_norm_backward(ctypes.byref(desc), p[0], p[1], p[2], None, p[3], p[4], p[5], None, p[6], need, None)
    torch.cuda.synchronize()
    assert rc == flare.OK and torch.equal(dx, want.dx) and torch.equal(dw, want.dweight)
