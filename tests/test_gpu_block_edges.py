"""Norms and joins around a block at the edges of what is asked of them (needs a B200)."""
import ctypes

import pytest
import torch

from paper_2508_12594_b200 import flare

pytestmark = pytest.mark.gpu


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
