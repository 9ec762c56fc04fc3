"""Host side of the operators around a block: descriptor checks that need no GPU."""
import ctypes

import pytest

from paper_2508_12594_b200 import build, flare


@pytest.fixture(scope="module")
def lib():
    build.build()
    return flare.load()


def desc(**kw):
    d = dict(rows=100, width=64, dtype=flare.DTYPE_BF16, residual_dtype=flare.DTYPE_BF16, pre_norm=flare.NORM_LAYER, post_norm=flare.NORM_RMS,
             gate=flare.GATE_SIGMOID, gate_rows=1, pre_eps=1e-5, post_eps=1e-5, residual_scale=1.0)
    return flare.FlareBlockDesc(**{**d, **kw})


def test_workspace_is_a_row_of_sums_per_thread_block(lib):
    need = lambda **kw: lib.flare_block_workspace_bytes(ctypes.byref(desc(**kw)))  # noqa: E731
    assert need() > 0
    assert need(rows=0) > 0
    # at most two blocks an SM, four sums of a row each
    assert need(rows=1 << 20) <= 2 * 148 * 4 * 64 * 4 + 256
    # wide rows add two floats a row; groups of rows that share a gate row never share a block
    assert need(rows=1 << 16, width=8192) <= 2 * 148 * 4 * 8192 * 4 + 8 * (1 << 16) + 512
    assert need(rows=1 << 12, gate_rows=2) >= (1 << 11) * 4 * 64 * 4


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(width=0), dict(width=16385), dict(dtype=3), dict(residual_dtype=flare.DTYPE_F16),
                                 dict(dtype=flare.DTYPE_F32), dict(pre_norm=3), dict(gate=3), dict(gate_rows=0), dict(gate_rows=3), dict(pre_eps=-1e-5),
                                 dict(post_eps=float("nan")), dict(residual_scale=float("inf")), dict(stride_x=63), dict(rows=1 << 31)], ids=str)
def test_invalid_descriptors(lib, bad):
    d = desc(**bad)
    assert lib.flare_block_workspace_bytes(ctypes.byref(d)) == 0
    rc = lib.flare_join_forward(ctypes.byref(d), *[None] * 12)
    assert rc in (flare.ERR_INVALID_ARG, flare.ERR_UNSUPPORTED)


def test_missing_tensors(lib):
    assert lib.flare_join_forward(ctypes.byref(desc()), *[None] * 12) == flare.ERR_INVALID_ARG
    assert lib.flare_norm_forward(ctypes.byref(desc()), *[None] * 6) == flare.ERR_INVALID_ARG
    assert lib.flare_norm_forward(ctypes.byref(desc(pre_norm=flare.NORM_NONE)), *[None] * 6) == flare.ERR_INVALID_ARG
    assert lib.flare_norm_backward(ctypes.byref(desc()), *[None] * 9, 0, None) == flare.ERR_INVALID_ARG
    assert lib.flare_join_backward(ctypes.byref(desc()), *[None] * 19, 0, None) == flare.ERR_INVALID_ARG
    assert lib.flare_join_forward(None, *[None] * 12) == flare.ERR_INVALID_ARG
