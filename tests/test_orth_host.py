"""Host side of the orthogonalised updates: descriptor checks that need no GPU."""
import ctypes

import pytest

from paper_2508_12594_b200 import build, flare


@pytest.fixture(scope="module")
def lib():
    build.build()
    return flare.load()


def desc(coefficients=flare.NEWTON_SCHULZ, **kw):
    d = dict(count=2, rows=300, cols=500, dtype=flare.DTYPE_BF16, weight_dtype=flare.DTYPE_F32, steps=5, eps=1e-7)
    return flare.FlareOrthDesc(coefficients=(ctypes.c_float * 3)(*coefficients), **{**d, **kw})


def test_workspace(lib):
    need = lambda **kw: lib.flare_orthogonalize_workspace_bytes(ctypes.byref(desc(**kw)))  # noqa: E731
    # two copies of X, A and B, in two 16-bit halves each, at most a tile of 128 x 128 sums per SM, and little else; nothing but the header for what one
    # thread block holds
    halves = 2 * 2 * 2 * (2 * 300 * 504 + 2 * 300 * 304)
    assert halves <= need() <= halves + 148 * 128 * 128 * 4 + (1 << 16)
    assert need(rows=128, cols=128) == 256 and need(rows=1024, cols=32) == 256
    assert need(rows=500, cols=300) == need()
    assert need(count=0) > 0


@pytest.mark.parametrize("bad", [dict(count=-1), dict(rows=0), dict(cols=0), dict(rows=65537), dict(rows=65536, cols=32768), dict(count=32768), dict(dtype=3),
                                 dict(weight_dtype=-1), dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=float("inf")), dict(stride_row=499),
                                 dict(coefficients=(float("nan"), 0.0, 0.0)), dict(coefficients=(4.0, 1.0, 1.0))], ids=str)
def test_invalid_descriptors(lib, bad):
    d = desc(**bad)
    assert lib.flare_orthogonalize_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.flare_orthogonalize(ctypes.byref(d), None, None, None, 0, None) in (flare.ERR_INVALID_ARG, flare.ERR_UNSUPPORTED)


def test_missing_tensors(lib):
    assert lib.flare_orthogonalize(ctypes.byref(desc()), None, None, None, 0, None) == flare.ERR_INVALID_ARG
    assert lib.flare_muon_update(ctypes.byref(desc()), None, *[None] * 6, 0, None) == flare.ERR_INVALID_ARG
    assert lib.flare_muon_update(ctypes.byref(desc()), ctypes.byref(flare.FlareMuon(0.1, 0.9, 0.0, 1.0, 1)), *[None] * 6, 0, None) == flare.ERR_INVALID_ARG
