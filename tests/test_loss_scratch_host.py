"""Scratch of the loss over a vocabulary: no place for copies that no call makes (no GPU needed)."""
import ctypes

import pytest

from paper_2508_12594_b200 import build, flare

ALIGNED = 2                                                   # FLARE_LOSS_ALIGNED


@pytest.fixture(scope="module")
def need():
    build.build()
    lib = flare.load()

    def bytes_of(backward, **kw):
        d = flare.FlareLossDesc(**{**dict(rows=8192, width=1024, vocab=128256, dtype=flare.DTYPE_BF16, label_bits=64, scale=1.0, dloss_scale=1.0), **kw})
        return lib.flare_loss_workspace_bytes(ctypes.byref(d), backward)

    return bytes_of


@pytest.mark.parametrize("backward", [0, 1])
def test_no_copy_of_aligned_weights(need, backward):
    w = 2 * 1024 * 128256
    assert w <= need(backward) - need(backward | ALIGNED) <= w + 256
    assert need(backward, dtype=flare.DTYPE_F16) - need(backward | ALIGNED, dtype=flare.DTYPE_F16) >= w
    for kw in (dict(dtype=flare.DTYPE_F32), dict(stride_w=1028), dict(width=1020)):                     # packed wherever they begin
        assert need(backward, **kw) == need(backward | ALIGNED, **kw) > 0


def test_no_copies_where_rows_are_scored_as_they_stand(need):
    small = dict(vocab=2048, rows=100000, width=512)
    x, w = 2 * 512 * 100000, 2 * 512 * 2048
    assert need(0, **small) - need(ALIGNED, **small) >= x + w
    assert need(ALIGNED, **small) <= 100352 * (8 * 16 + 8 + 12) + (1 << 20)                             # parts, rows' numbers
    for rows in (1, 4, 8):
        assert need(0, rows=rows, dtype=flare.DTYPE_F32) <= 4 << 20


def test_enough_wherever_they_begin(need):
    """Five to eight aligned rows are scored by other kernels than unaligned ones, whose parts are fewer."""
    for dtype in (flare.DTYPE_BF16, flare.DTYPE_F16):
        for rows in (1, 5, 8, 9, 256, 300):
            for vocab in (5, 2000, 1 << 20):
                for backward in (0, 1):
                    kw = dict(rows=rows, vocab=vocab, width=8, dtype=dtype)
                    assert need(backward, **kw) >= need(backward | ALIGNED, **kw)
