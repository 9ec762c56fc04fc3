"""Host side of the token operators: the generator's known answers, descriptor checks that need no GPU."""
import ctypes

import pytest

from paper_2508_12594_b200 import build, flare
from tests import _tokens


@pytest.fixture(scope="module")
def lib():
    build.build()
    return flare.load()


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_the_generators_known_answers(counter, key, want):
    assert tuple(int(x) for x in _tokens.philox(counter, key)) == want


def dropout_desc(**kw):
    return flare.FlareDropoutDesc(**{**dict(rows=10, width=64, dtype=flare.DTYPE_BF16, residual_dtype=flare.DTYPE_F32), **kw})


def embed_desc(**kw):
    return flare.FlareEmbedDesc(**{**dict(rows=12, positions=0, width=64, vocab=100, dtype=flare.DTYPE_F32, out_dtype=flare.DTYPE_BF16, token_bits=64, scale=1.0), **kw})


def loss_desc(**kw):
    return flare.FlareLossDesc(**{**dict(rows=12, width=64, vocab=100, dtype=flare.DTYPE_BF16, label_bits=64, scale=1.0, dloss_scale=1.0), **kw})


DROP = flare.FlareDrop(0.1, 1, 2, None)
INVALID, UNSUPPORTED = flare.ERR_INVALID_ARG, flare.ERR_UNSUPPORTED


@pytest.mark.parametrize("bad,status", [(dict(rows=-1), INVALID), (dict(width=0), INVALID), (dict(stride_x=63), INVALID), (dict(stride_y=-1), INVALID),
                                        (dict(dtype=3), UNSUPPORTED), (dict(residual_dtype=flare.DTYPE_F16), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED), (dict(), INVALID)], ids=str)
def test_dropout_is_refused(lib, bad, status):
    """(The last: sound, but without tensors.)"""
    d = dropout_desc(**bad)
    assert lib.flare_dropout_forward(ctypes.byref(d), ctypes.byref(DROP), None, None, None, None) == status
    assert lib.flare_dropout_backward(ctypes.byref(d), ctypes.byref(DROP), None, None, None) == status


@pytest.mark.parametrize("p", [-0.1, 1.1, float("nan"), float("inf")])
def test_shares_that_are_none_are_refused(lib, p):
    drop = flare.FlareDrop(p, 1, 2, None)
    assert lib.flare_dropout_forward(ctypes.byref(dropout_desc(rows=0)), ctypes.byref(drop), None, None, None, None) == INVALID
    assert lib.flare_embed_forward(ctypes.byref(embed_desc(rows=0)), ctypes.byref(drop), None, 64, None, None, None) == INVALID
    assert lib.flare_dropout_forward(ctypes.byref(dropout_desc(rows=0)), None, None, None, None, None) == INVALID


@pytest.mark.parametrize("bad,status", [(dict(rows=-1), INVALID), (dict(width=0), INVALID), (dict(vocab=0), INVALID), (dict(positions=-1), INVALID), (dict(positions=5), INVALID),
                                        (dict(token_bits=16), INVALID), (dict(scale=float("nan")), INVALID), (dict(stride_table=63), INVALID), (dict(stride_out=1), INVALID),
                                        (dict(dtype=7), UNSUPPORTED), (dict(dtype=flare.DTYPE_F16), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED)], ids=str)
def test_embedding_is_refused(lib, bad, status):
    d = embed_desc(**bad)
    assert lib.flare_embed_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.flare_embed_forward(ctypes.byref(d), None, 64, 64, None, 64, None) == status
    assert lib.flare_embed_backward(ctypes.byref(d), None, 64, 64, 64, None, 0, 64, 0, None) == status


def test_embedding_without_its_tensors(lib):
    d, e = embed_desc(), embed_desc(positions=4)
    assert lib.flare_embed_workspace_bytes(ctypes.byref(d)) > 0
    assert lib.flare_embed_forward(ctypes.byref(d), None, None, 64, None, 64, None) == INVALID
    assert lib.flare_embed_forward(ctypes.byref(d), None, 64, None, None, 64, None) == INVALID
    assert lib.flare_embed_forward(ctypes.byref(d), None, 64, 64, 64, 64, None) == INVALID      # positions that the descriptor has none of
    assert lib.flare_embed_forward(ctypes.byref(e), None, 64, 64, None, 64, None) == INVALID    # and the other way round
    assert lib.flare_embed_forward(ctypes.byref(d), None, 68, 64, None, 64, None) == INVALID    # 64-bit tokens off 8 bytes
    assert lib.flare_embed_backward(ctypes.byref(d), None, 64, 64, 64, 64, 0, 64, 1 << 20, None) == INVALID
    assert lib.flare_embed_backward(ctypes.byref(d), None, 64, 64, 64, None, 0, None, 0, None) == INVALID
    assert lib.flare_embed_backward(ctypes.byref(d), None, 64, 64, 64, None, 0, 72, 1 << 20, None) == INVALID


@pytest.mark.parametrize("bad,status", [(dict(rows=-1), INVALID), (dict(width=0), INVALID), (dict(vocab=0), INVALID), (dict(label_bits=8), INVALID), (dict(scale=0.0), INVALID),
                                        (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID), (dict(dloss_scale=float("nan")), INVALID), (dict(stride_x=63), INVALID),
                                        (dict(stride_dw=63), INVALID), (dict(dtype=4), UNSUPPORTED), (dict(width=16385), UNSUPPORTED), (dict(vocab=(1 << 28) + 1), UNSUPPORTED),
                                        (dict(rows=(1 << 30) + 1), UNSUPPORTED)], ids=str)
def test_loss_is_refused(lib, bad, status):
    d = loss_desc(**bad)
    for backward in (0, 1):
        assert lib.flare_loss_workspace_bytes(ctypes.byref(d), backward) == 0
    assert lib.flare_loss_forward(ctypes.byref(d), 64, 64, 64, 64, 64, 64, 1 << 30, None) == status
    assert lib.flare_loss_backward(ctypes.byref(d), 64, 64, 64, 64, None, 64, 64, 64, 1 << 30, None) == status


def test_loss_without_its_tensors(lib):
    d = loss_desc()
    ok = [64, 64, 64, 64, 64, 64, 1 << 30]
    for i in range(6):
        assert lib.flare_loss_forward(ctypes.byref(d), *[None if j == i else v for j, v in enumerate(ok)], None) == INVALID
    ok = [64, 64, 64, 64, None, 64, 64, 64, 1 << 30]
    for i in (0, 1, 2, 3, 7):
        assert lib.flare_loss_backward(ctypes.byref(d), *[None if j == i else v for j, v in enumerate(ok)], None) == INVALID
    assert lib.flare_loss_backward(ctypes.byref(d), 64, 64, 64, 64, None, None, None, 64, 1 << 30, None) == INVALID     # neither gradient
    assert lib.flare_loss_forward(ctypes.byref(d), 65, 64, 64, 64, 64, 64, 1 << 30, None) == INVALID                   # off two bytes


def test_scratch_of_the_loss_is_bounded(lib):
    """Never rows x vocabulary: the piece of the weights is 512 MB, or 256 words of every row."""
    need = lambda back, **kw: lib.flare_loss_workspace_bytes(ctypes.byref(loss_desc(**kw)), back)  # noqa: E731
    rows, vocab, width = 8192, 128256, 1024
    packed = 2 * width * (rows + vocab)
    assert need(1, rows=rows, vocab=vocab, width=width) <= packed + (512 << 20) + 4 * rows * width + (48 << 20)
    assert need(0, rows=rows, vocab=vocab, width=width) <= packed + 16 * rows * (vocab // 256 + 1) + (1 << 20)
    # a million rows: 512 bytes each
    assert need(1, rows=1 << 20, vocab=vocab, width=64) <= (1 << 20) * (512 + 2 * 64 + 4 * 128 + 64) + 2 * vocab * 64 + (32 << 20)
