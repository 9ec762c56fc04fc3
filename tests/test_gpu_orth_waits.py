"""Waits of the blocks that orthogonalise a matrix together: one that gives up ends them all, with a status (needs a B200)."""
import pytest
import torch

from paper_2508_12594_b200 import flare

pytestmark = pytest.mark.gpu


def _run(gone):
    ws = torch.full((512,), 255, dtype=torch.uint8, device="cuda")
    flare.flare_selftest_team(ws, gone, 1_000_000)               # one millisecond
    torch.cuda.synchronize()
    words = ws.view(torch.int32)
    return ws, words[65:65 + 24].view(2, 12).tolist(), words[89:91].tolist()


def test_blocks_that_all_come_go_on():
    ws, saw, waited = _run(0)
    assert max(waited) < 500_000
    flare.flare_check(ws)
    assert saw == [[3] * 12] * 2


def test_a_warp_that_gave_up_takes_the_others_with_it():
    """Its block's result warps agree not to go on instead of waiting for it; the block leaves at the first meeting, the other one at the second."""
    ws, saw, waited = _run(1)
    assert waited[0] >= 1_000_000                                # for what it might have had in flight
    assert saw == [[1] * 4 + [0] * 8, [1] * 12]
    with pytest.raises(flare.FlareError) as e:
        flare.flare_check(ws)
    assert e.value.status == flare.ERR_TIMEOUT


def test_a_block_that_never_comes():
    ws, saw, _ = _run(2)
    assert saw == [[1] * 12] * 2
    with pytest.raises(flare.FlareError) as e:
        flare.flare_check(ws)
    assert e.value.status == flare.ERR_TIMEOUT


def test_refusals():
    ws = torch.zeros(512, dtype=torch.uint8, device="cuda")
    for gone in (-1, 3):
        with pytest.raises(flare.FlareError) as e:
            flare.flare_selftest_team(ws, gone, 1000)
        assert e.value.status == flare.ERR_INVALID_ARG
