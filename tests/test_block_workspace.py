"""Host side of the operators around a block: the size of a backward's workspace for whichever of the two is called with the descriptor."""
import ctypes

import pytest

from paper_2508_12594_b200 import build, flare


@pytest.fixture(scope="module")
def lib():
    build.build()
    return flare.load()


@pytest.mark.parametrize("rows", [0, 1024, 131072, 1 << 20])
@pytest.mark.parametrize("width", [128, 333, 4096])
@pytest.mark.parametrize("gate_rows", [1, 2, 1024])
def test_a_gate_does_not_take_room_from_the_norm(lib, rows, width, gate_rows):
    """flare_norm_backward does not look at the gate: what the gated descriptor is told is at least what the same one without it is."""
    def need(gate):
        d = flare.FlareBlockDesc(rows=rows, width=width, dtype=flare.DTYPE_BF16, residual_dtype=flare.DTYPE_BF16, pre_norm=flare.NORM_RMS,
                                 post_norm=flare.NORM_NONE, gate=gate, gate_rows=gate_rows, pre_eps=1e-5, post_eps=0.0, residual_scale=1.0)
        return lib.flare_block_workspace_bytes(ctypes.byref(d))
    assert need(flare.GATE_SIGMOID) >= need(flare.GATE_NONE) > 0
