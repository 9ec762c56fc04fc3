"""Orthogonalised updates at the edges of what is asked of them (needs a B200)."""
import ctypes

import pytest
import torch

from paper_2508_12594_b200 import flare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(8, 12), (300, 500)])
def test_no_matrices_report_nothing(rows, cols):
    """Whatever the workspace held before: a call without matrices leaves a header that says that no wait gave up."""
    lib = flare.load()
    desc = flare.FlareOrthDesc(count=0, rows=rows, cols=cols, steps=5, coefficients=(ctypes.c_float * 3)(*flare.NEWTON_SCHULZ), eps=1e-7)
    need = lib.flare_orthogonalize_workspace_bytes(ctypes.byref(desc))
    rule = flare.FlareMuon(0.1, 0.9, 0.0, 1.0, 1)
    for call in (lambda p: lib.flare_orthogonalize(ctypes.byref(desc), None, None, p, need, None),
                 lambda p: lib.flare_muon_update(ctypes.byref(desc), ctypes.byref(rule), None, None, None, None, None, p, need, None)):
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        assert call(ctypes.c_void_p(ws.data_ptr())) == flare.OK
        flare.flare_check(ws)
    none = torch.empty(0, rows, cols, device="cuda")
    assert flare.orthogonalize(none, check=True).shape == none.shape
    flare.muon_update(none, none, none, lr=0.1, check=True)


def test_steps_beyond_32_bits_are_not_taken_for_others():
    """2^32 + 5 is not 5."""
    for steps, status in ((2 ** 32 + 5, flare.ERR_UNSUPPORTED), (-2 ** 32 + 5, flare.ERR_INVALID_ARG)):
        with pytest.raises(flare.FlareError) as e:
            flare.orthogonalize(torch.zeros(8, 12, device="cuda"), steps=steps)
        assert e.value.status == status


def test_updates_of_what_is_no_matrix_are_refused_as_that():
    v, none = torch.zeros(12, device="cuda"), torch.zeros(5, 0, device="cuda")
    with pytest.raises(ValueError, match="matrices"):
        flare.muon_update(v, v, v, lr=0.1)
    with pytest.raises(flare.FlareError) as e:
        flare.muon_update(none, none, none, lr=0.1)
    assert e.value.status == flare.ERR_INVALID_ARG
