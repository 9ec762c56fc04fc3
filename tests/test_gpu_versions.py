"""What a call writes in place counts as written for autograd (needs a B200)."""
import pytest
import torch

from paper_2508_12594_b200 import flare

pytestmark = pytest.mark.gpu


def test_tensors_that_are_written_have_a_new_version():
    x, o = torch.randn(2, 40, 64, device="cuda"), torch.randn(2, 40, 64, device="cuda")
    norm = flare.Norm("rms", torch.ones(64, device="cuda"))
    h, stats = torch.empty_like(x), torch.empty(80, 4, device="cuda")
    written = [torch.empty_like(x), torch.empty_like(norm.weight)]

    def version(ts):
        return [t._version for t in ts]

    before = version((x, h, stats, *written))
    flare.block_norm(x, norm, out=(h, stats))
    flare.block_norm_backward(x, stats, o, norm, out=(*written, None))
    assert version((x, h, stats, *written)) == [before[0]] + [v + 1 for v in before[1:]]
    v = x._version, h._version
    flare.block_join(x, o, pre=norm, out=(x, h, None))
    assert (x._version, h._version) == (v[0] + 1, v[1] + 1)
    v = o._version
    flare.block_join_backward(o, x, stats, None, h, pre=norm, out=(None, o) + (None,) * 6)
    assert o._version == v + 1
    w, m, g = (torch.randn(30, 50, device="cuda") for _ in range(3))
    v = version((w, m, g))
    flare.muon_update(w, m, g, lr=0.1)
    assert version((w, m, g)) == [v[0] + 1, v[1] + 1, v[2]]
    flare.orthogonalize(g, out=g)
    assert g._version == v[2] + 1


def test_a_weight_that_a_graph_still_wants_is_missed():
    w = torch.randn(30, 50, device="cuda", requires_grad=True)
    m, g = torch.zeros(30, 50, device="cuda"), torch.randn(30, 50, device="cuda")
    loss = (w * w).sum()
    flare.muon_update(w, m, g, lr=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_tensors_without_a_version():
    with torch.inference_mode():
        w, m, g = (torch.randn(30, 50, device="cuda") for _ in range(3))
    want = w.clone()
    flare.muon_update(w, m, g, lr=0.1)
    assert not torch.equal(w, want)
