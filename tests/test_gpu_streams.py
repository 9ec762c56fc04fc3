"""Whose memory the results of the one-line calls are, where a call is given a stream that is not the current one (needs a B200).

Results are written by kernels on the call's stream, so they come from its share of the allocator's memory: what the current stream has just given back
may still be used by work queued there, and what the caller drops may still be written.
"""
import pytest
import torch

from paper_2508_12594_b200 import flare, workloads
from tests._util import dev

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _inputs():
    g = torch.Generator(device="cuda").manual_seed(3)

    def randn(*s, dtype=BF16):
        return torch.randn(*s, device="cuda", generator=g).to(dtype)

    x, o, gate, dy, dh = (randn(4, 500, 256) for _ in range(5))
    norm = flare.Norm("layer", randn(256, dtype=torch.float32), randn(256, dtype=torch.float32))
    s = randn(256, dtype=torch.float32)
    y, h, stats = flare.block_join(x, o, post=norm, pre=norm, gate=gate, scale=s)
    w = randn(3, 150, 300, dtype=torch.float32)
    inp = workloads.make_random(1, 2, 3000, 64, 32, dtype="bf16", seed=3, with_dy=True)
    Q, K, V, dY = dev(inp.Q), dev(inp.K), dev(inp.V), dev(inp.dY)
    return {
        "norm": lambda stream=None: flare.block_norm(x, norm, stream=stream),
        "norm backward": lambda stream=None: flare.block_norm_backward(y, stats, dh, norm, dy=dy, stream=stream),
        "join": lambda stream=None: flare.block_join(x, o, post=norm, pre=norm, gate=gate, scale=s, stream=stream),
        "join backward": lambda stream=None: flare.block_join_backward(o, y, stats, dy, dh, post=norm, pre=norm, gate=gate, scale=s, stream=stream),
        "orthogonalize": lambda stream=None: [flare.orthogonalize(w, stream=stream)],
        "mixer": lambda stream=None: [flare.forward(Q, K, V, stream=stream)],
        "mixer with statistics": lambda stream=None: flare.forward(Q, K, V, want_stats=True, stream=stream),
        "mixer step": lambda stream=None: flare.forward_backward(Q, K, V, dY, stream=stream),
    }


CALLS = ("norm", "norm backward", "join", "join backward", "orthogonalize", "mixer", "mixer with statistics", "mixer step")


def _stream_of(t):
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]


@pytest.mark.parametrize("name", CALLS)
def test_results_are_of_the_calls_stream(name):
    call = _inputs()[name]
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = list(call(side))
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want, strict=True))
    assert {_stream_of(t) for t in got} == {side.cuda_stream}


@pytest.mark.parametrize("name", CALLS)
def test_memory_given_back_on_the_current_stream_is_not_written_while_in_use(name):
    call = _inputs()[name]
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    old = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                                # some 50 ms, and behind it the last use of `old`
    for t in old:
        t.fill_(float("nan"))
    del old, t
    got = call(side)
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want, strict=True))


@pytest.mark.parametrize("name", CALLS)
def test_results_that_are_dropped_are_not_written_over_what_comes_next(name):
    call = _inputs()[name]
    shapes = [(t.shape, t.dtype) for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    call(side)                                                    # (its results are gone before its kernels have begun)
    fresh = [torch.zeros(s, dtype=d, device="cuda") for s, d in shapes]
    torch.cuda.synchronize()
    assert all((t == 0).all() for t in fresh)


@pytest.mark.parametrize("name", CALLS)
def test_results_in_use_on_the_current_stream_are_not_handed_on(name):
    """A result of another stream that the current one still reads when it is dropped."""
    call = _inputs()[name]
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = list(call(side))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(100_000_000)
    kept = [t.clone() for t in got]                               # queued behind the wait
    shapes = [(t.shape, t.dtype) for t in got]
    del got
    with torch.cuda.stream(side):
        over = [torch.full(s, float("nan"), dtype=d, device="cuda") for s, d in shapes]
    torch.cuda.synchronize()
    assert len(over) == len(kept) and all(torch.equal(k, w) for k, w in zip(kept, want))


def test_without_statistics():
    """An inference call need not have the statistics of its rows."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, o = (torch.randn(3, 70, 96, device="cuda", generator=g, dtype=BF16) for _ in range(2))
    norm = flare.Norm("rms", eps=1e-6)
    h, stats = flare.block_norm(x, norm, want_stats=False)
    assert stats is None and torch.equal(h, flare.block_norm(x, norm)[0])
    y, h, stats = flare.block_join(x, o, post=norm, pre=norm, want_stats=False)
    a, b, _ = flare.block_join(x, o, post=norm, pre=norm)
    assert stats is None and torch.equal(y, a) and torch.equal(h, b)
    with pytest.raises(ValueError, match="stats"):
        flare.block_norm(x, norm, out=(None, torch.empty(210, 4, device="cuda")), want_stats=False)
