"""Calls of the token operators as a program makes them: on other streams, captured, one behind the other without a pause, into tensors that are given, and calls that are refused
(needs a B200)."""
import pytest
import torch

from paper_2508_12594_b200 import flare
from tests._tokens import close, factors, stored

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def inputs(seed=3, V=5000, B=4, L=500, C=96, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*s, dtype=dtype):
        return torch.randn(*s, device="cuda", generator=g).to(dtype)

    t = torch.randint(-1, V, (B, L), device="cuda", generator=g)
    table, pos, dy, x, res = randn(V, C), randn(L, C), randn(B, L, C), randn(B, L, C), randn(B, L, C, dtype=torch.float32)
    labels = torch.randint(-1, V, (B, L), device="cuda", generator=g)
    few = labels[0, :3].clamp(min=0).contiguous()
    d = flare.Drop(0.3, 17, 4)
    lse = flare.token_loss(x, table, labels)[1]
    return {
        "dropout": lambda stream=None: [flare.dropout(x, d, residual=res, stream=stream)],
        "dropout backward": lambda stream=None: [flare.dropout_backward(res, d, dtype=dtype, stream=stream)],
        "embed": lambda stream=None: [flare.embed(t, table, positions=pos, scale=2.0, drop=d, stream=stream)],
        "embed backward": lambda stream=None: flare.embed_backward(t, dy, V, positions=L, scale=2.0, drop=d, stream=stream),
        "embed backward of a large table": lambda stream=None: [flare.embed_backward(t, dy, 200_000, dtype=torch.float32 if dtype == BF16 else dtype, stream=stream).dtable],
        "loss": lambda stream=None: flare.token_loss(x, table, labels, stream=stream),
        "loss of a few rows": lambda stream=None: flare.token_loss(x[0, :3], table, few, stream=stream),
        "loss of one tile of rows": lambda stream=None: flare.token_loss(x[0, :200], table, labels[0, :200].contiguous(), stream=stream),
        "loss backward": lambda stream=None: flare.token_loss_backward(x, table, labels, lse, stream=stream),
    }


CALLS = tuple(["dropout", "dropout backward", "embed", "embed backward", "embed backward of a large table", "loss", "loss of a few rows", "loss of one tile of rows", "loss backward"])


def _stream_of(t):
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]


@pytest.mark.parametrize("name", CALLS)
def test_results_are_of_the_calls_stream(name):
    call = inputs()[name]
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = list(call(side))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want, strict=True))
    assert {_stream_of(t) for t in got} == {side.cuda_stream}


@pytest.mark.parametrize("name", CALLS)
def test_captured_and_replayed(name):
    call = inputs()[name]
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = list(call())
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want, strict=True))


def test_one_behind_the_other():
    """All calls in changing order without a pause between them, on inputs of several shapes: the same, bit for bit, as one at a time."""
    sets = [inputs(3), inputs(4, V=300, B=1, L=1000, C=32), inputs(5, V=20000, B=2, L=77, C=130), inputs(6, V=1500, B=3, L=300, C=64, dtype=torch.float32)]
    want = []
    for s in sets:
        for name in CALLS:
            want.append([t.clone() for t in s[name]()])
            torch.cuda.synchronize()
    order = list(range(len(want)))
    for turn in range(3):
        got = {i: list(sets[i // len(CALLS)][CALLS[i % len(CALLS)]]()) for i in order}
        torch.cuda.synchronize()
        for i in order:
            assert all(torch.equal(a, b) for a, b in zip(got[i], want[i], strict=True)), (turn, i // len(CALLS), CALLS[i % len(CALLS)])
        order = order[5:] + order[:5] if turn else order[::-1]


def test_on_two_streams_at_once():
    sets = [inputs(3), inputs(4, V=3000, L=700)]
    want = [[[t.clone() for t in s[name]()] for name in CALLS] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[None] * len(CALLS) for _ in sets]
    for i, name in enumerate(CALLS):
        for k, (s, stream) in enumerate(zip(sets, streams)):
            got[k][i] = list(s[name](stream))
    torch.cuda.synchronize()
    for k in range(2):
        for i, name in enumerate(CALLS):
            assert all(torch.equal(a, b) for a, b in zip(got[k][i], want[k][i], strict=True)), (k, name)


def test_what_follows_a_gradient_sees_all_of_it():
    """The zeros of a large table are written beside the sums: a copy right behind the call has them."""
    g = torch.Generator(device="cuda").manual_seed(1)
    V, C = 60000, 512
    for n in (1, 40, 3000):
        t = torch.randint(0, V, (n,), device="cuda", generator=g)
        dy = torch.randn(n, C, device="cuda", generator=g)
        want = torch.zeros(V, C, dtype=torch.float64, device="cuda").index_add_(0, t, dy.double())
        out = torch.empty(V, C, device="cuda")
        for _ in range(4):
            out.fill_(float("nan"))
            flare.embed_backward(t, dy, V, out=(out, None))
            copy = out.clone()
            flare.dropout(copy, flare.Drop(0.0, 1), out=out)
            assert not copy.isnan().any()
            assert (copy.double() - want).abs().max() <= 8 * 2.0 ** -24 * want.abs().max()


def test_tensors_that_are_written_have_a_new_version():
    x, t = torch.randn(3, 40, 64, device="cuda"), torch.randint(0, 90, (3, 40), device="cuda")
    table, d = torch.randn(90, 64, device="cuda"), flare.Drop(0.2, 1)
    y, dt, dp, loss, lse, dx, dw = (torch.empty(s, device="cuda") for s in ((3, 40, 64), (90, 64), (40, 64), (3, 40), (3, 40), (3, 40, 64), (90, 64)))
    all_of_them = [x, t, table, y, dt, dp, loss, lse, dx, dw]
    before = [v._version for v in all_of_them]
    flare.dropout(x, d, out=y)
    flare.embed(t, table, out=y)
    flare.embed_backward(t, x, 90, positions=40, out=(dt, dp))
    flare.token_loss(x, table, t, out=(loss, None))
    flare.token_loss(x, table, t, out=(None, lse))
    flare.token_loss_backward(x, table, t, lse, out=(dx, dw))
    assert [v._version - b for v, b in zip(all_of_them, before)] == [0, 0, 0, 2, 1, 1, 1, 1, 1, 1]


def test_inputs_of_a_graph_and_scalars():
    """Inputs are taken without their graph; a single token without a leading dimension."""
    table = torch.randn(50, 24, device="cuda", requires_grad=True)
    y = flare.embed(torch.tensor(7, device="cuda"), table)
    assert y.shape == (24,) and not y.requires_grad and torch.equal(y, table.detach()[7])
    loss, lse = flare.token_loss(y, table, torch.tensor(3, device="cuda"))
    assert loss.shape == ()
    ref = torch.nn.functional.cross_entropy((table.detach().double() @ y.double())[None], torch.tensor([3], device="cuda"))
    assert abs(float(loss) - float(ref)) <= 1e-5
    d = flare.token_loss_backward(y, table, torch.tensor(3, device="cuda"), lse)
    assert d.dx.shape == (24,)


def test_the_largest_seeds():
    x = torch.ones(40, 16, device="cuda")
    for seed, offset in ((2 ** 64 - 1, 2 ** 64 - 1), (0, 0), (1 << 63, 1 << 32)):
        close(flare.dropout(x, flare.Drop(0.5, seed, offset)), factors(40, 16, 0.5, seed, offset).cuda(), stored(torch.float32, x.double()))


@pytest.mark.parametrize("call,error", [
    (lambda x, t, w: flare.dropout(x, None), flare.FlareError),
    (lambda x, t, w: flare.dropout(x, flare.Drop(1.5, 1)), flare.FlareError),
    (lambda x, t, w: flare.dropout(x, flare.Drop(0.5, -1)), OverflowError),
    (lambda x, t, w: flare.dropout(x, flare.Drop(0.5, 1 << 64)), OverflowError),
    (lambda x, t, w: flare.dropout(x, flare.Drop(0.5, 1, 0, t)), TypeError),
    (lambda x, t, w: flare.dropout(x, flare.Drop(0.5, 1, 0, torch.zeros(1, dtype=torch.int64))), ValueError),
    (lambda x, t, w: flare.dropout(x, (0.5, 1)), TypeError),
    (lambda x, t, w: flare.dropout(x, flare.Drop(0.5, 1), residual=x.half()), flare.FlareError),
    (lambda x, t, w: flare.dropout_backward(x.half(), flare.Drop(0.5, 1), dtype=torch.float32), flare.FlareError),
    (lambda x, t, w: flare.dropout(x.double(), flare.Drop(0.5, 1)), TypeError),
    (lambda x, t, w: flare.dropout(x.transpose(0, 1), flare.Drop(0.5, 1)), ValueError),
    (lambda x, t, w: flare.dropout(x, flare.Drop(0.5, 1), out=x[:, :8]), ValueError),
    (lambda x, t, w: flare.dropout(x.cpu(), flare.Drop(0.5, 1)), ValueError),
    (lambda x, t, w: flare.embed(t.float(), w), TypeError),
    (lambda x, t, w: flare.embed(t.cpu(), w), ValueError),
    (lambda x, t, w: flare.embed(t[::2], w), ValueError),
    (lambda x, t, w: flare.embed(t, w[0]), ValueError),
    (lambda x, t, w: flare.embed(t, w, positions=w), ValueError),
    (lambda x, t, w: flare.embed(t, w, positions=x.half()), TypeError),
    (lambda x, t, w: flare.embed(t, w, scale=float("nan")), flare.FlareError),
    (lambda x, t, w: flare.embed(t, w.half(), dtype=BF16), flare.FlareError),
    (lambda x, t, w: flare.embed(t, w, dtype=torch.float64), TypeError),
    (lambda x, t, w: flare.embed_backward(t, x, 0), ValueError),
    (lambda x, t, w: flare.embed_backward(t, x[:5], 30), ValueError),
    (lambda x, t, w: flare.embed_backward(t, x, 30, positions=7), ValueError),
    (lambda x, t, w: flare.embed_backward(t, x, 30, accumulate=True), ValueError),
    (lambda x, t, w: flare.embed_backward(t, x, 30, out=(w.T, None)), ValueError),
    (lambda x, t, w: flare.embed_backward(t, x, 30, out=(w[:29], None)), ValueError),
    (lambda x, t, w: flare.token_loss(x, w[:, :8], t), ValueError),
    (lambda x, t, w: flare.token_loss(x, w.half(), t), TypeError),
    (lambda x, t, w: flare.token_loss(x, w, t[:5]), ValueError),
    (lambda x, t, w: flare.token_loss(x, w, t.float()), TypeError),
    (lambda x, t, w: flare.token_loss(x, w, t, scale=0.0), flare.FlareError),
    (lambda x, t, w: flare.token_loss(x, w, t, scale=float("nan")), flare.FlareError),
    (lambda x, t, w: flare.token_loss(x, w, t, out=(x, None)), ValueError),
    (lambda x, t, w: flare.token_loss(x.cpu(), w, t), ValueError),
    (lambda x, t, w: flare.token_loss_backward(x, w, t, x[:, 0]), ValueError),
    (lambda x, t, w: flare.token_loss_backward(x, w, t, x[:, 0].contiguous(), dloss=x[:, 0].double()), (TypeError, ValueError)),
    (lambda x, t, w: flare.token_loss_backward(x, w, t, x[:, 0].contiguous(), dloss=float("inf")), flare.FlareError),
    (lambda x, t, w: flare.token_loss_backward(x, w, t, x[:, 0].contiguous(), dloss="1"), TypeError)], ids=str)
def test_refused(call, error):
    x, t, w = torch.randn(20, 16, device="cuda"), torch.randint(0, 30, (20,), device="cuda"), torch.randn(30, 16, device="cuda")
    kept = x.clone(), t.clone(), w.clone()
    with pytest.raises(error):
        call(x, t, w)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((x, t, w), kept))


def test_rows_that_are_all_the_same_place_are_refused():
    """Expanded tensors, one row in memory under many: not read as rows behind one another."""
    row, t, w = torch.zeros(64, dtype=BF16, device="cuda"), torch.zeros(2, 300, dtype=torch.int64, device="cuda"), torch.zeros(10, 64, dtype=BF16, device="cuda")
    items = torch.zeros(2, 1, 64, dtype=BF16, device="cuda").expand(2, 300, 64)
    for x in (row.expand(2, 300, 64), items, row.expand(1, 300, 64).expand(2, 300, 64)):
        for call in (lambda: flare.token_loss(x, w, t), lambda: flare.embed_backward(t, x, 10), lambda: flare.dropout(x, flare.Drop(0.1, 1, 1)), lambda: flare.dropout_backward(x, flare.Drop(0.1, 1, 1)),
                     lambda: flare.token_loss(torch.zeros(2, 300, 64, dtype=BF16, device="cuda"), row.expand(10, 64), t),
                     lambda: flare.embed(t, row.expand(10, 64))):
            with pytest.raises(ValueError):
                call()
    # one row is a row whatever its strides say
    one = row.as_strided((1, 64), (0, 1))
    assert flare.token_loss(one, w, t[0, :1])[0].shape == (1,)


def test_matrices_that_are_all_the_same_place_are_refused():
    m = torch.zeros(3, 1, 16, 16, device="cuda")
    for g in (m.expand(3, 2, 16, 16), m[:1, 0].expand(4, 16, 16)):
        with pytest.raises(ValueError):
            flare.orthogonalize(g)
