"""Embedding, its gradient, and dropout against 64-bit implementations (needs a B200).

Bounds: a stored value is off by half a step of its type; float32 arithmetic in between by half a step of float32 for every operation, relative to the
magnitudes it adds up (a sum of k values: k steps of the sum of their magnitudes, whatever the order).
"""
import pytest
import torch

from paper_2508_12594_b200 import flare
from tests._tokens import U32, close, factors, rows_at, stored

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
PAIRS = [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32)]          # x, residual stream
TABLES = PAIRS + [(F32, BF16), (F32, F16)]                                       # table, rows


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


SEED, OFFSET = 0x9E3779B97F4A7C15, 0x1_0000_0003


def held(y, kept):
    """Nothing but zeros where nothing is kept."""
    assert (y[(kept == 0).to(y.device)] == 0).all()


@pytest.mark.parametrize("types", PAIRS, ids=str)
@pytest.mark.parametrize("rows,width,stride,offset", [(1, 1, 1, 0), (3, 7, 7, 0), (1000, 8, 8, 0), (257, 333, 333, 0), (70, 520, 528, 8), (70, 520, 521, 1), (5, 4104, 4104, 0)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.75, 1.0])
def test_dropout(types, rows, width, stride, offset, p):
    T, R = types
    g = gen(rows + width)
    x, res = rows_at(randn(g, rows, width, dtype=T), stride, offset), rows_at(randn(g, rows, width, dtype=R), stride, offset)
    d = flare.Drop(p, SEED, OFFSET)
    f = factors(rows, width, p, SEED, OFFSET).cuda()
    fx = f * x.double()
    y = flare.dropout(x, d)
    assert y.dtype == T
    close(y, fx, stored(T, fx) + 2 * U32 * fx.abs(), "y")
    held(y, f)
    y = flare.dropout(x, d, residual=res)
    assert y.dtype == R
    ref = fx + res.double()
    close(y, ref, stored(R, ref) + 4 * U32 * (fx.abs() + res.double().abs()), "y with a residual")
    dx = flare.dropout_backward(res, d, dtype=T)
    ref = f * res.double()
    close(dx, ref, stored(T, ref) + 2 * U32 * ref.abs(), "dx")
    held(dx, f)


def test_dropout_in_place_and_into_slices():
    g = gen(3)
    x, res = randn(g, 5, 40, 96, dtype=BF16), randn(g, 5, 40, 96)
    d = flare.Drop(0.3, 7)
    want = flare.dropout(x, d, residual=res)
    wide = torch.full((5, 40, 200), float("nan"), device="cuda")
    out = wide[..., 5:101]
    assert flare.dropout(x, d, residual=res, out=out) is out and torch.equal(out, want)
    assert wide[..., :5].isnan().all() and wide[..., 101:].isnan().all()
    r = res.clone()
    flare.dropout(x, d, residual=r, out=r)
    assert torch.equal(r, want)
    plain = flare.dropout(x, d)
    y = x.clone()
    flare.dropout(y, d, out=y)
    assert torch.equal(y, plain)


def test_dropout_of_nan_and_infinity():
    """What is dropped is 0 whatever it was; what is kept is passed on."""
    x = torch.full((64, 64), float("nan"), device="cuda")
    x[::2] = float("inf")
    d = flare.Drop(0.5, 11)
    f = factors(64, 64, 0.5, 11, 0).cuda()
    y = flare.dropout(x, d)
    assert (y[f == 0] == 0).all() and y[1::2][f[1::2] > 0].isnan().all() and (y[::2][f[::2] > 0] == float("inf")).all()


def test_dropout_of_nothing():
    d = flare.Drop(0.5, 1)
    assert flare.dropout(torch.empty(0, 24, device="cuda"), d).shape == (0, 24)
    assert flare.dropout_backward(torch.empty(3, 0, 24, device="cuda"), d).shape == (3, 0, 24)


def test_dropout_step_in_a_graph():
    """A captured step counter: every replay drops other elements, the ones that the offset says, forward and backward alike."""
    x = torch.ones(50, 120, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = flare.Drop(0.4, 99, 1000, step)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    flare.dropout(x, d, out=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flare.dropout(x, d, out=y)
        flare.dropout_backward(x, d, out=dx)
        step.add_(1)
    for i in range(3):
        graph.replay()
        want = factors(50, 120, 0.4, 99, 1000 + i).cuda()
        assert torch.equal(y > 0, want > 0) and torch.equal(dx > 0, want > 0), i
    step.fill_(-1000)
    assert torch.equal(flare.dropout(x, d) > 0, factors(50, 120, 0.4, 99, 0).cuda() > 0)


def test_dropped_share():
    """Of 2^22 elements the share p, to five standard deviations, in every one of a group's eight places."""
    for p in (0.1, 0.5, 0.9):
        y = flare.dropout(torch.ones(4096, 1024, device="cuda"), flare.Drop(p, 123456789))
        share = (y == 0).double().view(-1, 8).mean(0).cpu()
        assert ((share - p).abs() <= 5 * (p * (1 - p) / 2 ** 19) ** 0.5 + 2.0 ** -17).all(), (p, share)


# ---------------------------------------------------------------- embedding

def tokens_of(g, shape, vocab, kind):
    n = int(torch.tensor(shape).prod())
    if kind == "uniform":
        t = torch.randint(0, vocab, (n,), device="cuda", generator=g)
    elif kind == "same":
        t = torch.full((n,), vocab - 1, device="cuda")
    elif kind == "none":
        t = torch.full((n,), -1, device="cuda")
        t[::2] = vocab
    else:                                                    # a few are met all the time, some are no token
        t = (torch.rand(n, device="cuda", generator=g).pow(4) * vocab).long().clamp_(max=vocab - 1)
        t[torch.rand(n, device="cuda", generator=g) < 0.1] = -1
        t[torch.rand(n, device="cuda", generator=g) < 0.02] = vocab
    return t.view(shape)


def embed_reference(t, table, positions, scale, f, vocab):
    there = ((t >= 0) & (t < vocab)).reshape(-1)
    y = table.double()[t.reshape(-1).clamp(0, vocab - 1)] * scale * there[:, None]
    if positions is not None:
        y = y + positions.double().repeat(t.numel() // positions.shape[0], 1)
    return y * f


@pytest.mark.parametrize("types", TABLES, ids=str)
@pytest.mark.parametrize("B,L,vocab,width", [(1, 1, 1, 1), (1, 1, 1000, 1024), (3, 17, 20, 333), (2, 130, 50, 64), (1, 37, 5000, 2056)])
@pytest.mark.parametrize("positions,p", [(False, 0.0), (True, 0.25), (False, 0.5)])
def test_embed(types, B, L, vocab, width, positions, p):
    T, O = types
    g = gen(B + L + width)
    t = tokens_of(g, (B, L), vocab, "mixed")
    table = randn(g, vocab, width, dtype=T)
    pos = randn(g, L, width, dtype=T) if positions else None
    scale = 1.7
    f = factors(B * L, width, p, SEED, OFFSET).cuda()
    ref = embed_reference(t, table, pos, scale, f, vocab)
    size = embed_reference(t, table.abs(), pos.abs() if positions else None, scale, f, vocab)
    d = flare.Drop(p, SEED, OFFSET) if p > 0 else None
    for tok in (t, t.int()):
        y = flare.embed(tok, table, positions=pos, scale=scale, drop=d, dtype=O)
        assert y.shape == (B, L, width) and y.dtype == O
        close(y.view(B * L, width), ref, stored(O, ref) + 5 * U32 * size, "y")
    held(y.view(B * L, width), f)
    # rows off 16-byte boundaries, in and out
    odd, out = rows_at(table, width + 3, 1), torch.full((B, L, width + 5), float("nan"), dtype=O, device="cuda")
    assert torch.equal(flare.embed(t, odd, positions=pos, scale=scale, drop=d, out=out[..., :width]), y)
    assert out[..., width:].isnan().all()


def grads_reference(t, d, vocab, positions, scale, f):
    dy = d.double().view(-1, d.shape[-1]) * f
    there = ((t >= 0) & (t < vocab)).reshape(-1)
    table = torch.zeros(vocab + 1, dy.shape[1], dtype=torch.float64, device="cuda")
    table.index_add_(0, torch.where(there, t.reshape(-1), vocab), dy)
    size = torch.zeros_like(table).index_add_(0, torch.where(there, t.reshape(-1), vocab), dy.abs())
    count = torch.bincount(torch.where(there, t.reshape(-1), vocab), minlength=vocab + 1).double()[:, None]
    pos = dy.view(-1, positions, dy.shape[1]) if positions else None
    return table[:-1] * scale, (size * scale * (count + 4) * U32)[:-1], pos


@pytest.mark.parametrize("types", TABLES, ids=str)
@pytest.mark.parametrize("B,L,vocab,width,kind", [
    (1, 1, 1, 1, "uniform"), (1, 1, 70000, 16, "uniform"), (3, 17, 20, 333, "mixed"), (4, 1000, 256, 64, "mixed"), (2, 3001, 1023, 40, "uniform"), (2, 3001, 1024, 40, "mixed"),
    (1, 5000, 40000, 24, "mixed"), (7, 999, 3, 128, "same"), (2, 500, 9, 72, "none"), (1, 2000, 50, 2312, "mixed")])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_embed_backward(types, B, L, vocab, width, kind, p):
    T, O = types
    g = gen(B + L + width)
    t = tokens_of(g, (B, L), vocab, kind)
    dy = randn(g, B, L, width, dtype=O)
    f = factors(B * L, width, p, SEED, OFFSET).cuda()
    ref, bound, pos = grads_reference(t, dy, vocab, L, 1.7, f)
    d = flare.Drop(p, SEED, OFFSET) if p > 0 else None
    r = flare.embed_backward(t, dy, vocab, positions=L, scale=1.7, drop=d, dtype=T)
    assert r.dtable.shape == (vocab, width) and r.dtable.dtype == T and r.dpositions.shape == (L, width)
    close(r.dtable, ref, stored(T, ref) + bound, "dtable")
    want, size = pos.sum(0), pos.abs().sum(0)
    close(r.dpositions, want, stored(T, want) + (B + 4) * U32 * size, "dpositions")
    # the same from 32-bit tokens and from rows that are slices of wider ones, without positions; and again
    wide = torch.full((B, L, width + 3), float("nan"), dtype=O, device="cuda")
    wide[..., 1:1 + width] = dy
    for _ in range(2):
        s = flare.embed_backward(t.int(), wide[..., 1:1 + width], vocab, scale=1.7, drop=d, dtype=T)
        assert s.dpositions is None and torch.equal(s.dtable, r.dtable)
    # added to what is there: rows that no token has met stay as they are
    base, base_pos = randn(g, vocab, width, dtype=T), randn(g, L, width, dtype=T)
    a = flare.embed_backward(t, dy, vocab, positions=L, scale=1.7, drop=d, accumulate=True, out=(base.clone(), base_pos.clone()))
    total = ref + base.double()
    close(a.dtable, total, stored(T, total) + bound + 2 * U32 * (ref.abs() + base.double().abs()), "dtable added to")
    total = want + base_pos.double()
    close(a.dpositions, total, stored(T, total) + (B + 6) * U32 * (size + base_pos.double().abs()), "dpositions added to")
    met = torch.zeros(vocab + 1, dtype=torch.bool, device="cuda")
    met[torch.where((t >= 0) & (t < vocab), t, vocab).view(-1)] = True
    assert torch.equal(a.dtable[~met[:-1]], base[~met[:-1]])


@pytest.mark.parametrize("B,L,vocab,width,types", [
    (4, 10000, 50, 512, (BF16, BF16)), (1, 20000, 3000, 2064, (F32, F16)),     # sixteen columns a thread; chunks of 20, of 36 rows
    (2, 6000, 700, 4096, (BF16, BF16)), (2, 6000, 700, 4096, (BF16, F32)),     # of 44; float32 rows: eight columns a thread, of 40
    (8, 80000, 5, 128, (F32, BF16)), (3, 50000, 40000, 72, (F16, F16))],       # of 64 and 16 rows, blocks of 128 threads
    ids=str)
def test_embed_backward_of_many_elements(B, L, vocab, width, types):
    T, O = types
    g = gen(B + L + width)
    t = tokens_of(g, (B, L), vocab, "mixed")
    dy = randn(g, B, L, width, dtype=O)
    ref, bound, pos = grads_reference(t, dy, vocab, L, 0.7, torch.ones(1, width, device="cuda", dtype=torch.float64))
    r = flare.embed_backward(t, dy, vocab, positions=L, scale=0.7, dtype=T)
    close(r.dtable, ref, stored(T, ref) + bound, "dtable")
    close(r.dpositions, pos.sum(0), stored(T, pos.sum(0)) + (B + 4) * U32 * pos.abs().sum(0), "dpositions")
    s = flare.embed_backward(t, dy, vocab, positions=L, scale=0.7, dtype=T)
    assert torch.equal(s.dtable, r.dtable) and torch.equal(s.dpositions, r.dpositions)


def test_rows_without_a_token_give_nothing_away():
    """NaN and infinities in gradients of rows that have no token reach no row of the table."""
    g = gen(5)
    t = tokens_of(g, (4, 300), 40, "mixed")
    dy = randn(g, 4, 300, 48, dtype=BF16)
    want = flare.embed_backward(t, dy, 40)
    bad = dy.clone()
    bad[(t < 0) | (t >= 40)] = float("nan")
    assert torch.equal(flare.embed_backward(t, bad, 40).dtable, want.dtable)


def test_embedding_of_nothing():
    table = torch.randn(10, 24, device="cuda")
    t = torch.empty(3, 0, dtype=torch.int64, device="cuda")
    assert flare.embed(t, table).shape == (3, 0, 24)
    r = flare.embed_backward(t, torch.empty(3, 0, 24, device="cuda"), 10)
    assert (r.dtable == 0).all()


def test_many_rows():
    """More rows than one turn of the sort's warps takes, a vocabulary of three digits."""
    g = gen(8)
    n, V = 300_000, 1 << 21
    t = tokens_of(g, (n,), V, "mixed")
    dy = randn(g, n, 8, dtype=F32)
    ref, bound, _ = grads_reference(t, dy, V, 0, 1.0, torch.ones(1, 8, device="cuda", dtype=torch.float64))
    r = flare.embed_backward(t, dy, V)
    close(r.dtable, ref, stored(F32, ref) + bound, "dtable")
