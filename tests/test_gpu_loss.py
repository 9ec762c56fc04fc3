"""The loss over a vocabulary and its gradients against 64-bit implementations (needs a B200).

Bounds, element by element.  A logit l = scale x.w is off by D = scale max_v sum_c |x_c w_c| E, E the relative error of a product and of the additions: 16-bit factors
are multiplied exactly and added up 16 at a time with truncation, 2^-22 of what has been added up for each (half a unit of 24 bits lost by the sum and as much by the alignment of
what is added), width / 16 + 2 additions; float32 ones are held in 22 bits (3 * 2^-22 for both and the product of the low halves that is left out, and 2^-39 of the largest element for small
ones), with 24 additions before a sum leaves tensor memory, and width / 128 rounded ones behind it.  lse is off by as much, by the additions of exponentials (a thread 128,
then one per 2048 words, then 32 joins), 2^-24 each, exponentials (2^-22 each and 2^-24 of the exponent, at most 40 in units of ln 2 where they count), and its own rounding.  p = exp(l - lse) is off by its share of both.
"""
import pytest
import torch

from paper_2508_12594_b200 import flare
from tests._tokens import U32, UNIT, close, rows_at

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [BF16, F16, F32]


def problem(rows, vocab, width, dtype, seed=0, ignored=0.2, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + rows + 7 * vocab + 13 * width)
    x = (torch.randn(rows, width, device="cuda", generator=g) * size).to(dtype)
    w = (torch.randn(vocab, width, device="cuda", generator=g) * 2.0 / (width ** 0.5 * size)).to(dtype)
    labels = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    gone = torch.rand(rows, device="cuda", generator=g) < ignored
    labels[gone] = -100
    if rows > 2:
        labels[1] = vocab                                    # just beyond
        labels[2] = vocab - 1
    return x, w, labels, g


class Reference:
    """Values and bounds of one problem, float64."""

    def __init__(self, x, w, labels, dloss=1.0, scale=1.0):
        T, (n, C), V = x.dtype, x.shape, w.shape[0]
        there = (labels >= 0) & (labels < V)
        x, w = torch.where(there[:, None], x.double(), 0.0), w.double()
        l = scale * x @ w.T
        at = labels.clamp(0, V - 1)[:, None]
        zero = torch.zeros((), dtype=torch.float64, device="cuda")
        self.lse = torch.where(there, torch.logsumexp(l, 1), zero)
        self.loss = torch.where(there, self.lse - l.gather(1, at)[:, 0], zero)
        if T == F32:
            E = (3 + 24 + 8) * 2.0 ** -22 + (C / 128 + 2) * U32
            floor = 2.0 ** -38 * (x.abs().max() * w.abs().sum(1).max() + w.abs().max() * x.abs().sum(1).max()) * scale
        else:
            E, floor = (C / 16 + 2) * 2.0 ** -22, 0.0                           # (of the forward)
        size = scale * (x.abs() @ w.abs().T).max(1).values * E + floor          # of a row's logits
        sums = (128 + V / 2048 + 32 + 40 + 4) * U32
        self.lse_bound = torch.where(there, size + sums + 4 * U32 * self.lse.abs() + 2.0 ** -22, zero)
        self.loss_bound = torch.where(there, 2 * size + sums + 4 * U32 * (self.loss.abs() + 1) + 2.0 ** -22, zero)
        p = torch.exp(l - self.lse[:, None])
        q = p.scatter_add(1, at, -torch.ones_like(self.lse)[:, None])
        g = torch.where(there, dloss if isinstance(dloss, torch.Tensor) else torch.full_like(self.lse, dloss), 0.0).double() * scale
        self.dx, self.dw = g[:, None] * (q @ w), (g[:, None] * q).T @ x
        # Small bfloat16 vocabularies (W up to 2^22 elements) are multiplied as float16 times powers of two that put the largest element of X and of W between 2^14 and 2^15 and of q at 2^15: a value
        # that bfloat16 holds is held exactly down to 2^-14 of that scale (2^-28 of the largest), below to half of 2^-24, 2^-39 of the largest; q (times a row's mantissa of dloss) to 2^-11 and to 2^-39; x times powers of two of dloss not at all.
        half = T == BF16 and V * C <= 1 << 22
        # errors of q: of p, of its difference from the label's 1, and of its rounding (float32: 22 bits)
        if half:
            size = size + 2.0 ** -38 * (x.abs().max() * w.abs().sum(1).max() + w.abs().max() * x.abs().sum(1).max()) * scale
        eps = (size + self.lse_bound + 2.0 ** -21 + 42 * U32)[:, None] * p + 2 * U32 * (q.abs() + p)
        u = 2.0 ** -22 if T == F32 else UNIT[T]
        dq = (eps + q.abs() * u + (2.0 ** -40 if T == F32 else 2.0 ** -39 if T == F16 or half else 0.0)) * there[:, None]
        q = q.abs() * there[:, None]
        steps_x, steps_w = (V / 16 + 76) * 2.0 ** -22, (n / 16 + 76) * 2.0 ** -22
        if T == F32:
            steps_x, steps_w = (35 * 2.0 ** -22 + (V / 128 + 76) * U32), (35 * 2.0 ** -22 + (n / 128 + 76) * U32)
        ga = g.abs()[:, None]
        self.dx_bound = ga * (dq @ w.abs() + steps_x * (q @ w.abs())) + UNIT[T] * self.dx.abs()
        self.dw_bound = (ga * dq).T @ x.abs() + (steps_w + (u if T == F32 else 0.0)) * ((ga * q).T @ x.abs()) + UNIT[T] * self.dw.abs()
        if T == F16:                                         # results below the normal numbers; x times dloss / max dloss below them
            self.dx_bound += 2.0 ** -25
            self.dw_bound += 2.0 ** -25 + 2.0 ** -25 * g.abs().max() * q.sum(0)[:, None]
        if T == F32 or half:
            self.dw_bound += 2.0 ** -38 * x.abs().max() * g.abs().max() * q.sum(0)[:, None]
            self.dx_bound += 2.0 ** -38 * w.abs().max() * ga * q.sum(1)[:, None]


def check(x, w, labels, dloss=1.0, scale=1.0, view_x=None, view_w=None):
    """One problem through both calls, x and w as given or as the views of them."""
    r = Reference(x, w, labels, dloss, scale)
    x, w = x if view_x is None else view_x, w if view_w is None else view_w
    loss, lse = flare.token_loss(x, w, labels, scale=scale, check=True)
    close(lse, r.lse, r.lse_bound, "lse")
    close(loss, r.loss, r.loss_bound, "loss")
    d = flare.token_loss_backward(x, w, labels, lse, dloss, scale=scale, check=True)
    assert d.dx.dtype == x.dtype and d.dx.shape == x.shape and d.dw.dtype == x.dtype and d.dw.shape == w.shape
    close(d.dx, r.dx, r.dx_bound, "dx")
    close(d.dw, r.dw, r.dw_bound, "dw")
    return loss, lse, d


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,vocab,width", [(1, 1, 1), (1, 2, 8), (3, 10, 33), (128, 128, 64), (129, 257, 65), (256, 256, 128), (300, 1000, 200), (1000, 130, 72), (257, 5003, 130)])
def test_small(rows, vocab, width, dtype):
    x, w, labels, _ = problem(rows, vocab, width, dtype, ignored=0.0 if rows == 1 else 0.2)
    check(x, w, labels)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 9])
@pytest.mark.parametrize("vocab,width,offset", [(1, 8, 0), (5, 1, 0), (4099, 520, 0), (4098, 261, 0), (1001, 264, 1), (40000, 72, 0), (70, 12296, 0)])
def test_a_few_rows(rows, vocab, width, offset, dtype):
    """Up to eight rows have a forward of their own, where X fits shared memory."""
    x, w, labels, _ = problem(rows, vocab, width, dtype, ignored=0.0)
    view = rows_at(w, width + offset, offset) if offset else w
    check(x, w, labels, view_w=view, scale=0.7)
    check(x, w, labels.int(), view_x=rows_at(x, width + 1, 1))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_a_weight_for_every_row(dtype):
    x, w, labels, g = problem(700, 900, 136, dtype)
    dloss = torch.rand(700, device="cuda", generator=g) * 3e-3
    dloss[::5] = 0.0
    dloss[3] = -2e-3
    check(x, w, labels, dloss=dloss, scale=0.5)
    check(x, w, labels.int(), dloss=1.0 / 560, scale=2.0)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_rows_off_boundaries(dtype):
    """Rows of x and w that TMA could not take as they lie, NaN between them; results into slices of wider tensors."""
    x, w, labels, _ = problem(300, 400, 101, dtype)
    loss, lse, d = check(x, w, labels)
    vx, vw = rows_at(x, 107, 1), rows_at(w, 103, 3)
    a, b, e = check(x, w, labels, view_x=vx, view_w=vw)
    assert torch.equal(a, loss) and torch.equal(b, lse) and torch.equal(e.dx, d.dx) and torch.equal(e.dw, d.dw)
    dx, dw = torch.full((300, 120), float("nan"), dtype=dtype, device="cuda"), torch.full((400, 111), float("nan"), dtype=dtype, device="cuda")
    out = (dx[:, 1:102], dw[:, :101])
    flare.token_loss_backward(vx, vw, labels, lse, out=out, check=True)
    assert torch.equal(out[0], d.dx) and torch.equal(out[1], d.dw)
    assert dx[:, 102:].isnan().all() and dx[:, 0].isnan().all() and dw[:, 101:].isnan().all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("labelled", ["none", "first", "last", "every ninth"])
@pytest.mark.parametrize("vocab", [300, 2100])               # (16-bit rows over up to 2048 words are scored as they stand, others packed)
def test_few_rows_have_a_label(dtype, labelled, vocab):
    x, w, labels, _ = problem(1100, vocab, 96, dtype, ignored=0.0)
    keep = torch.zeros(1100, dtype=torch.bool, device="cuda")
    if labelled != "none":
        keep[{"first": slice(0, 1), "last": slice(1099, 1100), "every ninth": slice(0, 1100, 9)}[labelled]] = True
    labels = torch.where(keep, labels, -1)
    loss, lse, d = check(x, w, labels)
    assert (d.dx[~keep] == 0).all() and (loss[~keep] == 0).all() and (lse[~keep] == 0).all()
    # what those rows hold reaches nothing
    bad = torch.where(keep[:, None], x, float("nan"))
    bad[::2] = torch.where(keep[::2, None], x[::2], float("inf"))
    a, b = flare.token_loss(bad, w, labels)
    e = flare.token_loss_backward(bad, w, labels, b, check=True)
    assert torch.equal(a, loss) and torch.equal(b, lse) and torch.equal(e.dx, d.dx) and torch.equal(e.dw, d.dw)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_a_bad_row_spoils_its_own_loss_only(dtype):
    x, w, labels, _ = problem(400, 300, 64, dtype, ignored=0.0)
    want, lse = flare.token_loss(x, w, labels)
    x[7, 3], x[200, 0] = float("nan"), float("inf")
    loss, _ = flare.token_loss(x, w, labels, check=True)
    assert loss[7].isnan() and not loss[200].isfinite()
    rest = torch.ones(400, dtype=torch.bool, device="cuda")
    rest[[1, 7, 200]] = False                                # (row 1 has no label)
    # (float32: the largest element sets the scale of the halves, the same among the others)
    assert torch.allclose(loss[rest], want[rest], rtol=1e-6, atol=1e-6)


def test_large_logits():
    """Softmaxes with one word far ahead, and logits beyond what exp takes."""
    for dtype in TYPES:
        x, w, labels, _ = problem(260, 700, 64, dtype, ignored=0.0)
        x[:130] += (4.0 * w[labels.clamp(0, 699)][:130].float() * 8).to(dtype)
        check(x, w, labels, scale=8.0)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_sizes_far_from_one(dtype):
    """Large x against small w and the other way round: the halves' scales follow."""
    for size in (2.0 ** 9, 2.0 ** -9):
        x, w, labels, _ = problem(300, 500, 80, dtype, size=size)
        check(x, w, labels)


def test_tiny_and_huge_float32():
    for size in (1e12, 1e-12):
        x, w, labels, _ = problem(300, 500, 80, F32, size=size)
        check(x, w, labels)
    x, w, labels, _ = problem(64, 40, 16, F32)
    check(torch.zeros_like(x), w, labels)
    check(x, torch.zeros_like(w), labels)


@pytest.mark.parametrize("rows,vocab,width,dtype", [
    (4096, 9000, 512, BF16),                                  # full rounds of tiles and a rest that pairs share
    (20000, 256, 128, BF16),                                  # few tiles of dW, each shared by many pairs
    (600, 50021, 256, F16),                                   # the same of dX
    (2500, 12000, 1000, F16),
    (1500, 6000, 384, F32),
    (70000, 5000, 64, BF16),                                  # two pieces of the vocabulary
    (70000, 8000, 32, F16),                                   # three
    (40000, 3400, 72, F32),
    (130, 70, 4104, BF16), (130, 300, 2056, F32)])
def test_larger(rows, vocab, width, dtype):
    x, w, labels, g = problem(rows, vocab, width, dtype)
    check(x, w, labels, dloss=torch.rand(rows, device="cuda", generator=g) / rows)


def test_leading_dimensions_and_one_gradient():
    x, w, labels, _ = problem(600, 300, 64, BF16)
    loss, lse, d = check(x, w, labels)
    x3, l3 = x.view(3, 200, 64), labels.view(3, 200)
    a, b = flare.token_loss(x3, w, l3)
    assert a.shape == (3, 200) and torch.equal(a.view(-1), loss)
    e = flare.token_loss_backward(x3, w, l3, b)
    assert e.dx.shape == (3, 200, 64) and torch.equal(e.dx.view(600, 64), d.dx) and torch.equal(e.dw, d.dw)


def test_no_rows():
    w = torch.randn(50, 32, device="cuda")
    t = torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = flare.token_loss(torch.empty(0, 32, device="cuda"), w, t, check=True)
    assert loss.shape == (0,)
    d = flare.token_loss_backward(torch.empty(0, 32, device="cuda"), w, t, lse, check=True)
    assert d.dx.shape == (0, 32) and (d.dw == 0).all()


def test_the_same_twice():
    x, w, labels, _ = problem(3000, 3000, 200, BF16)
    a = flare.token_loss(x, w, labels)
    b = flare.token_loss(x, w, labels)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    d, e = (flare.token_loss_backward(x, w, labels, a[1]) for _ in range(2))
    assert torch.equal(d.dx, e.dx) and torch.equal(d.dw, e.dw)


def test_gradients_against_differences():
    """The float32 gradients along random directions against central differences of the loss in float64."""
    x, w, labels, g = problem(90, 120, 40, F32)
    wt = torch.rand(90, device="cuda", generator=g)

    def value(x, w):
        l, there = x @ w.T, (labels >= 0) & (labels < 120)
        return (torch.nn.functional.cross_entropy(l[there], labels[there], reduction="none") * wt.double()[there]).sum()

    _, lse = flare.token_loss(x, w, labels)
    d = flare.token_loss_backward(x, w, labels, lse, wt)
    h = 1e-4
    for _ in range(4):
        ux, uw = torch.randn(90, 40, device="cuda", generator=g), torch.randn(120, 40, device="cuda", generator=g)
        slope = (value(x.double() + h * ux.double(), w.double() + h * uw.double()) - value(x.double() - h * ux.double(), w.double() - h * uw.double())) / (2 * h)
        got = (d.dx.double() * ux.double()).sum() + (d.dw.double() * uw.double()).sum()
        # third derivatives of a sum of 90 losses with logits of order one, times h^2: below 1e-4; the gradients' own error is below 1e-5 of theirs
        assert abs(float(got - slope)) <= 1e-4 + 1e-5 * float(d.dx.double().abs().sum() + d.dw.double().abs().sum())


def test_captured_and_replayed():
    x, w, labels, _ = problem(900, 700, 128, BF16)
    want, lse = flare.token_loss(x, w, labels)
    d = flare.token_loss_backward(x, w, labels, lse)
    out = (torch.empty_like(want), torch.empty_like(lse), torch.empty_like(x), torch.empty_like(w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        flare.token_loss(x, w, labels, out=out[:2])
        flare.token_loss_backward(x, w, labels, out[1], out=out[2:])
    for _ in range(2):
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        assert torch.equal(out[0], want) and torch.equal(out[2], d.dx) and torch.equal(out[3], d.dw)
    # other labels, fewer of them: the number of rows is the device's affair
    other = torch.where(torch.arange(900, device="cuda") % 3 == 0, labels, -1)
    want, lse = flare.token_loss(x, w, other)
    d = flare.token_loss_backward(x, w, other, lse)
    labels.copy_(other)
    graph.replay()
    assert torch.equal(out[0], want) and torch.equal(out[2], d.dx) and torch.equal(out[3], d.dw)
