"""The loss over a vocabulary where sizes differ by many powers of two: one finite element far above all others reaches its own row (of x) or word (of w) and nothing else, whatever
the type; sizes near either end of float32 (needs a B200).

Bounds, element by element, relative to a row's own magnitudes.  A logit is off by scale max_v sum_c |x_c w_c| E.  16-bit factors are multiplied exactly and added up 16 at a time with truncation,
2^-22 of what has been added up for each addition (half a unit of 24 bits lost by the sum and as much by the alignment of what is added): width / 16 + 2 of them.  float32 factors are three bfloat16
values each, which hold all 24 bits; of their nine products six are formed, the others are up to 2^-24 of it; 24 additions before a sum leaves tensor memory, and width / 64 rounded ones behind it.  lse is off by as
much, by the additions of exponentials (a thread 128, then one per 2048 words, then 32 joins), 2^-24 each, by the exponentials (2^-22 each, and 2^-24 of an exponent of at most 40 that counts), and by
its own rounding; p = exp(l - lse) by its share of both.
"""
import pytest
import torch

from paper_2508_12594_b200 import flare
from tests._tokens import U32, UNIT, close

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def problem(rows, vocab, width, dtype, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(rows + 7 * vocab + 13 * width)
    x = (torch.randn(rows, width, device="cuda", generator=g) * size).to(dtype)
    w = (torch.randn(vocab, width, device="cuda", generator=g) * 2.0 / (width ** 0.5 * size)).to(dtype)
    labels = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    labels[torch.rand(rows, device="cuda", generator=g) < 0.1] = -100
    labels[0], labels[1] = 1, 2
    return x, w, labels, g


class Reference:
    """Values and bounds of the rows that have a label, float64."""

    def __init__(self, x, w, labels, dloss=1.0, scale=1.0):
        T, (n, C), V = x.dtype, x.shape, w.shape[0]
        there = (labels >= 0) & (labels < V)
        x, w = torch.where(there[:, None], x.double(), 0.0), w.double()
        l = scale * x @ w.T
        at = labels.clamp(0, V - 1)[:, None]
        zero = torch.zeros((), dtype=torch.float64, device="cuda")
        self.lse = torch.where(there, torch.logsumexp(l, 1), zero)
        self.loss = torch.where(there, self.lse - l.gather(1, at)[:, 0], zero)
        E = 2.0 ** -24 + (24 + 2) * 2.0 ** -22 + (C / 64 + 2) * U32 if T == F32 else (C / 16 + 2) * 2.0 ** -22
        size = scale * (x.abs() @ w.abs().T).max(1).values * E
        sums = (128 + V / 2048 + 32 + 40 + 4) * U32
        self.lse_bound = torch.where(there, size + sums + 4 * U32 * self.lse.abs() + 2.0 ** -22, zero)
        self.loss_bound = torch.where(there, 2 * size + sums + 4 * U32 * (self.loss.abs() + 1) + 2.0 ** -22, zero)
        p = torch.exp(l - self.lse[:, None])
        q = p.scatter_add(1, at, -torch.ones_like(self.lse)[:, None])
        g = torch.where(there, dloss if isinstance(dloss, torch.Tensor) else torch.full_like(self.lse, dloss), 0.0).double() * scale
        self.dx, self.dw = g[:, None] * (q @ w), (g[:, None] * q).T @ x
        # q: of p, of its difference from the label's 1, of its rounding: 24 bits (float32), two 16-bit values' (up to 256 rows, or up to 8192 words and w of up to 2^22 elements), or one's, float16's down to 2^-39
        two = T != F32 and (n <= 256 or (V <= 8192 and V * C <= 1 << 22))
        u = U32 if T == F32 else 2 * (UNIT[T] / 2) ** 2 if two else UNIT[T]
        eps = (size + self.lse_bound + 2.0 ** -21 + 42 * U32)[:, None] * p + 2 * U32 * (q.abs() + p)
        dq = (eps + q.abs() * u + (2.0 ** -39 if T == F16 else 0.0)) * there[:, None]
        q, products = q.abs() * there[:, None], 2 if two else 1
        steps_x, steps_w = (products * V / 16 + 76) * 2.0 ** -22, (products * n / 16 + 76) * 2.0 ** -22
        if T == F32:
            steps_x, steps_w = 2.0 ** -24 + 26 * 2.0 ** -22 + (V / 64 + 76) * U32, 2.0 ** -24 + 26 * 2.0 ** -22 + (n / 64 + 76) * U32
        ga = g.abs()[:, None]
        self.dx_bound = ga * (dq @ w.abs() + steps_x * (q @ w.abs())) + UNIT[T] * self.dx.abs()
        self.dw_bound = (ga * dq).T @ x.abs() + steps_w * ((ga * q).T @ x.abs()) + UNIT[T] * self.dw.abs()
        if T == F16:                                         # below the normal numbers: results; and x times a row's power of two, whose largest is between 2^14 and 2^15
            self.dx_bound += 2.0 ** -25
            self.dw_bound += 2.0 ** -25 + 2.0 ** -38 * (x.abs().max(1).values * g.abs()).max() * q.sum(0)[:, None]


def run(x, w, labels, dloss=1.0, scale=1.0):
    loss, lse = flare.token_loss(x, w, labels, scale=scale, check=True)
    return (loss, lse, *flare.token_loss_backward(x, w, labels, lse, dloss, scale=scale, check=True))


def held(got, r, rows=slice(None), words=slice(None)):
    loss, lse, dx, dw = got
    close(lse[rows], r.lse[rows], r.lse_bound[rows], "lse")
    close(loss[rows], r.loss[rows], r.loss_bound[rows], "loss")
    close(dx[rows], r.dx[rows], r.dx_bound[rows], "dx")
    close(dw[words], r.dw[words], r.dw_bound[words], "dw")


SIZES = [(300, 500, 80, F32), (40, 1000, 200, F32), (5, 3000, 64, F32), (300, 500, 80, BF16), (2100, 256, 128, BF16), (300, 70000, 64, BF16)]


@pytest.mark.parametrize("value", [1e6, 1e9, 1e13, 1e30])
@pytest.mark.parametrize("rows,vocab,width,dtype", SIZES, ids=str)
def test_one_large_element_of_x(rows, vocab, width, dtype, value):
    """The other rows are as without it.  Its own row's softmax is one word, so that of dw only that word and the label are its business."""
    x, w, labels, _ = problem(rows, vocab, width, dtype)
    x[0] = 0.0
    x[0, 3] = value
    top = 9
    w[top, 3] = 4.0                                          # (the others': 0.2 on average)
    without = labels.clone()
    without[0] = -1
    loss, lse, dx, dw = got = run(x, w, labels)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[0] = False
    others = torch.ones(vocab, dtype=torch.bool, device="cuda")
    others[[top, 1]] = False
    held(got, Reference(x, w, without), rest, others)
    r = Reference(x[:1], w, labels[:1])
    close(lse[:1], r.lse, r.lse_bound, "its lse")
    close(loss[:1], r.loss, r.loss_bound, "its loss")
    # one word's p is 1, all others' 0: the logits of the forward and the backward are the same
    close(dx[:1], r.dx, 4 * UNIT[dtype] * (w[top].double().abs() + w[1].double().abs()), "its dx")
    full = Reference(x, w, labels)
    size = 4 * UNIT[dtype] * value + full.dw.abs() * UNIT[dtype]
    close(dw[[top, 1], 3], full.dw[[top, 1], 3], size[[top, 1], 3], "its dw")


@pytest.mark.parametrize("value", [1e6, 1e13, 1e30])
@pytest.mark.parametrize("rows,vocab,width,dtype", SIZES, ids=str)
def test_one_large_element_of_w(rows, vocab, width, dtype, value):
    """A word far ahead of all others for some rows, far behind for the rest: those are as without it."""
    x, w, labels, _ = problem(rows, vocab, width, dtype)
    x[:, 5] = torch.where(torch.arange(rows, device="cuda") % 2 == 0, 1.0, -1.0).to(dtype)
    labels[1::2] = torch.where(labels[1::2] == 7, 8, labels[1::2])
    plain = w.clone()
    w[7] = 0.0
    w[7, 5] = value
    behind = torch.arange(rows, device="cuda") % 2 == 1
    keep = [v for v in range(vocab) if v != 7]
    kept_labels = torch.where(labels > 7, labels - 1, labels)
    loss, lse, dx, dw = run(x, w, labels)
    r = Reference(x, plain[keep], kept_labels)
    close(lse[behind], r.lse[behind], r.lse_bound[behind], "lse")
    close(loss[behind], r.loss[behind], r.loss_bound[behind], "loss")
    close(dx[behind], r.dx[behind], r.dx_bound[behind], "dx")


@pytest.mark.parametrize("rows,vocab,width", [(300, 500, 80), (1500, 6000, 64)])
@pytest.mark.parametrize("dtype,value", [(F32, 1e4), (F32, 1e12), (F32, 1e25), (BF16, 1e4), (BF16, 1e12), (BF16, 1e25), (F16, 1e4)], ids=str)
def test_one_large_weight_of_a_row(rows, vocab, width, dtype, value):
    """dloss: the other rows' part in dw, seen in words that the row with the large weight has nothing to do with."""
    x, w, labels, g = problem(rows, vocab, width, dtype)
    x[0] = (100.0 * w[1].float()).to(dtype)                  # certain of its label: |w|^2 is about 4, other products about 0.5
    dloss = (torch.rand(rows, device="cuda", generator=g) + 0.5) * 1e-3
    dloss[0] = value
    none = torch.softmax(x[0].double() @ w.double().T, 0) * value < 1e-30
    assert int(none.sum()) > 0.99 * vocab
    without = labels.clone()
    without[0] = -1
    got = run(x, w, labels, dloss)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[0] = False
    r = Reference(x, w, without, dloss)
    if dtype == F16:                                         # (what x times a power of two is held down to is by the largest, which is that row's)
        q = (torch.softmax(x.double() @ w.double().T, 1) - torch.nn.functional.one_hot(labels.clamp(0), vocab)).abs()
        r.dw_bound += 2.0 ** -38 * value * float(x[0].abs().max()) * (q * ((without >= 0) & (without < vocab))[:, None]).sum(0)[:, None]
    held(got, r, rest, none)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_weights_of_nothing(dtype):
    """dloss of zeros, of one row only, of the smallest numbers beside one."""
    x, w, labels, _ = problem(300, 500, 80, dtype)
    dloss = torch.zeros(300, device="cuda")
    for tiny in (0.0, 1e-38, 1e-42):
        dloss[:] = tiny
        loss, lse, dx, dw = run(x, w, labels, dloss)
        assert (dx.abs() <= 1e-34).all() and (dw.abs() <= 1e-34).all()
        dloss[1] = 1.0
        r = Reference(x, w, labels, dloss)
        r.dx_bound += 1e-34                                  # (what is below float32's normal numbers: 300 rows of 1e-38 times up to 5)
        r.dw_bound += 1e-34
        held(run(x, w, labels, dloss), r)


@pytest.mark.parametrize("size", [1e25, 1e-25, 1e15, 1e-15])
@pytest.mark.parametrize("rows,vocab,width", [(300, 500, 80), (1500, 6000, 200)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_sizes_near_either_end(rows, vocab, width, dtype, size):
    x, w, labels, g = problem(rows, vocab, width, dtype, size=size)
    held(run(x, w, labels), Reference(x, w, labels))


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("rows,vocab,width", [(300, 500, 80), (600, 5003, 136), (200, 20000, 264), (2, 9000, 520), (7, 9000, 261)])
def test_results_to_their_types_rounding(rows, vocab, width, dtype):
    """What q is held in, 16 bits in bfloat16 (w up to 2^22 elements), shows in the gradients."""
    x, w, labels, g = problem(rows, vocab, width, dtype)
    held(run(x, w, labels, scale=0.5), Reference(x, w, labels, scale=0.5))
    dloss = torch.rand(rows, device="cuda", generator=g)
    held(run(x, w, labels, dloss, scale=0.5), Reference(x, w, labels, dloss, scale=0.5))


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("width", [64, 520, 1096])
@pytest.mark.parametrize("vocab", [300, 2100])
def test_logits_far_beyond_what_their_difference_needs(dtype, width, vocab):
    """Certain rows with logits up to 1e8: their loss is 0 or the distance to the label, their p 1 or 0."""
    x, w, labels, _ = problem(300, vocab, width, dtype)
    scale = 1e7 if dtype == F16 else 0.7
    if dtype != F16:
        x = (x.float() * 1e8).to(dtype)
    l = scale * (x.double() @ w.double().T)
    top, two = l.argmax(1), l.topk(2, 1).values
    labels = torch.where(torch.arange(300, device="cuda") % 2 == 0, top, labels)
    certain = (two[:, 0] - two[:, 1] > 1e-3 * two[:, 0]) & (labels >= 0)
    assert int(certain.sum()) > 150
    loss, lse, dx, _ = run(x, w, labels, 1.0 / scale, scale)
    r = Reference(x, w, labels, scale=scale)
    close(lse[certain], r.lse[certain], r.lse_bound[certain], "lse")
    close(loss[certain], r.loss[certain], r.loss_bound[certain], "loss")
    learned = certain & (labels == top)
    assert int(learned.sum()) > 100 and (loss[learned] == 0).all() and (dx[learned] == 0).all()
    others = certain & ~learned
    a, b = w.double()[top][others], w.double()[labels.clamp(min=0)][others]
    close(dx[others], a - b, 4 * UNIT[dtype] * (a.abs() + b.abs()) + 2.0 ** -24, "dx")


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("rows,width", [(1, 64), (3, 520), (4, 100), (8, 1001)])
def test_logits_far_beyond_of_a_few_rows(dtype, rows, width):
    """The same, scored by the kernels of few rows."""
    x, w, labels, _ = problem(300, 500, width, dtype)
    scale = 1e7 if dtype == F16 else 0.7
    x = x[:rows] if dtype == F16 else (x[:rows].float() * 1e8).to(dtype)
    l = scale * (x.double() @ w.double().T)
    labels = l.argmax(1)
    two = l.topk(2, 1).values
    certain = two[:, 0] - two[:, 1] > 1e-3 * two[:, 0]
    loss, lse, dx, dw = run(x, w, labels, 1.0 / scale, scale)
    r = Reference(x, w, labels, scale=scale)
    close(lse, r.lse, r.lse_bound, "lse")
    assert (loss[certain] == 0).all() and (dx[certain] == 0).all() and dw.isfinite().all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 8, 9, 300])
@pytest.mark.parametrize("vocab,width", [(3, 4032), (300, 1001), (2100, 264)])
def test_rows_that_have_learned_their_label(dtype, rows, vocab, width):
    """What is left of their gradient is 1 - p: p is formed from the very logits that lse was, so that errors of the label's logit, which lse is next to, do not count.

    1 - p and the other p are off by their share of what differences of logits are, and of the sums of exponentials; lse's rounding and that of a logit, 2^-24 each of their size, and an exponential near 1, 2^-22,
    count whole."""
    x, w, _, g = problem(300, vocab, width, dtype)
    labels = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    x = (x[:rows].float() + 3.0 * w[labels].float()).to(dtype)
    loss, lse, dx, dw = run(x, w, labels)
    r = Reference(x, w, labels)
    xd, wd, at = x.double(), w.double(), labels[:, None]
    l = xd @ wd.T
    p = torch.exp(l - r.lse[:, None])
    others = p.scatter(1, at, 0.0)
    one = others.sum(1, keepdim=True)
    q = others.scatter(1, at, -one)
    E = 2.0 ** -24 + (24 + 2) * 2.0 ** -22 + (width / 64 + 2) * U32 if dtype == F32 else (width / 16 + 2) * 2.0 ** -22
    size = (xd.abs() @ wd.abs().T).max(1, keepdim=True).values * E
    share = 2 * size + (128 + vocab / 2048 + 80) * U32 + 2.0 ** -20
    whole = 4 * U32 * (r.lse[:, None].abs() + l.abs() + 1)
    two = dtype != F32                                       # (vocab x width up to 2^22)
    u = U32 if dtype == F32 else 2 * (UNIT[dtype] / 2) ** 2 if two else UNIT[dtype]
    dq = others * (share + whole)
    dq.scatter_(1, at, one * share + whole.gather(1, at) + 2.0 ** -21)
    dq += q.abs() * u + (2.0 ** -39 if dtype == F16 else 0.0)
    steps = (2 if two else 1) * (max(vocab, rows) / 16 + 76) * 2.0 ** -22
    floor = 2.0 ** -25 if dtype == F16 else 0.0
    want = q @ wd
    close(dx, want, dq @ wd.abs() + steps * (q.abs() @ wd.abs()) + UNIT[dtype] * want.abs() + floor, "dx")
    want = q.T @ xd
    close(dw, want, dq.T @ xd.abs() + steps * (q.abs().T @ xd.abs()) + UNIT[dtype] * want.abs() + floor, "dw")
