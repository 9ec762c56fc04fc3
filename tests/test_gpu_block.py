"""The norms around a block, its gate and residual scale, against float64 (needs a B200).

The reference is the definition in float64: plain operations forward, automatic differentiation backward, and central differences.
Bounds, derived before the first run.  A float32 row result goes through a sum of C terms (8 in a thread, then halving: about
8 + log2 C additions) and some ten operations, each 2^-24 relative to what it handles, which is at most a few times RMS + |value|: 2e-5 of
that leaves room for a factor of ten.  Stored in 16 bits, half a unit in the last place more (2^-8, 2^-11 relative; float16 below its normal
range 2^-25).  J^T d is a difference of terms of the size of rstd d w, which with few columns cancel: 2e-6 of their RMS beside that.  A sum over
rows is off by a share of the sum of its terms' absolute values (1e-5 of that is 168 roundings in a row), and by its terms' own errors,
which go with the RMS of the terms.
"""
import ctypes

import pytest
import torch

from paper_2508_12594_b200 import flare
from tests._util import STORE_ULP

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {torch.float32: 0.0, torch.bfloat16: STORE_ULP["bf16"], torch.float16: STORE_ULP["f16"]}


def close(got, ref, what, terms=0.0):
    """terms: the size of what cancels in ref."""
    ref = ref.double()
    rms = ref.square().mean().sqrt() if ref.numel() else torch.zeros(())
    bound = 2e-5 * (rms + ref.abs()) + HALF_ULP[got.dtype] * ref.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 0.0) + 2e-6 * terms
    excess = ((got.double() - ref).abs() - bound).max() if ref.numel() else torch.zeros(())
    assert got.shape == ref.shape, what
    assert excess <= 0, f"{what}: over its bound by {float(excess):.3e} (RMS {float(rms):.3e})"


def size(t):
    return t.square().mean().sqrt()


def sum_close(got, ref, terms, rows, what):
    """A sum of `terms` over the dimensions `rows`."""
    count = 1
    for i in rows:
        count *= terms.shape[i]
    excess = ((got.double() - ref).abs() - 1e-5 * (terms.abs().sum(rows) + count * size(terms))).max()
    assert excess <= 0, f"{what}: over its bound by {float(excess):.3e}"


def ref_norm(v, kind, w, b, eps):
    mean = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(v[..., :1])
    rstd = ((v - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    out = (v - mean) * rstd
    out = out if w is None else out * w
    return (out if b is None else out + b), mean, rstd


class Problem:
    """Random inputs of one join (branch=True) or norm, their float64 copies, and the forward in float64."""

    def __init__(self, B, N, C, dtype="bf16", res=None, kind="layer", post=True, pre=True, gate="none", gate_kind="sigmoid", scale=True, bias=True,
                 weight=True, alpha=1.0, strided=False, branch=True, seed=0, mean=0.5):
        g = torch.Generator(device="cuda").manual_seed(seed)
        T, R = DT[dtype], DT[res or dtype]

        def rand(*s, dt=torch.float32, scale=1.0, mean=0.0):
            return (torch.randn(*s, device="cuda", generator=g) * scale + mean).to(dt)

        self.kind, self.alpha, self.gate_kind, self.branch, self.T, self.R = kind, alpha, gate_kind, branch, T, R
        lead = (B, N)

        def rows(dt, **kw):
            if not strided:
                return rand(*lead, C, dt=dt, **kw)
            # a slice of something wider, off its 16-byte boundaries
            return rand(*lead, 2 * C + 3, dt=dt, **kw)[..., 3:3 + C]

        self.x = rows(R, mean=mean)
        self.o = rows(T, mean=mean) if branch else None
        self.g = None if gate == "none" else rows(T) if gate == "token" else rand(B, C, dt=T, mean=1.0)
        self.s = rand(C, mean=0.5, scale=0.3) if scale and branch else None

        def norm():
            return flare.Norm(kind, rand(C, mean=1.0, scale=0.2) if weight else None, rand(C, scale=0.3) if bias else None, 1e-5)

        self.pre = norm() if pre else None
        self.post = norm() if post and branch else None
        self.dy = rows(R)
        self.dh = rows(T) if pre else None

    def leaves(self):
        """float64 copies that gradients are asked for, by name."""
        d = lambda t: None if t is None else t.detach().double().clone().requires_grad_(True)  # noqa: E731
        L = {"x": d(self.x), "o": d(self.o), "g": d(self.g), "s": d(self.s)}
        for name, n in (("post", self.post), ("pre", self.pre)):
            L[name + "_w"], L[name + "_b"] = (d(n.weight), d(n.bias)) if n else (None, None)
        return L

    def forward64(self, L):
        """(y, h, stats) of the definition."""
        x, o, g, s = L["x"], L["o"], L["g"], L["s"]
        zero = torch.zeros_like(x[..., :1])
        st = [zero, zero, zero, zero]
        y = x
        if self.branch:
            n = o
            if self.post:
                n, st[0], st[1] = ref_norm(o, self.kind, L["post_w"], L["post_b"], self.post.eps)
            if g is not None:
                a = torch.sigmoid(g) if self.gate_kind == "sigmoid" else g
                n = n * (a if a.dim() == n.dim() else a[:, None, :])
            n = n if s is None else n * s
            y = self.alpha * x + n
        h = None
        if self.pre:
            h, st[2], st[3] = ref_norm(y, self.kind, L["pre_w"], L["pre_b"], self.pre.eps)
        return y, h, torch.cat(st, -1).reshape(-1, 4)

    def forward(self, **kw):
        if not self.branch:
            h, stats = flare.block_norm(self.x, self.pre, dtype=self.T, **kw)
            return self.x, h, stats
        return flare.block_join(self.x, self.o, post=self.post, pre=self.pre, gate=self.g, gate_kind=self.gate_kind, scale=self.s, residual_scale=self.alpha, **kw)

    def backward(self, y, stats, **kw):
        if not self.branch:
            return flare.block_norm_backward(y, stats, self.dh, self.pre, dy=self.dy, **kw)
        return flare.block_join_backward(self.o, y, stats, self.dy, self.dh, post=self.post, pre=self.pre, gate=self.g, gate_kind=self.gate_kind,
                                         scale=self.s, residual_scale=self.alpha, **kw)


SHAPES = [
    # B, N, C: one row, one column; widths on both sides of a thread's, a warp's, a block's share and of what the registers hold; odd ones
    (1, 1, 1), (1, 3, 7), (2, 5, 8), (1, 37, 64), (3, 41, 72), (2, 150, 128), (1, 300, 129), (2, 33, 200), (1, 65, 256), (1, 19, 264),
    (2, 20, 333), (1, 31, 512), (1, 9, 1000), (3, 7, 2048), (1, 5, 2049), (1, 6, 2056), (2, 3, 4096), (1, 4, 4104), (1, 3, 8192), (2, 2, 9001),
    (1, 2, 16384), (1, 4000, 64), (2, 2500, 136), (1, 700, 1024), (1, 320, 2304), (1, 301, 4352),
]
TYPES = [("bf16", None), ("f16", "f32"), ("f32", None), ("bf16", "f32"), ("f16", None)]


def options(i):
    """A mixture of the options that goes through all values of each, and most pairs, as i runs."""
    return dict(kind=("layer", "rms")[i % 2], post=i % 3 != 2, gate=("token", "none", "item", "token")[(i // 2) % 4], gate_kind=("sigmoid", "linear")[(i // 3) % 2],
                scale=(i // 2) % 2 == 0, bias=(i // 4) % 2 == 0, weight=i % 7 != 5, alpha=(1.0, 0.7)[(i // 5) % 2], strided=i % 4 == 3, pre=i % 9 != 8)


CASES = [(shape, TYPES[(i + k) % 5], options(5 * i + 3 * k)) for i, shape in enumerate(SHAPES) for k in range(3)]


def check_forward(p):
    y, h, stats = p.forward()
    with torch.no_grad():
        y64, h64, st64 = p.forward64(p.leaves())
    if p.branch:
        close(y, y64, "y")
    assert (h is None) == (p.pre is None)
    if p.pre:
        close(h, h64, "h")
    # a mean of C values is off by a share of their size, not of its own
    largest = 2e-6 * (1.0 + p.x.double().abs().max() + (p.o.double().abs().max() if p.branch else 0.0))
    assert (stats[:, 0::2].double() - st64[:, 0::2]).abs().max() <= largest
    close(stats[:, 1::2], st64[:, 1::2], "rstd")


def check_backward(p):
    """Backward from the y and stats of float64 (y rounded as it is stored: what it stands for is then exactly what the kernel is given)."""
    L = p.leaves()
    with torch.no_grad():
        y64, _, st64 = p.forward64(L)
    y = p.x if not p.branch else y64.to(p.R)
    got = p.backward(y, st64.float().contiguous())
    # autograd of the definition with the next norm looking at the stored y, its statistics those given
    leaf = {k: v for k, v in L.items() if v is not None}
    yr = y.double().requires_grad_(True)
    st = st64.float().double().view(*p.x.shape[:-1], 4)
    rows = tuple(range(p.x.dim() - 1))
    dt, cancel = p.dy.double(), 0.0
    if p.pre:
        hat = (yr.detach() - st[..., 2:3]) * st[..., 3:4]
        w = 1.0 if p.pre.weight is None else p.pre.weight.double()
        d = p.dh.double() * w
        inner = d - hat * (d * hat).mean(-1, keepdim=True) - (d.mean(-1, keepdim=True) if p.kind == "layer" else 0.0)
        dt = dt + st[..., 3:4] * inner
        cancel = size(st[..., 3:4] * d)
        sums = [("dpre_weight" if p.branch else "dweight", p.pre.weight, p.dh.double() * hat), ("dpre_bias" if p.branch else "dbias", p.pre.bias, p.dh.double())]
        for name, present, terms in sums:
            v = getattr(got, name)
            assert (v is None) == (present is None)
            if v is not None:
                sum_close(v, terms.sum(rows), terms, rows, name)
    close(got.dx, p.alpha * dt if p.branch else dt, "dx", cancel)
    if not p.branch:
        return
    names = [k for k in ("o", "g", "s", "post_w", "post_b") if k in leaf]
    yy, _, _ = p.forward64(L)
    grads = dict(zip(names, torch.autograd.grad(yy, [leaf[k] for k in names], dt)))
    # what the terms of the sums over rows amount to
    with torch.no_grad():
        n = L["o"]
        hat = n
        if p.post:
            n, m, r = ref_norm(L["o"], p.kind, L["post_w"], L["post_b"], p.post.eps)
            hat = (L["o"] - m) * r
        a = 1.0
        if p.g is not None:
            a = torch.sigmoid(L["g"]) if p.gate_kind == "sigmoid" else L["g"]
            a = a if a.dim() == n.dim() else a[:, None, :]
        s = 1.0 if L["s"] is None else L["s"].abs()
        terms = {"s": (dt * a * n).abs(), "post_w": (dt * a * hat).abs() * s, "post_b": (dt * a * torch.ones_like(n)).abs() * s}
        # (n = w n^ + b: the parts are summed apart)
        apart = (dt * a * hat).abs() * (1.0 if L["post_w"] is None else L["post_w"].abs()) + (dt * a).abs() * (0.0 if L["post_b"] is None else L["post_b"].abs())
        terms["s"] = torch.maximum(terms["s"], apart)
        reach = (dt * a).abs() * s * (1.0 if L["post_w"] is None else L["post_w"].abs()) * (r if p.post else 1.0)
    close(got.dbranch, grads["o"], "dbranch", size(reach))
    for k, name in (("s", "dscale"), ("post_w", "dpost_weight"), ("post_b", "dpost_bias")):
        v = getattr(got, name)
        assert (v is None) == (k not in grads), name
        if v is not None:
            sum_close(v, grads[k], terms[k], rows, name)
    if p.g is None:
        assert got.dgate is None
    elif p.g.dim() == p.x.dim():
        close(got.dgate, grads["g"], "dgate")
    else:
        slope = (torch.sigmoid(L["g"]) * (1 - torch.sigmoid(L["g"])) if p.gate_kind == "sigmoid" else torch.ones_like(L["g"])).detach()
        each = (dt.abs() * ((hat.abs() * (1.0 if L["post_w"] is None else L["post_w"].abs())) + (0.0 if L["post_b"] is None else L["post_b"].abs())) * s)
        bound = 1e-5 * slope * (each.sum(1) + each.shape[1] * size(each)) + HALF_ULP[p.T] * grads["g"].abs() + (2.0 ** -25 if p.T == torch.float16 else 0.0)
        assert ((got.dgate.double() - grads["g"]).abs() <= bound.detach()).all(), "dgate"


@pytest.mark.parametrize("shape,types,opt", CASES, ids=str)
def test_join(shape, types, opt):
    p = Problem(*shape, dtype=types[0], res=types[1], seed=sum(shape), **opt)
    check_forward(p)
    check_backward(p)


@pytest.mark.parametrize("i", range(0, 2 * len(SHAPES), 2))
def test_norm(i):
    t = TYPES[i % 5]
    p = Problem(*SHAPES[i // 2], dtype=t[0], res=t[1], seed=i, kind=("layer", "rms")[(i // 2) % 2], bias=i % 3 != 0, weight=i % 7 != 4, strided=i % 4 == 2, branch=False)
    check_forward(p)
    check_backward(p)


# Widths on both sides of what one warp, one group of columns a thread, a block and a cluster hold; few rows.
@pytest.mark.parametrize("C", [264, 333, 2056, 4096, 4360, 8192])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gate", ["none", "token", "item"])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("types", [("bf16", None), ("f16", "f32"), ("f32", None)], ids=str)
def test_every_form_of_backward(C, kind, gate, bias, types):
    p = Problem(2, 5, C, dtype=types[0], res=types[1], kind=kind, gate=gate, gate_kind="sigmoid", bias=bias, alpha=0.7, seed=C + 1)
    check_forward(p)
    check_backward(p)
    if gate == "none":
        p = Problem(2, 5, C, dtype=types[0], res=types[1], kind=kind, bias=bias, seed=C + 2, branch=False)
        check_backward(p)


@pytest.mark.parametrize("first", [0, 1, 2, 3, 5, 7])
@pytest.mark.parametrize("C,extra", [(40, 0), (40, 3), (333, 0), (333, 2), (1001, 5)])
@pytest.mark.parametrize("types", [("bf16", None), ("f16", "f32"), ("f32", None)], ids=str)
def test_rows_off_boundaries(first, C, extra, types):
    """Tensors that begin at the `first` element of their memory and end with it, rows C + extra apart; what lies between is NaN."""
    p = Problem(2, 9, C, dtype=types[0], res=types[1], gate="token", gate_kind="sigmoid", seed=C + first)

    def moved(t, k):
        ld, rows = C + extra, t.shape[0] * t.shape[1]
        memory = torch.full((k + (rows - 1) * ld + C,), float("nan"), device="cuda", dtype=t.dtype)
        v = memory.as_strided(t.shape, (t.shape[1] * ld, ld, 1), k)
        return v.copy_(t)

    for i, name in enumerate(("x", "o", "g", "dy", "dh")):
        setattr(p, name, moved(getattr(p, name), (first + i) % 8 if first else 0))
    check_forward(p)
    check_backward(p)
    # outputs off boundaries: what lies between rows is not touched
    y, h, stats = p.forward()
    out_y, out_h = moved(y, first), moved(h, first)
    y2, h2, _ = p.forward(out=(out_y, out_h, None))
    assert torch.equal(y2, y) or C % 8 == 0                 # (40 columns on boundaries run by another form)
    close(y2, y.double(), "y")
    if extra:
        gaps = out_y.as_strided((17, extra), (C + extra, 1), out_y.storage_offset() + C)
        assert gaps.isnan().all()


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gate,gate_kind", [("token", "sigmoid"), ("item", "linear")])
def test_gradients_against_differences(kind, gate, gate_kind):
    """float32 gradients in a random direction against central differences of the float64 forward (step 1e-4: 1e-8 of curvature)."""
    p = Problem(2, 21, 96, dtype="f32", kind=kind, gate=gate, gate_kind=gate_kind, alpha=0.8, seed=3)
    y, _, stats = p.forward()
    got = p.backward(y, stats)
    L = p.leaves()
    by_name = {"x": got.dx, "o": got.dbranch, "g": got.dgate, "s": got.dscale, "post_w": got.dpost_weight, "post_b": got.dpost_bias, "pre_w": got.dpre_weight,
               "pre_b": got.dpre_bias}
    gen = torch.Generator(device="cuda").manual_seed(9)

    def loss(M):
        y64, h64, _ = p.forward64(M)
        return (y64 * p.dy.double()).sum() + (h64 * p.dh.double()).sum()

    with torch.no_grad():
        for name, grad in by_name.items():
            v = torch.randn(L[name].shape, device="cuda", generator=gen, dtype=torch.float64)
            step = 1e-4
            up, down = ({**L, name: L[name] + sgn * step * v} for sgn in (1, -1))
            diff = (loss(up) - loss(down)) / (2 * step)
            size = (grad.double() * v).abs().sum()
            assert abs(diff - (grad.double() * v).sum()) <= 2e-5 * size, name


@pytest.mark.parametrize("C", [128, 200, 333, 4096, 5000])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_rows_far_from_ordinary(C, kind):
    """Constant rows, zero rows, rows around a large mean, and rows with a NaN or an infinity, which must not reach other rows."""
    p = Problem(1, 12, C, dtype="f32", kind=kind, gate="token", seed=C)
    p.o[0, 1] = 0.0
    p.x[0, 2] = 3.0
    p.o[0, 2] = -7.0
    p.o[0, 3] += 1000.0
    p.g[0, 4] = 90.0
    p.g[0, 5] = -120.0
    p.g[0, 6, ::2] = float("inf")
    p.g[0, 6, 1::2] = -float("inf")
    clean_y, clean_h, _ = p.forward()
    bad = Problem(1, 12, C, dtype="f32", kind=kind, gate="token", seed=C)
    for name in ("x", "o", "g"):
        getattr(bad, name).copy_(getattr(p, name))
    bad.o[0, 8, C // 2] = float("nan")
    bad.x[0, 9, 0] = float("inf")
    bad.g[0, 10, C - 1] = float("nan")
    y, h, stats = bad.forward()
    fine = [0, 1, 2, 3, 4, 5, 6, 7, 11]
    assert torch.equal(y[0, fine], clean_y[0, fine]) and torch.equal(h[0, fine], clean_h[0, fine])
    assert y[0, 8].isnan().all() and h[0, 8].isnan().all() and h[0, 9].isnan().any() and torch.isinf(y[0, 9, 0]) and h[0, 10].isnan().all()
    assert y[0, 10].isnan().sum() == 1
    with torch.no_grad():
        y64, h64, _ = p.forward64(p.leaves())
    rows = [0, 1, 2, 4, 5, 6, 7, 11]
    close(y[0, rows], y64[0, rows], "y")
    close(h[0, rows], h64[0, rows], "h")
    # around a mean of 1000 every distance from it is off by up to 2^-24 of that: 6e-5
    assert (y[0, 3].double() - y64[0, 3]).abs().max() <= 5e-4
    g = bad.backward(y, stats)
    assert torch.isfinite(g.dx[0, fine]).all() and torch.isfinite(g.dbranch[0, fine]).all() and torch.isfinite(g.dgate[0, fine]).all()


@pytest.mark.parametrize("C", [64, 333, 8192])
def test_no_rows(C):
    p = Problem(1, 0, C, dtype="bf16", gate="token")
    y, h, stats = p.forward()
    assert y.shape == (1, 0, C) and h.shape == (1, 0, C) and stats.shape == (0, 4)
    g = p.backward(y, stats)
    for v in (g.dscale, g.dpost_weight, g.dpost_bias, g.dpre_weight, g.dpre_bias):
        assert (v == 0).all()


@pytest.mark.parametrize("C", [64, 136, 333, 4096, 6000])
def test_in_place_and_given_outputs(C):
    """y over x and dx over dy, outputs that are slices of wider tensors: the same bits, and nothing beside them is touched."""
    p = Problem(2, 29, C, dtype="bf16", gate="token", seed=C)
    y, h, stats = p.forward()
    g = p.backward(y, stats)
    wide = torch.full((2, 29, 2 * C + 16), 7.0, device="cuda", dtype=torch.bfloat16)
    x0, st = p.x.clone(), torch.empty_like(stats)
    p.x = x0.clone()
    y2, h2, st2 = p.forward(out=(p.x, wide[..., 8:8 + C], st))
    assert y2.data_ptr() == p.x.data_ptr() and st2 is st or torch.equal(st2, st)
    assert torch.equal(y2, y) and torch.equal(h2, h) and torch.equal(st, stats)
    assert (wide[..., :8] == 7).all() and (wide[..., 8 + C:] == 7).all()
    wide.fill_(7.0)
    dy = p.dy
    p.dy = dy.clone()
    g2 = p.backward(y, stats, out=(p.dy, wide[..., :C], wide[..., C + 8:2 * C + 8], None, None, None, None, None))
    for a, b in zip(g, g2):
        assert torch.equal(a, b)
    assert (wide[..., C:C + 8] == 7).all() and (wide[..., 2 * C + 8:] == 7).all()


def test_gate_rows_shared_by_few():
    """Groups of one, two and three rows, and one group of all rows."""
    for N in (1, 2, 3, 50):
        p = Problem(60 // N if N < 50 else 1, N, 72, dtype="f32", gate="item", gate_kind="sigmoid", seed=N)
        check_forward(p)
        check_backward(p)


def test_on_another_stream_and_captured():
    """Work queued behind a slow producer on a side stream; the same calls captured in a graph and replayed on new values."""
    p = Problem(2, 500, 256, dtype="bf16", gate="token", seed=4)
    want = p.forward()
    want_g = p.backward(want[0], want[2])
    side = torch.cuda.Stream()
    x = torch.zeros_like(p.x)
    src, p.x = p.x, x
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = torch.randn(4096, 4096, device="cuda")
        for _ in range(4):
            a = a @ a * 1e-2
        x.copy_(src)
    y, h, stats = p.forward(stream=side)
    g = p.backward(y, stats, stream=side)
    side.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(h, want[1])
    for u, v in zip(g, want_g):
        assert torch.equal(u, v)
    graph = torch.cuda.CUDAGraph()
    x.zero_()
    with torch.cuda.graph(graph):
        y, h, stats = p.forward()
        g = p.backward(y, stats)
    x.copy_(src)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want[0])
    for u, v in zip(g, want_g):
        assert torch.equal(u, v)


def test_repeated_calls_give_the_same_bits():
    p = Problem(4, 3000, 128, dtype="bf16", gate="item", gate_kind="linear", seed=6)
    y, _, stats = p.forward()
    first = p.backward(y, stats)
    for _ in range(3):
        for u, v in zip(first, p.backward(y, stats)):
            assert torch.equal(u, v)


def test_refusals():
    p = Problem(2, 5, 64, dtype="bf16", gate="token")
    y, h, stats = p.forward()
    n = p.pre
    with pytest.raises(ValueError, match="norm"):
        flare.block_norm(p.x, n._replace(kind="batch"))
    with pytest.raises(ValueError, match="weight"):
        flare.block_norm(p.x, n._replace(weight=torch.ones(63, device="cuda")))
    with pytest.raises(TypeError, match="float32"):
        flare.block_norm(p.x, n._replace(weight=torch.ones(64, device="cuda", dtype=torch.bfloat16)))
    with pytest.raises(TypeError, match="unsupported dtype"):
        flare.block_norm(p.x.double(), n)
    with pytest.raises(ValueError, match="CUDA"):
        flare.block_norm(p.x.cpu(), n)
    with pytest.raises(ValueError, match="rows of adjacent columns"):
        flare.block_norm(torch.empty(2, 64, 5, device="cuda", dtype=torch.bfloat16).mT, n)
    with pytest.raises(ValueError, match="rows of adjacent columns"):
        flare.block_join(p.x, torch.empty(5, 2, 64, device="cuda", dtype=torch.bfloat16).transpose(0, 1), pre=n)
    with pytest.raises(ValueError, match="branch"):
        flare.block_join(p.x, p.o[:, :4], pre=n)
    with pytest.raises(ValueError, match="gate"):
        flare.block_join(p.x, p.o, pre=n, gate=p.g[:1])
    with pytest.raises(ValueError, match="gate_kind"):
        flare.block_join(p.x, p.o, pre=n, gate=p.g, gate_kind="tanh")
    with pytest.raises(flare.FlareError) as e:
        flare.block_join(p.x, p.o.float(), pre=n)                # a 16-bit residual stream beside a float32 branch
    assert e.value.status == flare.ERR_UNSUPPORTED
    with pytest.raises(flare.FlareError) as e:
        flare.block_norm(p.x, n._replace(eps=-1.0))
    assert e.value.status == flare.ERR_INVALID_ARG
    with pytest.raises(flare.FlareError) as e:
        flare.block_norm(torch.zeros(1, 16392, device="cuda"), flare.Norm("rms"))
    assert e.value.status == flare.ERR_UNSUPPORTED
    with pytest.raises(flare.FlareError) as e:
        flare.block_join_backward(p.o, y, stats, None, None, post=p.post, pre=n, gate=p.g)
    assert e.value.status == flare.ERR_INVALID_ARG
    with pytest.raises(ValueError, match="shape"):
        flare.block_join_backward(p.o, y, stats[:3], p.dy, p.dh, post=p.post, pre=n, gate=p.g)
    lib = flare.load()
    desc = flare.FlareBlockDesc(rows=10, width=64, dtype=1, residual_dtype=1, pre_norm=1, pre_eps=1e-5, residual_scale=1.0)
    need = lib.flare_block_workspace_bytes(ctypes.byref(desc))
    dx = torch.empty_like(p.x)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    rc = lib.flare_norm_backward(ctypes.byref(desc), ptr(p.x), None, ptr(stats), None, ptr(p.dh), ptr(dx), None, None, ptr(dx), need - 1, None)
    assert rc == flare.ERR_WORKSPACE_TOO_SMALL
