"""Joins whose two norms differ, and rows beyond what 32 bits count, against float64 (needs a B200).

Bounds: those of tests.test_gpu_block (a float32 row result, a difference that cancels, a sum over rows).
"""
import pytest
import torch

from paper_2508_12594_b200 import flare
from tests.test_gpu_block import DT, close, ref_norm, size, sum_close

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")]
# which parameters the two norms have: (post weight, post bias, pre weight, pre bias)
PARAMETERS = [(True, False, False, True), (False, True, True, False), (True, False, True, False), (False, False, True, True)]


@pytest.mark.parametrize("C", [72, 264, 333, 1024, 2056, 4360, 8192])
@pytest.mark.parametrize("kinds", [("layer", "rms"), ("rms", "layer")], ids="-".join)
@pytest.mark.parametrize("gate", ["none", "token", "item"])
@pytest.mark.parametrize("types", TYPES, ids=str)
def test_norms_that_differ(C, kinds, gate, types):
    """A layer norm on one side and an rms norm on the other, parameters on one of them only, an eps of its own each, large enough to be seen."""
    k = (C + len(gate)) % 4
    T, R, B, N = DT[types[0]], DT[types[1]], 2, 7
    gen = torch.Generator(device="cuda").manual_seed(C + k)

    def rand(*s, dt=torch.float32, mean=0.0, scale=1.0):
        return (torch.randn(*s, device="cuda", generator=gen) * scale + mean).to(dt)

    x, o, dy, dh = rand(B, N, C, dt=R, mean=0.5), rand(B, N, C, dt=T, mean=-0.5), rand(B, N, C, dt=R), rand(B, N, C, dt=T)
    g = None if gate == "none" else rand(B, N, C, dt=T) if gate == "token" else rand(B, C, dt=T)
    s, alpha = rand(C, mean=0.5, scale=0.3), 1.3
    has = PARAMETERS[k]
    post = flare.Norm(kinds[0], rand(C, mean=1.0, scale=0.2) if has[0] else None, rand(C, scale=0.3) if has[1] else None, 0.1)
    pre = flare.Norm(kinds[1], rand(C, mean=1.0, scale=0.2) if has[2] else None, rand(C, scale=0.3) if has[3] else None, 0.01)
    D = lambda t: None if t is None else t.double()  # noqa: E731

    def definition(o, g, s, w, b):
        n, mean, rstd = ref_norm(o, post.kind, w, b, post.eps)
        a = 1.0 if g is None else torch.sigmoid(g)
        a = a[:, None, :] if g is not None and g.dim() == 2 else a
        return alpha * x.double() + s * a * n, (o - mean) * rstd, mean, rstd, a

    leaf = [None if t is None else t.double().requires_grad_(True) for t in (o, g, s, post.weight, post.bias)]
    y64, o_hat, mean_o, rstd_o, a = definition(*leaf)
    with torch.no_grad():
        h64, mean, rstd = ref_norm(y64, pre.kind, D(pre.weight), D(pre.bias), pre.eps)
    y, h, stats = flare.block_join(x, o, post=post, pre=pre, gate=g, scale=s, residual_scale=alpha)
    close(y, y64.detach(), "y")
    close(h, h64, "h")
    st64 = torch.cat([t.detach().expand(B, N, 1) for t in (mean_o, rstd_o, mean, rstd)], -1).reshape(-1, 4)
    assert ((stats[:, 0::2].double() - st64[:, 0::2]).abs() <= 2e-6 * (1.0 + x.double().abs().max() + o.double().abs().max())).all()
    close(stats[:, 1::2], st64[:, 1::2], "rstd")

    st = st64.float().contiguous()
    yr = y64.detach().to(R)
    got = flare.block_join_backward(o, yr, st, dy, dh, post=post, pre=pre, gate=g, scale=s, residual_scale=alpha)
    with torch.no_grad():
        hat = (yr.double() - st.double().view(B, N, 4)[..., 2:3]) * st.double().view(B, N, 4)[..., 3:4]
        d = dh.double() if pre.weight is None else dh.double() * pre.weight.double()
        inner = d - hat * (d * hat).mean(-1, keepdim=True) - (d.mean(-1, keepdim=True) if pre.kind == "layer" else 0.0)
        r = st.double().view(B, N, 4)[..., 3:4]
        dt = dy.double() + r * inner
    close(got.dx, alpha * dt, "dx", size(r * d))
    present = [t for t in leaf if t is not None]
    grads = iter(torch.autograd.grad(y64, present, dt))
    do, dg, ds, dw, db = (next(grads) if t is not None else None for t in leaf)
    with torch.no_grad():
        w, b = 1.0 if post.weight is None else D(post.weight).abs(), 0.0 if post.bias is None else D(post.bias).abs()
        close(got.dbranch, do, "dbranch", size((dt * a).abs() * s.double().abs() * w * rstd_o))
        rows = (0, 1)
        sum_close(got.dscale, ds, torch.maximum((dt * a).abs() * (o_hat.abs() * w + b), (dt * a).abs() * 1e-30), rows, "dscale")
        for value, want, terms, name in ((got.dpost_weight, dw, dt * a * s * o_hat, "dpost_weight"), (got.dpost_bias, db, (dt * a * s).expand_as(dt), "dpost_bias")):
            assert (value is None) == (want is None), name
            if want is not None:
                sum_close(value, want, terms, rows, name)
        for value, p, terms, name in ((got.dpre_weight, pre.weight, dh.double() * hat, "dpre_weight"), (got.dpre_bias, pre.bias, dh.double(), "dpre_bias")):
            assert (value is None) == (p is None), name
            if p is not None:
                sum_close(value, terms.sum(rows), terms, rows, name)
        if gate == "token":
            close(got.dgate, dg, "dgate")
        elif gate == "item":
            slope = torch.sigmoid(g.double()) * (1 - torch.sigmoid(g.double()))
            each = dt.abs() * (o_hat.abs() * w + b) * s.double().abs()
            half = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[T]
            bound = 1e-5 * slope * (each.sum(1) + N * size(each)) + half * dg.abs() + (2.0 ** -25 if T == torch.float16 else 0.0)
            assert ((got.dgate.double() - dg).abs() <= bound).all(), "dgate"
        else:
            assert got.dgate is None


@pytest.mark.parametrize("rows,C", [(8_400_000, 256), (6_460_000, 333)], ids=str)
def test_more_elements_than_32_bits_count(rows, C):
    """2.15 billion in every tensor: rows at both ends and around every 2^30th element are those of a call of their own."""
    assert rows * C > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(5)

    def rand():
        t = torch.empty(rows, C, device="cuda", dtype=torch.bfloat16)
        for i in range(0, rows, 1 << 20):
            t[i:i + (1 << 20)].normal_(generator=gen)
        return t

    x, o, g = rand(), rand(), rand()
    w = torch.rand(C, device="cuda") + 0.5
    norm = flare.Norm("layer", w, w - 1.0)
    places = [slice(0, 100)] + [slice(c - 50, c + 50) for c in (k * (1 << 30) // C for k in (1, 2)) if c + 50 < rows] + [slice(rows - 100, rows)]
    y, h, stats = flare.block_join(x, o, post=norm, pre=norm, gate=g, scale=w)
    for p in places:
        a, b, c = flare.block_join(x[p].clone(), o[p].clone(), post=norm, pre=norm, gate=g[p].clone(), scale=w)
        assert torch.equal(y[p], a) and torch.equal(h[p], b) and torch.equal(stats[p], c), p
    # backward: dy = x, dh = h; over dx = x
    r = flare.block_join_backward(o, y, stats, x, h, post=norm, pre=norm, gate=g, scale=w)
    for p in places:
        q = flare.block_join_backward(o[p].clone(), y[p].clone(), stats[p].clone(), x[p].clone(), h[p].clone(), post=norm, pre=norm, gate=g[p].clone(), scale=w)
        assert torch.equal(r.dx[p], q.dx) and torch.equal(r.dbranch[p], q.dbranch) and torch.equal(r.dgate[p], q.dgate), p
    # a sum over rows, by parts of them
    total = torch.zeros(C, device="cuda", dtype=torch.float64)
    size_of_terms = torch.zeros_like(total)
    for i in range(0, rows, 1 << 18):
        d = h[i:i + (1 << 18)].double()
        total += d.sum(0)
        size_of_terms += d.abs().sum(0)
    assert ((r.dpre_bias.double() - total).abs() <= 1e-5 * size_of_terms).all()
    del x, o, g, y, h, stats, r
    torch.cuda.empty_cache()
