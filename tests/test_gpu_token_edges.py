"""Calls of the token operators that a program may make and no other test does: inputs rewritten in place right before the call, one gradient without the other (needs a B200)."""
import ctypes

import pytest
import torch

from paper_2508_12594_b200 import flare
from tests.test_gpu_loss_outliers import Reference, problem
from tests._tokens import close

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("B,L,V,C,positions", [(4, 1000, 5000, 96, True), (1, 3000, 300, 512, False), (70, 64, 40, 24, True)])
def test_gradients_see_what_was_written_right_before_the_call(B, L, V, C, positions, accumulate):
    """Some of the gradient's launches begin beside the one before them: tokens, dy and the count of steps are what the copies right before the call have put into the same memory, every time."""
    g = torch.Generator(device="cuda").manual_seed(2)
    sets = [(torch.randint(-1, V, (B, L), device="cuda", generator=g), torch.randn(B, L, C, device="cuda", generator=g).to(BF16), torch.randn(V, C, device="cuda", generator=g),
             torch.randn(L, C, device="cuda", generator=g)) for _ in range(3)]
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = flare.Drop(0.25, 11, 5, step)

    def call(t, dy, out):
        return flare.embed_backward(t, dy, V, positions=L if positions else 0, drop=d, dtype=F32, accumulate=accumulate, out=out)

    want = []
    for i, (t, dy, a, b) in enumerate(sets):
        torch.cuda.synchronize()
        step.fill_(i)
        torch.cuda.synchronize()
        r = call(t, dy, (a.clone(), b.clone() if positions else None))
        torch.cuda.synchronize()
        want.append((r.dtable, r.dpositions))
    t, dy, a, b = (torch.empty_like(x) for x in sets[0])
    got = []
    for k in range(60):
        for to, of in zip((t, dy, a, b), sets[k % 3]):
            to.copy_(of)
        step.fill_(k % 3)
        call(t, dy, (a, b if positions else None))
        got.append((a.clone(), b.clone()))
    for k, (x, y) in enumerate(got):
        assert torch.equal(x, want[k % 3][0]), k
        assert not positions or torch.equal(y, want[k % 3][1]), k


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("rows,vocab,width,dtype", [
    (1, 1, 1, BF16), (3, 300, 40, F32), (300, 1000, 200, F16), (129, 257, 65, BF16), (2500, 12000, 264, BF16), (20000, 256, 128, BF16), (600, 50021, 64, F16), (1500, 6000, 384, F32),
    (70000, 5000, 64, F16), (70000, 5000, 64, BF16), (40000, 3400, 72, F32)], ids=str)      # (the last three: several pieces of the vocabulary)
def test_one_gradient_of_the_loss_alone(rows, vocab, width, dtype, weights):
    """Either is dealt out to the SMs by itself, so that its sums are added up in another order than beside the other."""
    x, w, labels, g = problem(max(rows, 2), vocab, width, dtype)
    x, labels = x[:rows].contiguous(), labels[:rows].clamp(max=vocab - 1).contiguous()
    dloss = torch.rand(rows, device="cuda", generator=g) / rows if weights else 1.0 / rows
    _, lse = flare.token_loss(x, w, labels)
    r = Reference(x, w, labels, dloss)
    dx, none = flare.token_loss_backward(x, w, labels, lse, dloss, check=True, want_dw=False)
    assert none is None
    close(dx, r.dx, r.dx_bound, "dx")
    none, dw = flare.token_loss_backward(x, w, labels, lse, dloss, check=True, want_dx=False)
    assert none is None
    close(dw, r.dw, r.dw_bound, "dw")


def test_one_gradient_of_the_loss_into_a_tensor():
    x, w, labels, _ = problem(300, 500, 80, BF16)
    _, lse = flare.token_loss(x, w, labels)
    want = flare.token_loss_backward(x, w, labels, lse, want_dx=False).dw
    out = torch.full_like(w, float("nan"))
    r = flare.token_loss_backward(x, w, labels, lse, out=(None, out), want_dx=False)
    assert r.dw.data_ptr() == out.data_ptr() and r.dx is None and torch.equal(out, want)
    for kw in (dict(want_dx=False, want_dw=False), dict(want_dw=False, out=(None, out)), dict(want_dx=False, out=(x.clone(), None))):
        with pytest.raises(ValueError):
            flare.token_loss_backward(x, w, labels, lse, **kw)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("B,L,V,C,table,out", [(1, 1, 1, 1, F32, F32), (4, 1000, 5000, 96, F32, BF16), (70, 64, 40, 24, F16, F16), (200, 33, 300, 520, BF16, BF16), (2, 3000, 100, 333, F32, F32)], ids=str)
def test_one_gradient_of_the_embedding_alone(B, L, V, C, table, out, accumulate):
    """The same numbers as beside the other, which is not touched: positions without the table (no sort), the table without positions, through the C-ABI."""
    g = torch.Generator(device="cuda").manual_seed(B + C)
    t = torch.randint(-1, V, (B, L), device="cuda", generator=g)
    dy = torch.randn(B, L, C, device="cuda", generator=g).to(out)
    a, b = torch.randn(V, C, device="cuda", generator=g).to(table), torch.randn(L, C, device="cuda", generator=g).to(table)
    d = flare.Drop(0.2, 3, 4)
    want = flare.embed_backward(t, dy, V, positions=L, scale=2.0, drop=d, dtype=table, accumulate=accumulate, out=(a.clone(), b.clone()))
    got = b.clone()
    r = flare.embed_backward(t, dy, V, positions=L, scale=2.0, drop=d, dtype=table, accumulate=accumulate, out=(None, got), want_dtable=False)
    assert r.dtable is None and torch.equal(got, want.dpositions)
    lib, code = flare.load(), {F32: flare.DTYPE_F32, BF16: flare.DTYPE_BF16, F16: flare.DTYPE_F16}
    desc = flare.FlareEmbedDesc(rows=B * L, positions=L, width=C, vocab=V, dtype=code[table], out_dtype=code[out], token_bits=64, scale=2.0)
    drop = flare.FlareDrop(0.2, 3, 4, None)
    need = lib.flare_embed_workspace_bytes(ctypes.byref(desc))
    ws, got = torch.empty(need, dtype=torch.uint8, device="cuda"), a.clone()
    torch.cuda.synchronize()
    assert lib.flare_embed_backward(ctypes.byref(desc), ctypes.byref(drop), t.data_ptr(), dy.data_ptr(), got.data_ptr(), None, int(accumulate), ws.data_ptr(), need, None) == flare.OK
    assert lib.flare_embed_backward(ctypes.byref(desc), ctypes.byref(drop), t.data_ptr(), dy.data_ptr(), None, None, int(accumulate), ws.data_ptr(), need, None) == flare.OK      # (neither: nothing)
    torch.cuda.synchronize()
    assert torch.equal(got, want.dtable)


def test_one_gradient_of_the_embedding_is_refused():
    t, dy = torch.zeros(2, 8, dtype=torch.int64, device="cuda"), torch.zeros(2, 8, 16, device="cuda")
    for kw in (dict(want_dtable=False), dict(positions=8, want_dtable=False, out=(torch.zeros(5, 16, device="cuda"), None)), dict(positions=8, want_dtable=False, accumulate=True)):
        with pytest.raises(ValueError):
            flare.embed_backward(t, dy, 5, **kw)


@pytest.mark.parametrize("rows,vocab,width,dtype", [(8, 300000, 8, BF16), (3, 1000, 64, F32), (6, 5000, 64, F16), (300, 1000, 64, BF16), (300, 5000, 64, F16), (300, 500, 64, F32)], ids=str)
@pytest.mark.parametrize("off", [(0, 0), (1, 0), (0, 1), (1, 1)], ids=str)
def test_the_scratch_that_is_asked_for_is_enough(rows, vocab, width, dtype, off):
    """Through the C-ABI, x and w on 16-byte boundaries or not, with a workspace of just the size that is given without and, where they are, with FLARE_LOSS_ALIGNED; what lies behind it stays as it is."""
    x, w, labels, _ = problem(rows, vocab, width, dtype)
    x, w = (torch.cat([torch.zeros(o, device="cuda", dtype=dtype), t.reshape(-1)])[o:].view(t.shape) for t, o in zip((x, w), off))
    want = flare.token_loss(x, w, labels)
    d = flare.token_loss_backward(x, w, labels, want[1])
    lib, code = flare.load(), {F32: flare.DTYPE_F32, BF16: flare.DTYPE_BF16, F16: flare.DTYPE_F16}
    desc = flare.FlareLossDesc(rows=rows, width=width, vocab=vocab, dtype=code[dtype], label_bits=64, scale=1.0, dloss_scale=1.0)
    for aligned in (0, 2):
        loss, lse, dx, dw = torch.empty_like(want[0]), torch.empty_like(want[1]), torch.empty_like(x), torch.empty_like(w)
        for backward in (0, 1):
            need = lib.flare_loss_workspace_bytes(ctypes.byref(desc), backward | aligned)
            ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            p = [t.data_ptr() for t in (x, w, labels, lse, loss, dx, dw, ws)]
            if backward:
                status = lib.flare_loss_backward(ctypes.byref(desc), p[0], p[1], p[2], p[3], None, p[5], p[6], p[7], need, None)
            else:
                status = lib.flare_loss_forward(ctypes.byref(desc), p[0], p[1], p[2], p[4], p[3], p[7], need, None)
            torch.cuda.synchronize()
            assert (ws[need:] == 0x5A).all()
            if aligned and any(off):
                assert status in (flare.OK, flare.ERR_WORKSPACE_TOO_SMALL)
                if status != flare.OK:
                    break
            assert status == flare.OK
        else:
            assert torch.equal(loss, want[0]) and torch.equal(lse, want[1]) and torch.equal(dx, d.dx) and torch.equal(dw, d.dw)
