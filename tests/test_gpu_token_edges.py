"""Calls of the token operators that a program may make and no other test does: inputs rewritten in place right before the call (needs a B200)."""
import pytest
import torch

from paper_2508_12594_b200 import flare

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
