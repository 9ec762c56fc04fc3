"""The example block: its gradients against float64 automatic differentiation of the same block, and a short training (needs a B200)."""
import pytest
import torch

from examples import flare_block

pytestmark = pytest.mark.gpu


def reference(block, x, target):
    """Loss and gradients in float64, weights and latents rounded to bfloat16 as the block uses them."""
    d = lambda t: t.double().clone().requires_grad_(True)  # noqa: E731
    W, Q, s, w = d(block.W.bfloat16()), d(block.Q.bfloat16()), d(block.s), d(block.w)
    norms = [d(t) for n in (block.norm_in, block.norm_out) for t in (n.weight, n.bias)]
    x = x.double()

    def ln(v, weight, bias):
        v = v - v.mean(-1, keepdim=True)
        return v / (v.square().mean(-1, keepdim=True) + 1e-5).sqrt() * weight + bias

    B, N, C = x.shape
    h = ln(x, norms[0], norms[1])
    heads = lambda t: t.view(B, N, block.H, block.D).transpose(1, 2)  # noqa: E731
    K, V, g = heads(h @ W[0]), heads(h @ W[1]), h @ W[2]
    S = Q @ K.mT
    Z = S.softmax(-1) @ V
    Y = (S.mT.softmax(-1) @ Z).transpose(1, 2).reshape(B, N, C)
    y = x + s * g.sigmoid() * (Y @ W[3])
    p = ln(y, norms[2], norms[3]) @ w
    loss = (p - target.double()).square().mean()
    return loss.detach(), torch.autograd.grad(loss, [W, Q, norms[0], norms[1], s, norms[2], norms[3], w])


def test_gradients_of_the_block():
    block, (x, target) = flare_block.Block(heads=4, latents=32, width=16, seed=3), flare_block.field(2, 500, 64, seed=4)
    loss, dW, dQ, dv = block.gradients(x, target)
    ref, grads = reference(block, x, target)
    assert abs(float(loss) - float(ref)) <= 1e-2 * float(ref)
    for got, want in zip([dW, dQ, *dv], grads):
        # half a dozen bfloat16 roundings (2^-8 each) of the activations on the way, 2-norm
        assert float((got.double() - want).norm() / want.norm()) <= 6 * 2.0 ** -8


def test_a_short_training_learns():
    losses = flare_block.train(steps=30, B=2, N=4096)
    assert losses[-1] < 0.5 * losses[0], losses
