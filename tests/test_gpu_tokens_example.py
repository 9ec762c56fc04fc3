"""The example over tokens: its gradients against float64 automatic differentiation of the same model, with the same elements dropped; that it runs (needs a B200)."""
import pytest
import torch

from examples import flare_tokens
from tests._tokens import factors

pytestmark = pytest.mark.gpu


def reference(model, tokens, labels):
    """Loss and gradients in float64, weights, latents and the loss's table rounded to bfloat16 as the model uses them."""
    d = lambda t: t.double().clone().requires_grad_(True)  # noqa: E731
    B, N = tokens.shape
    C = model.C
    W, Q, E, Eb, P, scale = d(model.W.bfloat16()), d(model.Q.bfloat16()), d(model.E), d(model.E.bfloat16()), d(model.P), d(model.scale)
    w_in, b_in, w_out = d(model.norm_in.weight), d(model.norm_in.bias), d(model.norm_out.weight)
    count = int(model.step_count)
    f1, f2 = (factors(B * N, C, model.p, x.seed, count).cuda().view(B, N, C) for x in model.drops())
    there = (tokens >= 0) & (tokens < model.vocab)
    x = (E[tokens.clamp(min=0)] * C ** 0.5 * there[..., None] + P) * f1
    v = x - x.mean(-1, keepdim=True)
    h = v / (v.square().mean(-1, keepdim=True) + 1e-5).sqrt() * w_in + b_in
    heads = lambda t: t.view(B, N, model.H, model.D).transpose(1, 2)  # noqa: E731
    K, V = heads(h @ W[0]), heads(h @ W[1])
    S = Q @ K.mT
    Z = S.masked_fill(~there[:, None, None, :], float("-inf")).softmax(-1) @ V
    Y = (S.mT.softmax(-1) @ Z).transpose(1, 2).reshape(B, N, C)
    y = x + scale * (f2 * (Y @ W[2]))
    f = y / (y.square().mean(-1, keepdim=True) + 1e-5).sqrt() * w_out
    loss = torch.nn.functional.cross_entropy((f @ Eb.mT).view(-1, model.vocab), labels.view(-1), ignore_index=-1)
    dE, dEb, *rest = torch.autograd.grad(loss, [E, Eb, P, W, Q, w_in, b_in, scale, w_out])
    return loss.detach(), [dE + dEb, *rest]


@pytest.mark.parametrize("p", [0.0, 0.2])
def test_gradients_of_the_model(p):
    model = flare_tokens.Model(vocab=300, length=400, heads=4, latents=32, width=16, p=p, seed=3)
    tokens, labels = flare_tokens.sequences(3, 400, 300, seed=4)
    model.step_count.fill_(7)
    loss, dE, dP, dW, dQ, dv = model.gradients(tokens, labels)
    ref, grads = reference(model, tokens, labels)
    assert abs(float(loss) - float(ref)) <= 1e-2 * float(ref)
    for got, want in zip([dE, dP, dW, dQ, *dv], grads, strict=True):
        # bfloat16 roundings (2^-8 each at most) of the activations on the way: h, K and V, the mixer's Y, Y Wo, what dropout makes of it, f, and as many of their gradients; 2-norm
        assert float((got.double() - want).norm() / want.norm()) <= 12 * 2.0 ** -8


def test_a_few_steps_run():
    losses = flare_tokens.train(steps=3, B=2, N=512)
    assert len(losses) == 3 and all(v == v for v in losses)
