"""A small model over token sequences: embedding, one FLARE block, loss over the vocabulary with the embedding's table as its weights, trained on synthetic
sequences: the operators over tokens, the mixer, the norms and join around it and the orthogonalised updates, as a training step uses them together.

    python examples/flare_tokens.py           # 40 steps on 8 sequences of 2048 tokens

    x = drop(s E[t] + P);  h = LN(x);  K, V = h Wk, h Wv;  o = mixer(Q, K, V) Wo;  d = drop(o);  y = x + scale d;  f = RMS(y);  loss = CE(f E^T, labels)

Everything between the projections (plain matrix products) runs in the library's kernels, forward and backward; tokens that are padding are none (-1) at both ends and
masked in the mixer.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_12594_b200 import flare  # noqa: E402


class Model:
    """Parameters in float32, activations, mixer and loss in bfloat16, residual stream in float32."""

    def __init__(self, vocab=256, length=2048, heads=4, latents=64, width=16, p=0.1, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        C = heads * width
        self.vocab, self.H, self.D, self.C, self.p = vocab, heads, width, C, p

        def rand(*s, scale=1.0):
            return torch.randn(*s, device=device, generator=g) * scale

        self.E, self.P = rand(vocab, C, scale=C ** -0.5), rand(length, C, scale=0.3)
        self.W = rand(3, C, C, scale=C ** -0.5)                   # Wk, Wv, Wo
        self.Q = rand(heads, latents, width)
        self.scale = torch.full((C,), 0.5, device=device)
        self.norm_in = flare.Norm("layer", torch.ones(C, device=device), torch.zeros(C, device=device))
        self.norm_out = flare.Norm("rms", torch.ones(C, device=device))
        self.momentum = torch.zeros_like(self.W), torch.zeros_like(self.Q)
        self.seed, self.step_count = seed, torch.zeros(1, dtype=torch.int64, device=device)

    def drops(self):
        """Dropout behind the embedding and behind the block: one generator each, counted up by the step."""
        return tuple(flare.Drop(self.p, self.seed * 2 + i, 0, self.step_count) for i in range(2))

    def gradients(self, tokens, labels):
        """tokens, labels [B, N] (outside [0, vocab): none) -> (loss, dE, dP, dW, dQ, gradients of the norms' weights and biases and of scale)."""
        B, N = tokens.shape
        C, bf16 = self.C, torch.bfloat16
        heads = (B, N, self.H, self.D)
        W, Q, E = self.W.to(bf16), self.Q.to(bf16), self.E.to(bf16)
        drop_in, drop_block = self.drops()
        mask = ((tokens >= 0) & (tokens < self.vocab)).to(torch.uint8)
        grow = C ** 0.5

        x = flare.embed(tokens, self.E, positions=self.P, scale=grow, drop=drop_in)
        h, stats = flare.block_norm(x, self.norm_in, dtype=bf16)
        K, V = ((h @ W[i]).view(heads) for i in range(2))
        Y, Z, lse_enc, lse_dec = flare.forward(Q, K, V, key_mask=mask, want_stats=True)
        o = flare.dropout(Y.view(B, N, C) @ W[2], drop_block)
        y, f, join_stats = flare.block_join(x, o, pre=self.norm_out, scale=self.scale)
        losses, lse = flare.token_loss(f, E, labels)
        weight = 1.0 / max(1, int(((labels >= 0) & (labels < self.vocab)).sum()))

        d = flare.token_loss_backward(f, E, labels, lse, weight)
        j = flare.block_join_backward(o, y, join_stats, None, d.dx, pre=self.norm_out, scale=self.scale)
        do = flare.dropout_backward(j.dbranch, drop_block)
        dY = (do @ W[2].mT).view(heads)
        desc = flare.make_desc(Q, K)
        dQ, dK, dV = torch.empty_like(self.Q), torch.empty_like(K), torch.empty_like(V)
        flare.flare_backward(desc, Q, K, V, mask, Y, dY, Z, lse_enc, lse_dec, dQ, dK, dV, flare.alloc_workspace(desc, flare.OP_BACKWARD))
        dK, dV = dK.view(B, N, C), dV.view(B, N, C)
        n = flare.block_norm_backward(x, stats, dK @ W[0].mT + dV @ W[1].mT, self.norm_in, dy=j.dx)
        # the table is the loss's too: what comes from the lookup is added to what came from there
        dE, dP = d.dw.float(), torch.zeros_like(self.P)
        flare.embed_backward(tokens, n.dx, self.vocab, positions=N, scale=grow, drop=drop_in, accumulate=True, out=(dE, dP))
        rows = h.view(-1, C).mT
        dW = torch.stack([rows @ dK.view(-1, C), rows @ dV.view(-1, C), Y.view(-1, C).mT @ do.view(-1, C)])
        return losses.sum() * weight, dE, dP, dW, dQ, [n.dweight, n.dbias, j.dscale, j.dpre_weight]

    def step(self, tokens, labels, lr=0.02, vector_lr=0.1):
        loss, dE, dP, dW, dQ, dv = self.gradients(tokens, labels)
        flare.muon_update(self.W, self.momentum[0], dW, lr)
        flare.muon_update(self.Q, self.momentum[1], dQ, lr)
        for p, d in zip([self.E, self.P, self.norm_in.weight, self.norm_in.bias, self.scale, self.norm_out.weight], [dE, dP, *dv]):
            p.sub_(d, alpha=vector_lr)
        self.step_count.add_(1)
        return loss


def sequences(B=8, N=2048, vocab=256, padding=0.1, seed=1, device="cuda"):
    """Tokens of which a few are frequent, each sequence padded by up to `padding` of its length; every token's label is the one in front of it."""
    g = torch.Generator(device=device).manual_seed(seed)
    t = (torch.rand(B, N, device=device, generator=g).pow(3) * vocab).long()
    length = N - (torch.rand(B, 1, device=device, generator=g) * padding * N).long()
    t = torch.where(torch.arange(N, device=device) < length, t, torch.full_like(t, -1))
    labels = torch.cat([torch.full_like(t[:, :1], -1), t[:, :-1]], 1)
    return t, torch.where(t >= 0, labels, torch.full_like(t, -1))


def train(steps=40, B=8, N=2048, verbose=False):
    model, (tokens, labels) = Model(length=N), sequences(B, N)
    losses = []
    for i in range(steps):
        losses.append(model.step(tokens, labels))
        if verbose and i % 10 == 0:
            print(f"step {i}: loss {float(losses[-1]):.4f}")
    return [float(v) for v in losses]


if __name__ == "__main__":
    result = train(verbose=True)
    print(f"loss {result[0]:.4f} -> {result[-1]:.4f}")
