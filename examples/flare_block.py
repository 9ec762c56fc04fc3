"""One FLARE block, X += FLARE(LN(X)) with a gate and a residual scale, trained on a synthetic field: the token mixer, the norms and the join around
it and the orthogonalised updates of its matrices, as a training step uses them together.

    python examples/flare_block.py            # 50 steps on 4 clouds of 16384 points

    h = LN(x);  K, V, g = h Wk, h Wv, h Wg;  o = mixer(Q, K, V) Wo;  y = x + s sigmoid(g) o;  p = LN(y) w;  loss = mean (p - target)^2

Everything between the projections (plain matrix products) runs in the library's kernels, forward and backward.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_12594_b200 import flare  # noqa: E402


class Block:
    """Parameters in float32, activations and mixer in bfloat16, residual stream in float32."""

    def __init__(self, heads=8, latents=64, width=16, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        C = heads * width
        self.H, self.D, self.C = heads, width, C

        def rand(*s, scale=1.0):
            return torch.randn(*s, device=device, generator=g) * scale

        self.W = rand(4, C, C, scale=C ** -0.5)                  # Wk, Wv, Wg, Wo
        self.Q = rand(heads, latents, width)
        self.w = rand(C, scale=C ** -0.5)
        self.s = torch.full((C,), 0.5, device=device)
        self.norm_in = flare.Norm("layer", torch.ones(C, device=device), torch.zeros(C, device=device))
        self.norm_out = flare.Norm("layer", torch.ones(C, device=device), torch.zeros(C, device=device))
        self.momentum = torch.zeros_like(self.W), torch.zeros_like(self.Q)

    def vectors(self):
        """The parameters that are not matrices, in the order of `gradients`."""
        return [self.norm_in.weight, self.norm_in.bias, self.s, self.norm_out.weight, self.norm_out.bias, self.w]

    def gradients(self, x, target):
        """x [B, N, C] float32, target [B, N] -> (loss, dW [4, C, C], dQ, gradients of vectors())."""
        B, N, C = x.shape
        heads = (B, N, self.H, self.D)
        bf16 = torch.bfloat16
        W, Q = self.W.to(bf16), self.Q.to(bf16)
        h, stats = flare.block_norm(x, self.norm_in, dtype=bf16)
        K, V, g = (h @ W[i] for i in range(3))
        K, V = K.view(heads), V.view(heads)
        Y, Z, lse_enc, lse_dec = flare.forward(Q, K, V, want_stats=True)
        o = Y.view(B, N, C) @ W[3]
        y, out, join_stats = flare.block_join(x, o, pre=self.norm_out, gate=g, scale=self.s)
        miss = out.float() @ self.w - target
        loss = miss.square().mean()

        dp = miss * (2.0 / miss.numel())
        dw = torch.einsum("bnc,bn->c", out.float(), dp)
        dout = (dp[..., None] * self.w).to(bf16)
        j = flare.block_join_backward(o, y, join_stats, None, dout, pre=self.norm_out, gate=g, scale=self.s)
        dY = (j.dbranch @ W[3].mT).view(heads)
        desc = flare.make_desc(Q, K)
        dQ, dK, dV = torch.empty_like(self.Q), torch.empty_like(K), torch.empty_like(V)
        flare.flare_backward(desc, Q, K, V, None, Y, dY, Z, lse_enc, lse_dec, dQ, dK, dV, flare.alloc_workspace(desc, flare.OP_BACKWARD))
        dK, dV = dK.view(B, N, C), dV.view(B, N, C)
        dh = dK @ W[0].mT + dV @ W[1].mT + j.dgate @ W[2].mT
        n = flare.block_norm_backward(x, stats, dh, self.norm_in, dy=j.dx)
        rows = h.view(-1, C).mT
        dW = torch.stack([rows @ dK.view(-1, C), rows @ dV.view(-1, C), rows @ j.dgate.view(-1, C), Y.view(-1, C).mT @ j.dbranch.view(-1, C)])
        return loss, dW, dQ, [n.dweight, n.dbias, j.dscale, j.dpre_weight, j.dpre_bias, dw]

    def step(self, x, target, lr=0.02, vector_lr=0.1):
        loss, dW, dQ, dv = self.gradients(x, target)
        flare.muon_update(self.W, self.momentum[0], dW, lr)
        flare.muon_update(self.Q, self.momentum[1], dQ, lr)
        for p, d in zip(self.vectors(), dv):
            p.sub_(d, alpha=vector_lr)
        return loss


def field(B=4, N=16384, C=128, seed=1, device="cuda"):
    """Points of a cloud with C features each, and a smooth function of where they are and of the cloud as a whole."""
    g = torch.Generator(device=device).manual_seed(seed)
    x = torch.randn(B, N, C, device=device, generator=g)
    xy = torch.rand(B, N, 2, device=device, generator=g)
    x[..., :2] = xy * 4.0 - 2.0
    return x, torch.sin(3.0 * xy[..., 0]) * xy[..., 1] + x[..., 2].mean(-1, keepdim=True) + 0.3 * x[..., 3]


def train(steps=50, B=4, N=16384, verbose=False):
    block, (x, target) = Block(), field(B, N)
    losses = []
    for i in range(steps):
        losses.append(block.step(x, target))
        if verbose and i % 10 == 0:
            print(f"step {i}: loss {float(losses[-1]):.4f}")
    return [float(v) for v in losses]


if __name__ == "__main__":
    result = train(verbose=True)
    print(f"loss {result[0]:.4f} -> {result[-1]:.4f}")
