"""Fine-tunes the adapters of SALR layers under a frozen language-model head: the layers' forward and backward pass, the head's
loss without storing its logits, clipping, and an optimiser step over all adapters, each on the GPU through the library's kernels.

    python examples/finetune_adapters.py --steps 60 --bits 8

The model is a stack of residual blocks h = h + layer(h) on embedded tokens, with random pruned weights and a random head; what it
learns is a fixed map from token to next token.  Prints the mean loss of the unmasked tokens.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_16991_amd as salr  # noqa: E402


class Layer:
    """One SALR layer [K -> K] with a trainable adapter: fp32 master weights, the bf16 copies that the kernels read, and gradients
    that the backward pass writes in place."""

    def __init__(self, K: int, R: int, gen: torch.Generator):
        w = torch.empty(K, K, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.3 / K ** 0.5, generator=gen)
        self.bitmap, self.values, self.offsets = salr.encode(salr.mask_rows(w, K - K // 2))
        self.master = [torch.randn(K, R, device="cuda", generator=gen) / K ** 0.5, torch.zeros(R, K, device="cuda")]
        self.copy = [p.to(torch.bfloat16) for p in self.master]
        self.grad = [torch.empty_like(c) for c in self.copy]

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        self.x = x
        return salr.linear(x, self.bitmap, self.values, self.offsets, *self.copy)

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        M, K = dy.shape
        dx = torch.empty_like(dy)
        need = salr.salr_linear_backward_workspace_bytes(M, K, K, self.copy[0].shape[1], True, True)
        workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        salr.salr_sparse_lowrank_linear_backward(self.x, dy, self.bitmap, self.values, self.offsets, *self.copy, dx, *self.grad, workspace)
        return dx


def train(steps: int = 60, T: int = 512, K: int = 512, V: int = 4099, R: int = 16, depth: int = 2, bits: int = 32, lr: float = 3e-3,
          max_norm: float = 1.0, seed: int = 0, log=print) -> list[float]:
    gen = torch.Generator(device="cuda").manual_seed(seed)
    layers = [Layer(K, R, gen) for _ in range(depth)]
    embedding = torch.randn(64, K, device="cuda", generator=gen).to(torch.bfloat16)
    head = torch.empty(V, K, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0 / K ** 0.5, generator=gen)
    follower = torch.randint(0, V, (64,), device="cuda", generator=gen)   # what comes after each token

    optimizer = salr.AdamW([p for l in layers for p in l.master], [g for l in layers for g in l.grad], copies=[c for l in layers for c in l.copy],
                           bits=bits)
    workspace = torch.empty(salr.salr_linear_cross_entropy_workspace_bytes(T, K, V, True, False), dtype=torch.uint8, device="cuda")
    losses = []
    for step in range(1, steps + 1):
        tokens = torch.randint(0, 64, (T,), device="cuda", generator=gen)
        targets = follower[tokens]
        targets[: T // 8] = -100   # a prompt: not trained on
        h = embedding[tokens]
        for layer in layers:
            h = h + layer.forward(h)
        loss, _, dh, _ = salr.linear_cross_entropy(h, head, targets, torch.full((T,), 1.0 / (T - T // 8), device="cuda"), workspace=workspace)
        for layer in reversed(layers):
            dh = dh + layer.backward(dh)
        norm = optimizer.grad_norm(max_norm)
        optimizer.step(lr=lr, step=step, weight_decay=0.01, grad_scale=norm[1:], seed=step)
        losses.append(loss.sum() / (T - T // 8))
        if log and (step == 1 or step % 10 == 0):
            log(f"step {step:4d}  loss {float(losses[-1]):.4f}  gradient norm {float(norm[0]):.4f}")
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=512, help="a multiple of 32 (the backward pass of the layers wants that)")
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32)
    args = ap.parse_args()
    train(args.steps, T=args.tokens, bits=args.bits)
