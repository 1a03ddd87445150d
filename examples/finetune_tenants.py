"""Fine-tunes the adapters of several tenants at once beside one frozen SALR model: every sequence of a batch belongs to a tenant, the layers' pruned weights are
shared, and each tenant has its own adapters, trained on dropped-out inputs behind a layer norm.

    python examples/finetune_tenants.py --steps 60 --tenants 4

The model is a stack of residual blocks h = h + layer(norm(h)) on embedded tokens, with random pruned weights and a random head; what tenant i learns is a
fixed map of its own from token to next token.  Prints the mean loss of the unmasked tokens.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_16991_amd as salr  # noqa: E402


class Block:
    """h + layer(norm(h)): a frozen SALR layer [K -> K] shared by all tenants, a norm that is trained with them, and an adapter for each tenant."""

    def __init__(self, K: int, ranks, dropout: float, number: int, gen: torch.Generator):
        w = torch.empty(K, K, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.3 / K ** 0.5, generator=gen)
        self.weight = salr.encode(salr.mask_rows(w, K - K // 2))
        n = len(ranks)
        self.master = [torch.randn(K, r, device="cuda", generator=gen) / K ** 0.5 for r in ranks] + [torch.zeros(r, K, device="cuda") for r in ranks]
        self.copy = [p.to(torch.bfloat16) for p in self.master]
        self.grad = [torch.empty_like(c) for c in self.copy]
        self.adapters = salr.AdapterSet(self.copy[:n], self.copy[n:], self.grad[:n], self.grad[n:])
        self.norm = [torch.ones(K, device="cuda"), torch.zeros(K, device="cuda")]
        self.norm_grad = [torch.empty(K, device="cuda"), torch.empty(K, device="cuda")]
        self.p, self.number = dropout, number

    def forward(self, h: torch.Tensor, add, ids: torch.Tensor, seed: int):
        """(the stream, what this block adds to it): the last block's part of the stream is added where the norm reads it."""
        self.ids, self.seed = ids, seed
        x, total, self.mean, self.rstd = salr.layer_norm(h, *self.norm, residual=add)
        self.stream = h if add is None else total
        self.x = salr.dropout(x, self.p, seed, self.number)
        y = salr.linear(x, *self.weight, None, None)
        return self.stream, self.adapters.add(self.x, ids, y, out=y)

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """The gradient of the stream, dy the one of h + layer(norm(h)); those of the weights are left in their places."""
        dx = salr.linear_backward(None, dy, *self.weight, None, None, need_dadb=False)[0]
        dropped, _, _ = self.adapters.backward(dy, self.x, self.ids)
        dx = salr.dropout(dropped, self.p, self.seed, self.number, residual=dx)
        got, dw, db = salr.layer_norm_backward(dx, self.stream, self.norm[0], self.mean, self.rstd, dsum=dy, need_dw=True, need_db=True)
        self.norm_grad[0].copy_(dw)
        self.norm_grad[1].copy_(db)
        return got


class Model:
    def __init__(self, K: int, V: int, ranks, depth: int, dropout: float, gen: torch.Generator):
        self.blocks = [Block(K, ranks, dropout, i, gen) for i in range(depth)]
        self.embedding = torch.randn(64, K, device="cuda", generator=gen).to(torch.bfloat16)
        self.head = torch.empty(V, K, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0 / K ** 0.5, generator=gen)

    def step(self, tokens, targets, ids, seed: int) -> torch.Tensor:
        """Mean loss of the unmasked tokens; the gradients are left in their places."""
        h, add = self.embedding[tokens], None
        for block in self.blocks:
            h, add = block.forward(h, add, ids, seed)
        live = (targets >= 0).sum().float()
        loss, _, dh, _ = salr.linear_cross_entropy(h + add, self.head, targets, (1.0 / live).expand(len(targets)).contiguous())
        for block in reversed(self.blocks):
            dh = block.backward(dh)
        return loss.sum() / live


def train(steps: int = 60, T: int = 512, K: int = 512, V: int = 4099, tenants: int = 4, depth: int = 2, dropout: float = 0.05, lr: float = 3e-3,
          max_norm: float = 1.0, seed: int = 0, log=print) -> list[float]:
    gen = torch.Generator(device="cuda").manual_seed(seed)
    model = Model(K, V, [8 * (1 + i % 3) for i in range(tenants)], depth, dropout, gen)
    followers = torch.randint(0, V, (tenants, 64), device="cuda", generator=gen)   # what comes after each token, by tenant
    blocks = model.blocks
    adapters = salr.AdamW([p for b in blocks for p in b.master], [g for b in blocks for g in b.grad], copies=[c for b in blocks for c in b.copy])
    norms = salr.AdamW([p for b in blocks for p in b.norm], [g for b in blocks for g in b.norm_grad])
    losses = []
    for step in range(1, steps + 1):
        ids = torch.sort(torch.randint(0, tenants, (T,), device="cuda", generator=gen, dtype=torch.int32)).values
        tokens = torch.randint(0, 64, (T,), device="cuda", generator=gen)
        targets = followers[ids.long(), tokens]
        targets[: T // 8] = -100   # a prompt: not trained on
        losses.append(model.step(tokens, targets, ids, step))
        scale = adapters.grad_norm(max_norm)[1:]
        adapters.step(lr=lr, step=step, weight_decay=0.01, grad_scale=scale)
        norms.step(lr=lr, step=step, grad_scale=scale)
        if log and (step == 1 or step % 10 == 0):
            log(f"step {step:4d}  loss {float(losses[-1]):.4f}")
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--tenants", type=int, default=4)
    args = ap.parse_args()
    train(args.steps, T=args.tokens, tenants=args.tenants)
