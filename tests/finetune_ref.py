"""Plain 64-bit implementations of the fine-tuning operators, on the CPU, for the tests."""
import math

import torch


def cross_entropy(h, w, targets, grad_loss):
    """(loss, lse, dh, dw, G) in float64; h's masked rows count as zeros."""
    live = targets >= 0
    x = torch.where(live[:, None], h.double(), torch.zeros((), dtype=torch.float64))
    wd = w.double()
    z = x @ wd.t()
    at = targets.clamp(min=0)[:, None]
    lse = torch.logsumexp(z, 1)
    # lse - z_target as log(1 + the others' sum over e^z_target): to full precision where the target is nearly certain
    rest = torch.logsumexp(z.scatter(1, at, -math.inf), 1) - z.gather(1, at)[:, 0]
    loss = torch.logaddexp(torch.zeros_like(rest), rest)
    loss = torch.where(rest < -30, torch.exp(rest), loss)
    G = torch.softmax(z, 1)
    # 1 - p of the target as the sum of the others
    others = G.scatter(1, at, torch.zeros_like(at, dtype=torch.float64)).sum(1)
    G = G.scatter(1, at, -others[:, None])
    G = G * torch.where(live, grad_loss.double(), 0.0)[:, None]
    zero = torch.zeros((), dtype=torch.float64)
    return torch.where(live, loss, zero), torch.where(live, lse, zero), G @ wd, G.t() @ x, G


def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step, c=1.0):
    """float64; v is the square."""
    g = g.double() * c
    m = beta1 * m.double() + (1 - beta1) * g
    v = beta2 * v.double() + (1 - beta2) * g * g
    p = p.double()
    p = p - lr * weight_decay * p - lr * (m / (1 - beta1 ** step)) / ((v / (1 - beta2 ** step)).sqrt() + eps)
    return p, m, v


def fp8_spacing(x):
    """Distance between neighbouring 8-bit values around |x| (4 exponent, 3 mantissa bits, bias 7)."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)


def random20(position, seed):
    x = (position.to(torch.int64) * 0x9E3779B1 + seed * 0x85157AF5) & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x6A09E667) & 0xFFFFFFFF
    x = ((x ^ (x >> 13)) * 0xBB67AE85) & 0xFFFFFFFF
    return x >> 12


def blocks_max(x, block=128):
    n = x.numel()
    pad = torch.zeros((n + block - 1) // block * block, dtype=x.dtype)
    pad[:n] = x
    return pad.view(-1, block).abs().amax(1)


def per_element(scale, n, block=128):
    return scale.repeat_interleave(block)[:n]


def close(a, b):
    return math.isclose(a, b, rel_tol=1e-6)
