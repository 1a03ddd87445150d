"""The operators of a fine-tuning step around the SALR layers, as cases that can be timed and compared.

A case is one pass through one of three operators:

    ce     ``linear_cross_entropy``   softmax cross entropy of a language-model head without keeping its logits, per token:
                                      the loss alone (scoring, evaluation), with the gradient of the hidden states (a frozen
                                      head), or with the head's gradient too
    adamw  ``AdamW.step``             an optimiser step over many tensors at once, states in 32 or in 8 bits
    norm   ``AdamW.grad_norm``        the norm of all gradients and the factor that clips them

With ``own`` false ``run`` computes them in plain torch, in 32 bits, rounded once at the end; with ``own`` true it calls the
framework's kernels.  Hidden states ~ N(0, 1) with a part of the target's row of the head added, so that some tokens are
predicted well and some are not, as in fine-tuning; the head ~ N(0, 0.02); a share of the tokens is masked (a prompt's).
Optimiser tensors lie one behind the other, each from a multiple of 128 elements on, as a training program's flat buffers do.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128            # elements that share the two scales of 8-bit states
FP8_MOST = 448.0       # largest value of the 8-bit type
TINY = 2.0 ** -100     # a block whose largest magnitude is below this is stored as zeros


def _ce(name, T, K, V, dh, dw):
    return {"name": name, "op": "ce", "T": T, "K": K, "V": V, "dh": dh, "dw": dw}


def _opt(name, op, tensors, K, N, R, bits, master, grad32, clip):
    return {"name": name, "op": op, "tensors": tensors, "K": K, "N": N, "R": R, "bits": bits, "master": master, "grad32": grad32, "clip": clip}


def listed():
    return [
        # log-probability of one token (scoring while decoding): the head is read once
        _ce("score_T1", 1, 4096, 131072, False, False),
        # a few candidate tokens on a wide model with a smaller vocabulary
        _ce("score_T24", 24, 8192, 32000, False, False),
        # perplexity of a validation batch: loss alone
        _ce("eval_T2048", 2048, 4096, 131072, False, False),
        # the smallest model of the workload list, an odd vocabulary: what is left is the call itself
        _ce("train_tiny", 48, 512, 4099, True, False),
        # fine-tuning with a frozen head: loss and gradient of the hidden states
        _ce("train_T4096", 4096, 4096, 131072, True, False),
        # nothing a multiple of anything, the head trained as well
        _ce("train_head_ragged", 1111, 2720, 50003, True, True),
        # adapters of 32 decoder blocks (seven layers each, A and B), f32 master weights with the bf16 copies the layers read
        _opt("adamw32_adapters", "adamw", 448, 4096, 14336, 32, 32, True, False, True),
        # the same with states in 8 bits
        _opt("adamw8_adapters", "adamw", 448, 4096, 14336, 32, 8, True, False, True),
        # adapters of one tiny block: what is left is the call itself
        _opt("adamw32_tiny", "adamw", 14, 512, 512, 8, 32, True, False, False),
        # odd sizes, bf16 weights without a master copy, f32 gradients
        _opt("adamw8_ragged", "adamw", 97, 2721, 5003, 13, 8, False, True, False),
        # clipping: the norm of all adapters' gradients, and of a tiny block's in f32
        _opt("norm_adapters", "norm", 448, 4096, 14336, 32, 32, True, False, True),
        _opt("norm_tiny", "norm", 14, 509, 517, 7, 32, True, True, True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# The sizes the listed cases stand for: 1 to 4096 tokens, hidden sizes 512 to 8192, vocabularies of 4096 to 131072; 2 to 448
# tensors of adapters of rank 4 to 64 on layers of 512 to 14336.
_MOST_PRODUCT = 4096 * 4096 * 131072
_MOST_ELEMENTS = 224 * 32 * (4096 + 14336)


def draw(rng):
    kind = rng.choice(["score", "eval", "train", "train", "head", "adamw", "adamw", "adamw", "norm"])
    if kind in ("adamw", "norm"):
        while True:
            tensors, R = _log_uniform(rng, 2, 448), _log_uniform(rng, 4, 64)
            K, N = _log_uniform(rng, 512, 14336), _log_uniform(rng, 512, 14336)
            if rng.random() < 0.5:
                K, N, R = K // 32 * 32, N // 32 * 32, max(4, R // 4 * 4)
            if tensors * R * (K + N) // 2 <= _MOST_ELEMENTS and 3072 not in (K, N):
                break
        return {"op": kind, "tensors": tensors, "K": K, "N": N, "R": R, "bits": rng.choice([8, 32]), "master": rng.random() < 0.6,
                "grad32": rng.random() < 0.3, "clip": rng.random() < 0.5}
    while True:
        K = max(512, _log_uniform(rng, 512, 8192) // 8 * 8)
        if rng.random() < 0.6:
            K = K // 128 * 128
        V = _log_uniform(rng, 4096, 131072)
        if rng.random() < 0.4:
            V = V // 128 * 128
        T = _log_uniform(rng, 1, 64) if kind == "score" else _log_uniform(rng, 32, 4096)
        products = {"score": 1, "eval": 1, "train": 2, "head": 3}[kind]
        if T * K * V * products <= _MOST_PRODUCT and 3072 not in (T, K, V):
            break
    return {"op": "ce", "T": T, "K": K, "V": V, "dh": kind in ("train", "head"), "dw": kind == "head"}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _counts(case):
    """Elements of the tensors: A [K, R] and B [R, N] in turn."""
    return [(case["K"] if i % 2 == 0 else case["N"]) * case["R"] for i in range(case["tensors"])]


def _ce_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, K, V = case["T"], case["K"], case["V"]
    w = torch.empty(V, K, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02, generator=gen)
    targets = torch.randint(0, V, (T,), device="cuda", generator=gen)
    # a row of the head has the squared length 4e-4 K: `sure` is how far the target's logit is lifted, 0 to 16
    sure = torch.rand(T, 1, device="cuda", generator=gen) * 16.0
    h = torch.randn(T, K, device="cuda", generator=gen)
    h = (h + w[targets].float() * (sure / (4e-4 * K))).to(torch.bfloat16)
    if T > 1:
        targets[torch.rand(T, device="cuda", generator=gen) < 0.2] = -100
    # the mean over the tokens that count
    grad_loss = torch.full((T,), 1.0 / max(1, int((targets >= 0).sum())), device="cuda")
    return {"h": h, "w": w, "targets": targets, "grad_loss": grad_loss}


def _opt_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    counts = _counts(case)
    starts, total = [], 0
    for n in counts:
        starts.append(total)
        total += (n + BLOCK - 1) // BLOCK * BLOCK
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for s, n in zip(starts, counts):
        inside[s:s + n] = True

    def normal(std):
        return torch.empty(total, device="cuda").normal_(0.0, std, generator=gen).mul_(inside)

    s = {"starts": starts, "counts": counts}
    # gradients of an adapter's elements differ by orders of magnitude; the averages go with them
    size = torch.exp2(-14.0 * torch.rand(total, device="cuda", generator=gen) ** 4)
    s["grad"] = (normal(1e-3) * size).to(torch.float32 if case["grad32"] else torch.bfloat16)
    if case["op"] == "norm":
        return s
    s["param"] = normal(0.02)
    if not case["master"]:
        s["param"] = s["param"].to(torch.bfloat16)
    s["copy"] = s["param"].to(torch.bfloat16) if case["master"] else None
    if case["bits"] == 32:
        s["exp_avg"] = normal(3e-4) * size
        s["exp_avg_sq"] = ((normal(4e-4).abs() + 6e-4 * inside) * size).square()
        s["scales"] = None
    else:
        s["exp_avg"] = (normal(60.0) * size).clamp_(-FP8_MOST, FP8_MOST).to(torch.float8_e4m3fn)
        s["exp_avg_sq"] = ((normal(80.0).abs() + 120.0) * size).clamp_(2.0 ** -9, FP8_MOST).mul_(inside).to(torch.float8_e4m3fn)
        s["scales"] = torch.empty(total // BLOCK, 2, device="cuda").uniform_(4e-6, 6e-6, generator=gen)
    s["grad_scale"] = torch.full((1,), 0.37, device="cuda") if case["clip"] else None
    # bf16 weights alone move only where a step is more than half of their last place
    s["hyper"] = {"lr": 2e-5 if case["master"] else 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01, "step": 20, "seed": seed & 0xFFFF}
    return s


def prepare(case, seed):
    if case["op"] == "ce":
        s = _ce_inputs(case, seed)
        s["workspace"] = None
    else:
        s = _opt_inputs(case, seed)
    s["case"] = dict(case)
    if own:   # what a training program keeps: the workspace of the loss, the optimiser with its list of tensors
        import paper_2601_16991_amd as salr
        if case["op"] == "ce":
            need = salr.salr_linear_cross_entropy_workspace_bytes(case["T"], case["K"], case["V"], case["dh"], case["dw"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        else:
            def views(t, per=1):
                return None if t is None else [t[a // per:a // per + (n + per - 1) // per] for a, n in zip(s["starts"], s["counts"])]
            if case["op"] == "norm":
                s["optimizer"] = salr.GradNorm(views(s["grad"]))
            else:
                s["optimizer"] = salr.AdamW(views(s["param"]), views(s["grad"]), views(s["exp_avg"]), views(s["exp_avg_sq"]),
                                            scales=views(s["scales"], BLOCK), copies=views(s["copy"]))
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms
def _plain_ce(h, w, targets, grad_loss, want_dh, want_dw):
    live = targets >= 0
    x = torch.where(live[:, None], h.float(), 0.0)   # a masked token's hidden state counts nowhere
    wf = w.float()
    logits = x @ wf.t()
    m = logits.max(dim=1, keepdim=True).values
    e = torch.exp(logits - m)
    total = e.sum(dim=1, keepdim=True)
    lse = m + torch.log(total)
    at = targets.clamp(min=0)[:, None]
    loss = torch.where(live, (lse - logits.gather(1, at))[:, 0], 0.0)
    out = {"loss": loss, "lse": torch.where(live, lse[:, 0], 0.0)}
    if want_dh or want_dw:
        del logits
        g = e.div_(total)
        g.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
        g.mul_(torch.where(live, grad_loss, 0.0)[:, None])
        if want_dh:
            out["dh"] = (g @ wf).to(torch.bfloat16)
        if want_dw:
            out["dw"] = (g.t() @ x).to(torch.bfloat16)
    return out


def _random20(total, seed):
    """Twenty bits for every position, from its number and the step's seed: 32-bit products and shifts."""
    x = torch.arange(total, dtype=torch.int64, device="cuda")
    x = (x * 0x9E3779B1 + seed * 0x85157AF5) & 0xFFFFFFFF
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 13)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x >> 12


def _plain_block_scale(t):
    most = t.abs().max(dim=1, keepdim=True).values
    fine = most >= TINY
    return torch.where(fine, FP8_MOST / most, 0.0), torch.where(fine, most / FP8_MOST, 0.0)


def _plain_random_round(x, bits):
    """x >= 0 to the 8-bit type, up with the probability of what is cut off; what is not zero stays so."""
    low = x < 2.0 ** -6   # subnormal there: 2^-6 on top gives such a value the same step
    t = torch.where(low, x + 2.0 ** -6, x)
    t = ((t.view(torch.int32) + bits.to(torch.int32)) & ~0xFFFFF).view(torch.float32)
    t = torch.where(low, t - 2.0 ** -6, t).clamp(max=FP8_MOST)
    return torch.where(x > 0, t.clamp(min=2.0 ** -9), 0.0)


def _plain_adamw(s):
    hy = s["hyper"]
    b1, b2, lr = hy["beta1"], hy["beta2"], hy["lr"]
    scale = s["grad_scale"]
    g = s["grad"].float()
    if scale is not None:
        g = g * scale
    if s["scales"] is None:
        m, v = s["exp_avg"], s["exp_avg_sq"]
    else:
        sc = s["scales"]
        m = (s["exp_avg"].float().view(-1, BLOCK) * sc[:, :1]).view(-1)
        v = (s["exp_avg_sq"].float().view(-1, BLOCK) * sc[:, 1:]).view(-1).square()
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    root = torch.sqrt(v)
    p = s["param"].float() * (1 - lr * hy["weight_decay"])
    denom = root * (1 / math.sqrt(1 - b2 ** hy["step"])) + hy["eps"]
    p = p - (m * (lr / (1 - b1 ** hy["step"]))) / denom
    s["param"].copy_(p)
    if s["copy"] is not None:
        s["copy"].copy_(p)
    if s["scales"] is None:
        s["exp_avg"].copy_(m)
        s["exp_avg_sq"].copy_(v)
    else:
        m, root = m.view(-1, BLOCK), root.view(-1, BLOCK)
        inv_m, scale_m = _plain_block_scale(m)
        inv_r, scale_r = _plain_block_scale(root)
        s["exp_avg"].copy_((m * inv_m).view(-1).to(torch.float8_e4m3fn))
        x = _plain_random_round((root * inv_r).view(-1), _random20(root.numel(), hy["seed"]))
        s["exp_avg_sq"].copy_(x.to(torch.float8_e4m3fn))
        s["scales"].copy_(torch.cat([scale_m, scale_r], dim=1))


def _plain_norm(grad):
    norm = torch.sqrt(grad.float().square().sum())
    return torch.stack([norm, torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)])


MAX_NORM = 1.0


def _opt_outputs(s):
    return {k: s[k] for k in ("param", "copy", "exp_avg", "exp_avg_sq", "scales") if s[k] is not None}


def run(s):
    case = s["case"]
    if case["op"] == "ce":
        if not own:
            return _plain_ce(s["h"], s["w"], s["targets"], s["grad_loss"], case["dh"], case["dw"])
        import paper_2601_16991_amd as salr
        got = salr.linear_cross_entropy(s["h"], s["w"], s["targets"], s["grad_loss"], need_dh=case["dh"], need_dw=case["dw"],
                                        workspace=s["workspace"])
        return {k: t for k, t in zip(("loss", "lse", "dh", "dw"), got) if t is not None}
    if case["op"] == "norm":
        return s["optimizer"](MAX_NORM) if own else _plain_norm(s["grad"])
    if own:
        s["optimizer"].step(grad_scale=s["grad_scale"], **s["hyper"])
    else:
        _plain_adamw(s)
    return _opt_outputs(s)


# ------------------------------------------------------------------------------------------------------------------ exact
def _exact_ce(case, s):
    h, w, t = s["h"].double(), s["w"].double(), s["targets"]
    T, V = case["T"], case["V"]
    loss, lse = (torch.zeros(T, dtype=torch.float64, device="cuda") for _ in range(2))
    rows = torch.nonzero(t >= 0)[:, 0]
    out = {"loss": loss, "lse": lse}
    if case["dh"]:
        out["dh"] = torch.zeros(T, case["K"], dtype=torch.float64, device="cuda")
    if case["dw"]:
        out["dw"] = torch.zeros(V, case["K"], dtype=torch.float64, device="cuda")
    for r in rows.split(1024):
        z = h[r] @ w.t()
        z_t = z[torch.arange(len(r), device="cuda"), t[r]].clone()
        lse[r] = torch.logsumexp(z, dim=1)
        loss[r] = lse[r] - z_t
        if case["dh"] or case["dw"]:
            prob = torch.softmax(z, dim=1)
            del z
            prob[torch.arange(len(r), device="cuda"), t[r]] -= 1.0
            prob *= s["grad_loss"][r].double()[:, None]
            if case["dh"]:
                out["dh"][r] = prob @ w
            if case["dw"]:
                out["dw"] += prob.t() @ h[r]
    return out


def _exact_adamw(s):
    hy = s["hyper"]
    b1, b2 = hy["beta1"], hy["beta2"]
    grad = s["grad"].double() * (s["grad_scale"].double() if s["grad_scale"] is not None else 1.0)
    eight = s["scales"] is not None
    per = s["scales"].double().repeat_interleave(BLOCK, dim=0) if eight else None
    m0 = s["exp_avg"].to(torch.float32).double() * (per[:, 0] if eight else 1.0)
    v0 = s["exp_avg_sq"].to(torch.float32).double()
    v0 = (v0 * per[:, 1]) ** 2 if eight else v0
    m, v = b1 * m0 + (1 - b1) * grad, b2 * v0 + (1 - b2) * grad ** 2
    m_hat, v_hat = m / (1 - b1 ** hy["step"]), v / (1 - b2 ** hy["step"])
    p = s["param"].double()
    p = p - hy["lr"] * hy["weight_decay"] * p - hy["lr"] * m_hat / (v_hat.sqrt() + hy["eps"])
    out = {"param": p, "exp_avg": m, "exp_avg_sq": v}
    if s["copy"] is not None:
        out["copy"] = p
    if eight:
        scales = []
        for name, t in (("exp_avg", m), ("exp_avg_sq", v.sqrt())):
            top = t.abs().view(-1, BLOCK).amax(dim=1)
            scales.append(top / FP8_MOST)
            x = (t.view(-1, BLOCK) / torch.where(top > 0, top, 1.0)[:, None] * FP8_MOST).view(-1)
            # spacing of the 8-bit values around x: 2^(e - 3), e the exponent and at least -6
            step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
            if name == "exp_avg":
                out[name] = torch.round(x / step) * step
            else:
                y = torch.floor(x / step + _random20(x.numel(), hy["seed"]).double() / 2 ** 20) * step
                out[name] = torch.where(x > 0, y.clamp(2.0 ** -9, FP8_MOST), 0.0)
        out["scales"] = torch.stack(scales, dim=1)
    return out


def exact(case, seed):
    """What ``run`` returns, in 64 bits."""
    if case["op"] == "ce":
        return _exact_ce(case, _ce_inputs(case, seed))
    s = _opt_inputs(case, seed)
    if case["op"] == "norm":
        norm = torch.linalg.vector_norm(s["grad"].double())
        return torch.stack([norm, torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)])
    return _exact_adamw(s)


def work(case):
    """Each input once in, each output once out; the products as many as the results asked for."""
    if case["op"] == "ce":
        T, K, V, dh, dw = case["T"], case["K"], case["V"], case["dh"], case["dw"]
        return {"bytes": 2 * K * (T + V) + 20 * T + 2 * K * (T * dh + V * dw), "flops": 2 * T * K * V * (1 + dh + dw)}
    n = sum(_counts(case))
    grad = 4 if case["grad32"] else 2
    if case["op"] == "norm":
        return {"bytes": n * grad, "flops": 2 * n}
    param = 10 if case["master"] else 4
    state = 16 if case["bits"] == 32 else 4
    return {"bytes": n * (grad + param + state) + (0 if case["bits"] == 32 else n // BLOCK * 16), "flops": 16 * n}
