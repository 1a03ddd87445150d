"""The operators on either side of a SALR layer, as cases that can be timed and compared.

A case is one pass through one of these:

    drop        ``dropout``                 y = keep ? x / (1 - p) : 0, plus a residual; the mask comes from a counter and is not stored (the backward
                                            pass is the same call on the gradient)
    norm        ``layer_norm``              layer norm of x, or of x + residual, which it then gives back too
    norm_grad   ``layer_norm_backward``     its gradient, of the input and of weight and bias
    serve       ``AdapterSet.add``          y = base + (x A_i) B_i where every token names its adapter i, or none: many requests beside one shared layer
    adapt_grad  ``AdapterSet.backward``     its gradient, of the input and of every adapter

With ``own`` false ``run`` computes them in plain torch, in 32 bits, rounded once at the end (the sum that ``layer_norm`` gives back is rounded
where it is defined to be: the norm is that of the stored sum); with ``own`` true it calls the framework's kernels.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
RANKS = (8, 16, 13, 32, 4, 64, 16, 24)   # of a set of adapters of several ranks, in turn, as far as they are no larger than the case's R


def _drop(name, T, K, f32, residual, p):
    return {"name": name, "op": "drop", "T": T, "K": K, "f32": f32, "residual": residual, "p": p}


def _norm(name, T, K, f32, w32, residual, bias):
    return {"name": name, "op": "norm", "T": T, "K": K, "f32": f32, "w32": w32, "residual": residual, "bias": bias}


def _norm_grad(name, T, K, f32, w32, residual, weights):
    return {"name": name, "op": "norm_grad", "T": T, "K": K, "f32": f32, "w32": w32, "residual": residual, "weights": weights}


def _adapters(name, op, T, K, N, R, mixed, loaded, used, prompts, bare):
    return {"name": name, "op": op, "T": T, "K": K, "N": N, "R": R, "mixed": mixed, "loaded": loaded, "used": used, "prompts": prompts, "bare": bare}


def listed():
    return [
        # in front of the adapters of the smallest layer of the workload list: what is left is the call itself
        _drop("drop_tiny", 48, 512, False, False, 0.1),
        # behind a layer, onto the residual stream, in a training step of 4096 tokens
        _drop("drop_residual_T4096", 4096, 4096, False, True, 0.1),
        # fp32 activations of odd sizes
        _drop("drop_f32_ragged", 1111, 2721, True, False, 0.35),
        # one token being decoded: the residual stream takes in a layer's output and is normalised
        _norm("norm_T1", 1, 4096, False, False, True, True),
        # the same for a training step or a prompt
        _norm("norm_T4096", 4096, 4096, False, False, True, True),
        # the backward pass of that, weights in fp32 and trained too
        _norm_grad("norm_grad_T4096", 4096, 4096, False, True, True, True),
        # fp32, odd sizes
        _norm_grad("norm_grad_ragged", 1111, 2721, True, True, False, True),
        # one request being decoded, 64 adapters loaded
        _adapters("serve_T1", "serve", 1, 4096, 4096, 16, False, 64, 1, False, False),
        # a full decoding batch: 64 requests of 40 tenants, adapters of several ranks, up projection
        _adapters("serve_T64", "serve", 64, 4096, 14336, 64, True, 64, 40, False, True),
        # prompts of seven requests, one after the other, one of them without an adapter; nothing a multiple of anything
        _adapters("prompt_T2001", "serve", 2001, 2720, 2731, 16, False, 64, 6, True, True),
        # adapters of eight tenants trained in one batch
        _adapters("adapt_grad_T4096", "adapt_grad", 4096, 4096, 14336, 32, False, 8, 8, True, False),
        # adapters of several ranks, some without a token in this batch, short sequences
        _adapters("adapt_grad_ragged", "adapt_grad", 777, 2720, 2744, 64, True, 16, 13, True, True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# The sizes the listed cases stand for: 1 to 4096 tokens, layers of 512 to 14336 features, adapters of rank 4 to 64 (and 128 in sets of few),
# 1 to 64 of them loaded.
def draw(rng):
    op = rng.choice(["drop", "norm", "norm_grad", "serve", "serve", "adapt_grad"])
    while True:
        T, K = _log_uniform(rng, 1, 4096), _log_uniform(rng, 512, 14336)
        if op in ("drop", "norm", "norm_grad"):
            if rng.random() < 0.6:
                K = K // 32 * 32
            f32 = rng.random() < 0.3
            if T * K * (2 if f32 else 1) > 4096 * 4096:
                continue
            if op == "drop":
                return {"op": op, "T": T, "K": K, "f32": f32, "residual": rng.random() < 0.5, "p": rng.choice([0.01, 0.05, 0.1, 0.2, 0.5])}
            case = {"op": op, "T": T, "K": K, "f32": f32, "w32": f32 or rng.random() < 0.5, "residual": rng.random() < 0.6}
            case["bias" if op == "norm" else "weights"] = rng.random() < 0.6
            return case
        K, N = K // 32 * 32, _log_uniform(rng, 512, 14336)
        if op == "adapt_grad" or rng.random() < 0.6:
            N = N // 8 * 8
        if K * N > 4096 * 14336:
            continue
        loaded = _log_uniform(rng, 1, 64)
        prompts = op == "adapt_grad" or rng.random() < 0.4
        used = min(loaded, T, _log_uniform(rng, 1, 64))
        R = rng.choice([4, 8, 16, 32, 64] + ([128] if loaded <= 4 and op == "serve" else []))
        if op == "adapt_grad" and (loaded * R > 512 or T * R > 4096 * 32):
            continue
        return {"op": op, "T": T, "K": K, "N": N, "R": R, "mixed": rng.random() < 0.4, "loaded": loaded, "used": used, "prompts": prompts,
                "bare": T > used and rng.random() < 0.5}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _ranks(case):
    """Ranks of the loaded adapters."""
    cycle = [r for r in RANKS if r <= case["R"]] if case["mixed"] else [case["R"]]
    return [cycle[i % len(cycle)] for i in range(case["loaded"])]


def _used(case):
    """The adapters that tokens of the batch name."""
    return [j * case["loaded"] // case["used"] for j in range(case["used"])]


def _bare(case):
    """Tokens without an adapter."""
    return min(max(1, case["T"] // 8), case["T"] - case["used"]) if case["bare"] else 0


def _type(f32):
    return torch.float32 if f32 else torch.bfloat16


def _activations(gen, T, K, dtype):
    """Rows of different size, a few features far larger than the rest, as a transformer's residual stream has them."""
    x = torch.randn(T, K, device="cuda", generator=gen)
    x *= torch.exp(0.5 * torch.randn(T, 1, device="cuda", generator=gen))
    x[:, :: 501] *= 12.0
    return x.to(dtype)


def _adapter_inputs(case, seed, gen):
    T, K, N = case["T"], case["K"], case["N"]
    used, bare = _used(case), _bare(case)
    host = torch.Generator().manual_seed(seed)
    # every adapter in use has a token at least, the other tokens go to the popular ones first
    weight = 1.0 / torch.arange(1, len(used) + 1, dtype=torch.float64)
    more = T - bare - len(used)
    picks = list(range(len(used))) + (torch.multinomial(weight, more, replacement=True, generator=host).tolist() if more else [])
    ids = [used[j] for j in picks] + [-1] * bare
    if case["prompts"]:   # one request behind the other
        order = {i: int(at) for i, at in zip(used + [-1], torch.randperm(len(used) + 1, generator=host))}
        ids.sort(key=lambda i: order[i])
    else:
        ids = [ids[j] for j in torch.randperm(T, generator=host).tolist()]
    ids = torch.tensor(ids, dtype=torch.int32)
    s = {"rows": [(i, torch.nonzero(ids == i)[:, 0].cuda()) for i in used], "ids": ids.cuda()}
    s["x"] = torch.randn(T, K, device="cuda", generator=gen).to(torch.bfloat16)
    s["A"] = [(torch.randn(K, r, device="cuda", generator=gen) / math.sqrt(K)).to(torch.bfloat16) for r in _ranks(case)]
    s["B"] = [(torch.randn(r, N, device="cuda", generator=gen) * (0.5 / math.sqrt(r))).to(torch.bfloat16) for r in _ranks(case)]
    if case["op"] == "serve":
        s["base"] = torch.randn(T, N, device="cuda", generator=gen).to(torch.bfloat16)
    else:
        s["dy"] = (torch.randn(T, N, device="cuda", generator=gen) * 1e-3).to(torch.bfloat16)
        s["dx_base"] = (torch.randn(T, K, device="cuda", generator=gen) * 1e-3).to(torch.bfloat16)
    return s


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    if op in ("serve", "adapt_grad"):
        return _adapter_inputs(case, seed, gen)
    T, K, dtype = case["T"], case["K"], _type(case["f32"])
    s = {"x": _activations(gen, T, K, dtype)}
    if op == "drop":
        s["residual"] = _activations(gen, T, K, dtype) if case["residual"] else None
        s["seed"], s["offset"] = 0x5DEECE66D * (seed + 1) & 0x7FFFFFFFFFFFFFFF, seed % 1000
        return s
    s["weight"] = (1.0 + 0.2 * torch.randn(K, device="cuda", generator=gen)).to(_type(case["w32"]))
    if op == "norm":
        s["bias"] = (0.1 * torch.randn(K, device="cuda", generator=gen)).to(_type(case["w32"])) if case["bias"] else None
        s["residual"] = _activations(gen, T, K, dtype) if case["residual"] else None
        return s
    xd = s["x"].double()   # what the forward pass kept
    s["mean"] = xd.mean(dim=1).float()
    s["rstd"] = (1.0 / torch.sqrt(xd.var(dim=1, unbiased=False) + EPS)).float()
    s["dy"] = (torch.randn(T, K, device="cuda", generator=gen) * 1e-3).to(dtype)
    s["dsum"] = (torch.randn(T, K, device="cuda", generator=gen) * 1e-3).to(dtype) if case["residual"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if own:   # what a program keeps: the set of adapters with the place of their gradients, the workspaces
        import paper_2601_16991_amd as salr
        op = case["op"]
        if op in ("serve", "adapt_grad"):
            train = op == "adapt_grad"
            s["set"] = salr.AdapterSet(s["A"], s["B"], *([[torch.empty_like(t) for t in s[k]] for k in "AB"] if train else []))
            need = s["set"].backward_workspace_bytes(case["T"]) if train else s["set"].workspace_bytes(case["T"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        elif op == "norm_grad":
            need = salr.salr_layer_norm_backward_workspace_bytes(case["T"], case["K"], case["weights"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------------ plain forms
_LOW = 0xFFFFFFFF


def _plain_sixteen_bits(count, seed, offset):
    """16 random bits for every position: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, 2011) of the counter (position / 8, offset) with the
    seed as key; a block's four words hold its eight positions' bits, the lower half of a word first."""
    block = torch.arange((count + 7) // 8, dtype=torch.int64, device="cuda")
    c0, c1 = block & _LOW, block >> 32
    c2, c3 = torch.full_like(block, offset & _LOW), torch.full_like(block, (offset >> 32) & _LOW)
    k0, k1 = seed & _LOW, (seed >> 32) & _LOW
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57   # 64-bit products that wrap into the sign: the shifts below are masked
        c0, c1, c2, c3 = ((p1 >> 32) & _LOW) ^ c1 ^ k0, p1 & _LOW, ((p0 >> 32) & _LOW) ^ c3 ^ k1, p0 & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    words = torch.stack([c0, c1, c2, c3], dim=1)
    return torch.stack([words & 0xFFFF, words >> 16], dim=2).view(-1)[:count]


def _plain_drop(s):
    x = s["x"]
    cut = int(s["case"]["p"] * 65536 + 0.5)   # of 65536: the probability is taken in steps of 2^-16
    keep = _plain_sixteen_bits(x.numel(), s["seed"], s["offset"]).view_as(x) >= cut
    y = torch.where(keep, x.float() * (65536.0 / (65536 - cut)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


def _plain_norm(s):
    x = s["x"]
    total = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    z = total.float()
    mean = z.mean(dim=1, keepdim=True)
    z = z - mean
    rstd = torch.rsqrt((z * z).mean(dim=1, keepdim=True) + EPS)
    y = z * rstd * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    out = {"y": y.to(x.dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if s["residual"] is not None:
        out["sum"] = total
    return out


def _plain_norm_grad(s):
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    xhat = (x - s["mean"][:, None]) * rstd
    g = dy * s["weight"].float()
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    out = {"dx": dx.to(s["x"].dtype)}
    if s["case"]["weights"]:
        out["dw"] = (dy * xhat).sum(dim=0).to(s["weight"].dtype)
        out["db"] = dy.sum(dim=0).to(s["weight"].dtype)
    return out


def _plain_serve(s):
    y = s["base"].float()
    for i, rows in s["rows"]:
        y[rows] += (s["x"][rows].float() @ s["A"][i].float()) @ s["B"][i].float()
    return y.to(torch.bfloat16)


def _plain_adapt_grad(s):
    dx = s["dx_base"].float()
    da, db = [torch.zeros_like(t) for t in s["A"]], [torch.zeros_like(t) for t in s["B"]]
    for i, rows in s["rows"]:
        x, dy, a, b = s["x"][rows].float(), s["dy"][rows].float(), s["A"][i].float(), s["B"][i].float()
        dt = dy @ b.t()
        dx[rows] += dt @ a.t()
        da[i] = (x.t() @ dt).to(torch.bfloat16)
        db[i] = ((x @ a).t() @ dy).to(torch.bfloat16)
    return {"dx": dx.to(torch.bfloat16), "da": da, "db": db}


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"drop": _plain_drop, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "serve": _plain_serve, "adapt_grad": _plain_adapt_grad}[op](s)
    import paper_2601_16991_amd as salr
    if op == "drop":
        return salr.dropout(s["x"], s["case"]["p"], s["seed"], s["offset"], residual=s["residual"])
    if op == "norm":
        y, total, mean, rstd = salr.layer_norm(s["x"], s["weight"], s["bias"], EPS, residual=s["residual"])
        out = {"y": y, "mean": mean, "rstd": rstd}
        if s["residual"] is not None:
            out["sum"] = total
        return out
    if op == "norm_grad":
        got = salr.layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], dsum=s["dsum"], need_dw=s["case"]["weights"],
                                       need_db=s["case"]["weights"], workspace=s["workspace"])
        return {k: t for k, t in zip(("dx", "dw", "db"), got) if t is not None}
    if op == "serve":
        return s["set"].add(s["x"], s["ids"], s["base"], workspace=s["workspace"])
    dx, da, db = s["set"].backward(s["dy"], s["x"], s["ids"], dx_base=s["dx_base"], workspace=s["workspace"])
    return {"dx": dx, "da": da, "db": db}


# ------------------------------------------------------------------------------------------------------------------ exact
def _times(a, m):
    """The upper and lower 32 bits of a * m, a an int64 tensor of 32-bit values, by halves of m: no product leaves 48 bits."""
    low, high = a * (m & 0xFFFF), a * (m >> 16)
    middle = (low >> 16) + high
    return middle >> 16, ((middle & 0xFFFF) << 16) | (low & 0xFFFF)


def _exact_drop(case, s):
    x = s["x"]
    n = x.numel()
    w = [torch.arange(-(-n // 8), device="cuda"), None, None, None]
    w[1], w[0] = w[0].div(2 ** 32, rounding_mode="floor"), w[0].remainder(2 ** 32)
    w[2], w[3] = (torch.zeros_like(w[0]) + part for part in (s["offset"] % 2 ** 32, s["offset"] // 2 ** 32))
    for r in range(10):
        key = [(s["seed"] + r * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32]
        (h0, l0), (h1, l1) = _times(w[0], 0xD2511F53), _times(w[2], 0xCD9E8D57)
        w = [torch.bitwise_xor(torch.bitwise_xor(h1, w[1]), torch.full_like(h1, key[0])), l1,
             torch.bitwise_xor(torch.bitwise_xor(h0, w[3]), torch.full_like(h0, key[1])), l0]
    at = torch.arange(n, device="cuda")
    cut = math.floor(case["p"] * 65536 + 0.5)
    y = torch.zeros(n, dtype=torch.float64, device="cuda")
    flat = x.reshape(-1).double() * (65536 / (65536 - cut))
    for j in range(4):
        bits = w[j][at[2 * j::8].div(8, rounding_mode="floor")]
        y[2 * j::8] = torch.where(bits.remainder(65536) >= cut, flat[2 * j::8], 0.0)
        bits = w[j][at[2 * j + 1::8].div(8, rounding_mode="floor")]
        y[2 * j + 1::8] = torch.where(bits.div(65536, rounding_mode="floor") >= cut, flat[2 * j + 1::8], 0.0)
    y = y.view_as(x)
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_norm(s):
    total = s["x"].double()
    if s["residual"] is not None:
        total = total + s["residual"].double()
    stored = total.to(s["x"].dtype).double()   # the norm is that of the sum as it is kept
    var, mean = torch.var_mean(stored, dim=1, correction=0)
    rstd = (var + EPS) ** -0.5
    y = (stored * rstd[:, None] - (mean * rstd)[:, None]) * s["weight"].double()
    if s["bias"] is not None:
        y = y + s["bias"].double()
    out = {"y": y, "mean": mean, "rstd": rstd}
    if s["residual"] is not None:
        out["sum"] = total
    return out


def _exact_norm_grad(case, s):
    x, dy, w, K = s["x"].double(), s["dy"].double(), s["weight"].double(), case["K"]
    mean, rstd = s["mean"].double(), s["rstd"].double()
    xhat = (x - mean[:, None]) * rstd[:, None]
    along, aligned = dy @ w / K, torch.sum(dy * xhat * w, dim=1) / K
    dx = (dy * w - along[:, None] - xhat * aligned[:, None]) * rstd[:, None]
    out = {"dx": dx if s["dsum"] is None else dx + s["dsum"].double()}
    if case["weights"]:
        out["dw"] = torch.sum(dy * xhat, dim=0)
        out["db"] = torch.ones(case["T"], dtype=torch.float64, device="cuda") @ dy
    return out


def _exact_serve(s):
    y = s["base"].double()
    for i, rows in s["rows"]:
        y.index_add_(0, rows, s["x"][rows].double() @ s["A"][i].double() @ s["B"][i].double())
    return y


def _exact_adapt_grad(s):
    dx = s["dx_base"].double()
    da, db = ([torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in s[k]] for k in "AB")
    for i, rows in s["rows"]:
        x, dy, a, b = s["x"][rows].double(), s["dy"][rows].double(), s["A"][i].double(), s["B"][i].double()
        at_t = (b @ dy.t()).t().contiguous()
        dx.index_add_(0, rows, at_t @ a.t().contiguous())
        da[i] = x.t().contiguous() @ at_t
        db[i] = a.t().contiguous() @ x.t().contiguous() @ dy
    return {"dx": dx, "da": da, "db": db}


def exact(case, seed):
    """What ``run`` returns, in 64 bits."""
    s = _inputs(case, seed)
    op = case["op"]
    if op == "drop":
        return _exact_drop(case, s)
    if op == "norm":
        return _exact_norm(s)
    if op == "norm_grad":
        return _exact_norm_grad(case, s)
    return _exact_serve(s) if op == "serve" else _exact_adapt_grad(s)


def work(case):
    """Each input once in, each output once out; adapters in use alone, but the gradients of all."""
    op, T, K = case["op"], case["T"], case["K"]
    if op in ("drop", "norm", "norm_grad"):
        size = 4 if case["f32"] else 2
        if op == "drop":
            return {"bytes": T * K * size * (3 if case["residual"] else 2), "flops": T * K * (2 if case["residual"] else 1)}
        w = 4 if case["w32"] else 2
        if op == "norm":
            return {"bytes": T * K * size * (4 if case["residual"] else 2) + K * w * (1 + case["bias"]) + 8 * T, "flops": 8 * T * K}
        return {"bytes": T * K * size * (4 if case["residual"] else 3) + K * w * (1 + 2 * case["weights"]) + 8 * T, "flops": 14 * T * K}
    N, used, ranks = case["N"], _used(case), _ranks(case)
    rank = sum(ranks[i] for i in used)
    live = T - _bare(case)
    if op == "serve":
        return {"bytes": 2 * K * live + 4 * T * N + 2 * rank * (K + N) + 4 * T, "flops": 2 * live * rank // len(used) * (K + N)}
    return {"bytes": 2 * live * (K + N) + 4 * T * K + 2 * rank * (K + N) + 2 * sum(ranks) * (K + N) + 4 * T,
            "flops": 2 * live * rank // len(used) * (3 * K + 2 * N)}
