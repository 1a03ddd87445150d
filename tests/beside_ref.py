"""Plain 64-bit implementations of the operators beside a layer, on the CPU, for the tests."""
import numpy as np
import torch

U = 2.0 ** -24
HALVES = 2.0 ** -16   # 2^-8 of 2^-8, of a value held as two bf16


def half(dtype):
    """Most that rounding to the type is off by, relative to the value."""
    return torch.finfo(dtype).eps / 2


def philox(counter, key):
    """Philox4x32-10: counter four 32-bit words (Python numbers or uint64 arrays), key two."""
    c, k = [np.asarray(x, dtype=np.uint64) for x in counter], [int(x) for x in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(count, p, seed, offset):
    block = np.arange((count + 7) // 8, dtype=np.uint64)
    seed, offset = seed & (2 ** 64 - 1), offset & (2 ** 64 - 1)
    full = lambda x: np.full_like(block, x)   # noqa: E731
    words = philox([block & np.uint64(0xFFFFFFFF), block >> np.uint64(32), full(offset & 0xFFFFFFFF), full(offset >> 32)], [seed & 0xFFFFFFFF, seed >> 32])
    bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1).reshape(-1)[:count]
    return torch.from_numpy((bits >= int(p * 65536 + 0.5)).copy())


def dropout(x, p, seed, offset, residual=None):
    """(y in 64 bits, how far fp32 arithmetic may be from it before the last rounding)."""
    cut = int(p * 65536 + 0.5)
    keep = keep_mask(x.numel(), p, seed, offset).view(x.shape)
    y = torch.where(keep, x.double() * (65536 / (65536 - cut)), 0.0)
    r = 0.0 if residual is None else residual.double()
    # the factor, the product and the sum are rounded once each
    return y + r, 2 * U * y.abs() + U * (y + r).abs()


def layer_norm(s, weight, bias, eps):
    """(y, mean, rstd) of s as it is, and their tolerances.  A sum over a row goes through at most 32 additions in a lane, 6 over the wave's lanes and 16
    over the team: 54 roundings.  A mean that is off by d moves the variance by d^2 (differences to the exact mean cancel)."""
    z, w = s.double(), weight.double()
    mean = z.mean(1, keepdim=True)
    d = z - mean
    rstd = (d.square().mean(1, keepdim=True) + eps).rsqrt()
    y = d * rstd * w + (0.0 if bias is None else bias.double())
    off = 56 * U * z.abs().mean(1, keepdim=True)
    rel = 64 * U + (off * rstd).square()      # of rstd: half of the variance's 56 U, its division, root and quotient
    b = torch.zeros(()) if bias is None else bias.double()
    tol_y = w.abs() * ((d * rstd).abs() * (rel + 4 * U) + off * rstd) + 2 * U * (y.abs() + b.abs())
    return (y, mean[:, 0], rstd[:, 0]), (tol_y, off[:, 0] + U * mean[:, 0].abs(), (rel * rstd)[:, 0])


def layer_norm_backward(dy, x, weight, mean, rstd, dsum):
    """(dx, dw, db) and their tolerances: xhat is off by two roundings, g by one, a row's sums by 54 more and their products; a column's sum by as many
    as it has rows, and 50 for what is joined."""
    K, T = x.shape[1], x.shape[0]
    d, xd, w = dy.double(), x.double(), weight.double()
    r = rstd.double()[:, None]
    xhat = (xd - mean.double()[:, None]) * r
    g = d * w
    gm, along = g.sum(1, keepdim=True) / K, (g * xhat).sum(1, keepdim=True) / K
    dx = r * (g - gm - xhat * along)
    size = g.abs() + gm.abs() + (xhat * along).abs()
    tol = r * (58 * U * g.abs().mean(1, keepdim=True) + xhat.abs() * 62 * U * (g * xhat).abs().mean(1, keepdim=True) + 8 * U * size)
    if dsum is not None:
        dx = dx + dsum.double()
        tol = tol + U * dx.abs()
    p = d * xhat
    return (dx, p.sum(0), d.sum(0)), (tol, (T + 54) * U * p.abs().sum(0), (T + 50) * U * d.abs().sum(0))


def adapters(x, ids, a, b, base):
    """(y, tolerance before the last rounding): x A is summed in fp32 (K additions at most) and taken as two bf16 values, the second within half a
    step of what the first leaves; then 2 r additions more."""
    T, N = x.shape[0], b[0].shape[1]
    y = torch.zeros(T, N, dtype=torch.float64) if base is None else base.double().clone()
    size, tol = y.abs().clone(), torch.zeros_like(y)
    for i in range(len(a)):
        rows = torch.nonzero(ids == i)[:, 0]
        if len(rows) == 0 or a[i].shape[1] == 0:
            continue
        xd, ad, bd = x[rows].double(), a[i].double(), b[i].double()
        t = xd @ ad
        off = HALVES * t.abs() * 1.01 + (ad.shape[0] + 40) * U * (xd.abs() @ ad.abs())
        y[rows] += t @ bd
        size[rows] += t.abs() @ bd.abs()
        tol[rows] += off @ bd.abs() + (2 * ad.shape[1] + 2) * U * (1.01 * t.abs() @ bd.abs())
    y[ids >= len(a)] = float("nan")
    return y, tol + 2 * U * size


def adapters_backward(dy, x, ids, a, b, dx_base):
    """(dx, da, db) with their tolerances."""
    K = a[0].shape[0]
    dx, tol = adapters(dy, ids, [m.t() for m in b], [m.t() for m in a], dx_base if dx_base is not None else torch.zeros(dy.shape[0], K))
    da, db = [], []
    for i in range(len(a)):
        rows = torch.nonzero(ids == i)[:, 0]
        xd, dyd, ad, bd = x[rows].double(), dy[rows].double(), a[i].double(), b[i].double()
        dt, t = dyd @ bd.t(), xd @ ad
        off_dt = HALVES * 1.01 * dt.abs() + (bd.shape[1] + 40) * U * (dyd.abs() @ bd.abs().t())
        off_t = HALVES * 1.01 * t.abs() + (ad.shape[0] + 40) * U * (xd.abs() @ ad.abs())
        n = (2 * len(rows) + 2) * U * 1.01
        da.append((xd.t() @ dt, xd.abs().t() @ (off_dt + n * dt.abs())))
        db.append((t.t() @ dyd, (off_t + n * t.abs()).t() @ dyd.abs()))
    return (dx, tol), da, db


def close(got, want, tol, dtype):
    """got, of `dtype`, is want off by tol and rounded.  NaN where want is."""
    got = got.detach().cpu().double()
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(got), bad), "NaN elsewhere"
    off = (got - want).abs()
    room = tol + (half(dtype) * (want.abs() + tol) if dtype != torch.float32 else 0.0) + 1e-37
    over = torch.where(bad, torch.zeros_like(off), off - room)
    where = int(over.argmax()) if over.numel() else 0
    assert over.numel() == 0 or over.max() <= 0, (where, got.reshape(-1)[where].item(), want.reshape(-1)[where].item(), room.reshape(-1)[where].item())
