"""GPU tests of the layer norm's gradient with dw and db over more rows than go in one launch, against 64 bits: every team and number of vectors a lane, rows of
whole vectors and of odd lengths.  Which of the two ways a call took is seen from its workspace, which the one-launch form leaves alone.

Tolerances are those of tests/beside_ref.py but for the additions of a row's sum: 8 a vector of a lane, 6 over the wave, one a wave of the team.
"""
import pytest
import torch

import beside_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu

# (rows, length, waves of a team, vectors of a lane)
FORMS = [(514, 264, 1, 1), (2100, 509, 1, 1), (513, 1024, 1, 2), (600, 777, 1, 2), (4200, 515, 1, 2), (520, 2048, 2, 2), (530, 1031, 2, 2), (515, 4096, 4, 2),
         (1111, 2721, 4, 2), (513, 2049, 4, 2), (515, 8192, 8, 2), (515, 4097, 8, 2), (514, 14336, 8, 4), (514, 16384, 8, 4), (513, 8195, 8, 4), (513, 32768, 8, 8),
         (514, 16391, 8, 8), (513, 32761, 8, 8)]


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    return salr


def _reference(dy, x, weight, mean, rstd, dsum, additions):
    """(dx, dw, db) and tolerances: g is off by a rounding, xhat by two, a row's sums by `additions` more and their division, what is formed of them by 8."""
    T, K = x.shape
    d, w, r = dy.double(), weight.double(), rstd.double()[:, None]
    xhat = (x.double() - mean.double()[:, None]) * r
    g = d * w
    g_mean, along = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    dx = r * (g - g_mean - xhat * along)
    tol = r * ((additions + 4) * ref.U * g.abs().mean(1, keepdim=True) + xhat.abs() * (additions + 8) * ref.U * (g * xhat).abs().mean(1, keepdim=True)
               + 8 * ref.U * (g.abs() + g_mean.abs() + (xhat * along).abs()))
    if dsum is not None:
        dx = dx + dsum.double()
        tol = tol + ref.U * dx.abs()
    p = d * xhat
    return (dx, p.sum(0), d.sum(0)), (tol, (T + 54) * ref.U * p.abs().sum(0), (T + 50) * ref.U * d.abs().sum(0))


@pytest.mark.parametrize("T,K,team,units", FORMS)
@pytest.mark.parametrize("dtype,wtype", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
def test_backward(salr, T, K, team, units, dtype, wtype):
    gen = torch.Generator().manual_seed(T + K)
    x = (torch.randn(T, K, generator=gen) * (1 + torch.rand(T, 1, generator=gen)) + torch.randn(T, 1, generator=gen)).to(dtype)
    dy, dsum = torch.randn(T, K, generator=gen).to(dtype), torch.randn(T, K, generator=gen).to(dtype)
    weight = (1 + 0.3 * torch.randn(K, generator=gen)).to(wtype)
    mean = x.double().mean(1)
    rstd = ((x.double() - mean[:, None]).square().mean(1) + 1e-5).rsqrt().float()
    mean = mean.float()
    want, tol = _reference(dy, x, weight, mean, rstd, dsum, 8 * units + 6 + team)
    host = {"dy": dy, "x": x, "dsum": dsum}
    w, stats = weight.to(dev()), (mean.to(dev()), rstd.to(dev()))
    ws = torch.empty(salr.salr_layer_norm_backward_workspace_bytes(T, K, True), dtype=torch.uint8, device=dev())
    first = None
    for place in ("apart", "dy", "x", "dsum", "none"):
        d = {k: t.to(dev()) for k, t in host.items()}
        dx = torch.empty_like(d["x"]) if place == "apart" else d.get(place)
        dw, db = torch.empty_like(w), torch.empty_like(w)
        ws.fill_(255)
        salr.salr_layer_norm_backward(d["dy"], d["x"], w, *stats, d["dsum"], dx, dw, db, ws)
        assert bool((ws != 255).any()), "one launch: more rows are needed here"
        if first is None:
            for got, value, t, kind in zip((dx, dw, db), want, tol, (dtype, wtype, wtype)):
                ref.close(got, value, t, kind)
            first = dx, dw, db
        else:   # wherever dx goes, and without it: the same bits
            assert dx is None or torch.equal(dx, first[0]), place
            assert torch.equal(dw, first[1]) and torch.equal(db, first[2]), place
    got = salr.layer_norm_backward(d["dy"], d["x"], w, *stats, need_db=True)   # one of the two alone, no dsum
    want, tol = _reference(dy, x, weight, mean, rstd, None, 8 * units + 6 + team)
    ref.close(got[0], want[0], tol[0], dtype)
    assert got[1] is None and torch.equal(got[2], first[2])


@pytest.mark.parametrize("K", [515, 4099])
def test_neighbours_stay(salr, K):
    """dx at an element's address between guards, rows of odd lengths."""
    T = 520
    gen = torch.Generator().manual_seed(K)
    dy, x = (torch.randn(T, K, generator=gen).bfloat16().to(dev()) for _ in range(2))
    w = torch.ones(K, device=dev())
    _, _, mean, rstd = salr.layer_norm(x, w)
    want = salr.layer_norm_backward(dy, x, w, mean, rstd, need_dw=True, need_db=True)
    buf = torch.full((T * K + 40,), 3.0, dtype=torch.bfloat16, device=dev())
    sums = torch.full((2 * K + 40,), 3.0, device=dev())
    dx, dw, db = buf[5:5 + T * K].view(T, K), sums[3:3 + K], sums[20 + K:20 + 2 * K]
    dx.copy_(dy)
    ws = torch.full((salr.salr_layer_norm_backward_workspace_bytes(T, K, True) + 64,), 255, dtype=torch.uint8, device=dev())
    salr.salr_layer_norm_backward(dx, x, w, mean, rstd, None, dx, dw, db, ws[:-64])
    assert bool((ws[:-64] != 255).any()) and bool((ws[-64:] == 255).all())
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), want))
    assert bool((buf[:5] == 3).all()) and bool((buf[5 + T * K:] == 3).all())
    assert bool((sums[:3] == 3).all()) and bool((sums[3 + K:20 + K] == 3).all()) and bool((sums[20 + 2 * K:] == 3).all())


@pytest.mark.parametrize("T,K", [(1, 5), (300, 1031), (512, 4096), (130, 32768)])
def test_one_launch_leaves_its_workspace_alone(salr, T, K):
    gen = torch.Generator().manual_seed(T + K)
    dy, x = (torch.randn(T, K, generator=gen).to(dev()) for _ in range(2))
    w = torch.ones(K, device=dev())
    _, _, mean, rstd = salr.layer_norm(x, w)
    want = salr.layer_norm_backward(dy, x, w, mean, rstd, need_dw=True, need_db=True)
    need = salr.salr_layer_norm_backward_workspace_bytes(T, K, True)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=dev())
    got = salr.layer_norm_backward(dy, x, w, mean, rstd, need_dw=True, need_db=True, workspace=ws[:need])
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and bool((ws == 255).all())
