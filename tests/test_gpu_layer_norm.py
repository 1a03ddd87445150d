"""GPU tests of salr_layer_norm and its gradient against 64 bits (tests/beside_ref.py derives the tolerances)."""
import pytest
import torch

import beside_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 7), (3, 8), (5, 9), (2, 511), (7, 512), (4, 513), (3, 1024), (5, 1031), (3, 2048), (33, 2049), (2, 2720), (1, 4096), (130, 4096), (3, 4097),
          (2, 8192), (3, 8195), (2, 14336), (2, 16384), (2, 16391), (1, 28672), (3, 32768), (1100, 264)]


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    return salr


def _inputs(T, K, dtype, wtype, seed=0):
    gen = torch.Generator().manual_seed(seed + T + K)
    x = torch.randn(T, K, generator=gen) * torch.exp(torch.randn(T, 1, generator=gen)) + 3 * torch.randn(T, 1, generator=gen)
    x[:, ::100] *= 20
    return {"x": x.to(dtype), "residual": torch.randn(T, K, generator=gen).to(dtype), "weight": (1 + 0.3 * torch.randn(K, generator=gen)).to(wtype),
            "bias": torch.randn(K, generator=gen).to(wtype), "dy": torch.randn(T, K, generator=gen).to(dtype), "dsum": torch.randn(T, K, generator=gen).to(dtype)}


def _forward(salr, s, residual, bias, eps=1e-5):
    d = {k: t.to(dev()) for k, t in s.items()}
    return salr.layer_norm(d["x"], d["weight"], d["bias"] if bias else None, eps, residual=d["residual"] if residual else None)


@pytest.mark.parametrize("T,K", SHAPES)
@pytest.mark.parametrize("dtype,wtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32), (torch.float32, torch.bfloat16)])
def test_forward(salr, T, K, dtype, wtype):
    s = _inputs(T, K, dtype, wtype)
    for residual, bias in ((False, True), (True, False)):
        y, total, mean, rstd = _forward(salr, s, residual, bias)
        kept = (s["x"].float() + s["residual"].float()).to(dtype) if residual else s["x"]
        assert (total is not None) == residual
        if residual:
            assert torch.equal(total.cpu(), kept)
        want, tol = ref.layer_norm(kept, s["weight"], s["bias"] if bias else None, 1e-5)
        for got, w, t, kind in zip((y, mean, rstd), want, tol, (dtype, torch.float32, torch.float32)):
            ref.close(got, w, t, kind)


@pytest.mark.parametrize("T,K", SHAPES)
@pytest.mark.parametrize("dtype,wtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
def test_backward(salr, T, K, dtype, wtype):
    s = _inputs(T, K, dtype, wtype, 5)
    x = s["x"].double()
    mean = x.mean(1).float()
    rstd = (x.var(1, unbiased=False) + 1e-5).rsqrt().float()
    d = {k: t.to(dev()) for k, t in s.items()}
    args = (d["dy"], d["x"], d["weight"], mean.to(dev()), rstd.to(dev()))
    for dsum, weights in ((True, True), (False, False), (True, False), (False, True)):
        dx, dw, db = salr.layer_norm_backward(*args, dsum=d["dsum"] if dsum else None, need_dw=weights, need_db=weights)
        want, tol = ref.layer_norm_backward(s["dy"], s["x"], s["weight"], mean, rstd, s["dsum"] if dsum else None)
        ref.close(dx, want[0], tol[0], dtype)
        if weights:
            ref.close(dw, want[1], tol[1], wtype)
            ref.close(db, want[2], tol[2], wtype)
        else:
            assert dw is None and db is None
    only = salr.layer_norm_backward(*args, need_dx=False, need_dw=True)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dw)
    only = salr.layer_norm_backward(*args, need_dx=False, need_db=True)
    assert only[0] is None and only[1] is None and torch.equal(only[2], db)


def test_gradient_against_differences(salr):
    """fp32, the loss sum(y dy) in 64 bits from the kernel's y at x +- h e: each y is off by its tolerance, and the second difference by h^2."""
    s = _inputs(4, 300, torch.float32, torch.float32, 9)
    s["x"] = torch.randn(4, 300, generator=torch.Generator().manual_seed(3))
    y, _, mean, rstd = _forward(salr, s, False, True)
    d = {k: t.to(dev()) for k, t in s.items()}
    dx, dw, db = salr.layer_norm_backward(d["dy"], d["x"], d["weight"], mean, rstd, need_dw=True, need_db=True)
    _, tols = ref.layer_norm_backward(s["dy"], s["x"], s["weight"], mean.cpu(), rstd.cpu(), None)
    gen = torch.Generator().manual_seed(1)
    h = 2.0 ** -6
    for name, grad, grad_tol in zip(("x", "weight", "bias"), (dx, dw, db), tols):
        e = torch.randn(s[name].shape, generator=gen)
        values, exact = [], []
        for sign in (1, -1):
            moved = dict(s, **{name: s[name] + sign * h * e})
            y2, _, _, _ = _forward(salr, moved, False, True)
            want, tol = ref.layer_norm(moved["x"], moved["weight"], moved["bias"], 1e-5)
            values.append(float((y2.cpu().double() * s["dy"].double()).sum()))
            exact.append(float((want[0] * s["dy"].double()).sum()))
        noise = float((tol[0] * s["dy"].abs().double()).sum()) / h
        # what the difference quotient itself is off by, from the same quotient in 64 bits at an eighth of the step
        slopes = []
        for step in (h, h / 8):
            f = [float((ref.layer_norm(*[(s[k].double() + (sign * step * e.double() if k == name else 0)) for k in ("x", "weight", "bias")], 1e-5)[0][0]
                        * s["dy"].double()).sum()) for sign in (1, -1)]
            slopes.append((f[0] - f[1]) / (2 * step))
        rounding = abs((exact[0] - exact[1]) / (2 * h) - slopes[0])   # of x +- h e to fp32
        slope = float((grad.cpu().double() * e.double()).sum())
        # the gradient's own tolerance, of at least eight roundings of its terms; mean and rstd are off by up to 130 of them
        grad_tol = 25 * float((grad_tol * e.abs().double()).sum())
        assert abs((values[0] - values[1]) / (2 * h) - slope) <= 1.1 * abs(slopes[0] - slopes[1]) + noise + rounding + grad_tol, name


def test_means_far_from_zero(salr):
    """Squares alone would lose this: a mean of 1000 with a deviation of 0.1."""
    x = 1000 + 0.1 * torch.randn(6, 4096, generator=torch.Generator().manual_seed(2))
    w = torch.ones(4096)
    y, _, mean, rstd = salr.layer_norm(x.to(dev()), w.to(dev()))
    want, tol = ref.layer_norm(x, w, None, 1e-5)
    for got, a, t in zip((y, mean, rstd), want, tol):
        ref.close(got, a, t, torch.float32)
    assert float((rstd.cpu().double() / want[2] - 1).abs().max()) < 1e-3


def test_constant_rows_and_eps(salr):
    x = torch.full((3, 100), 2.5)
    y, _, mean, rstd = salr.layer_norm(x.to(dev()), torch.ones(100, device=dev()), eps=1e-6)
    assert bool((y == 0).all()) and bool((mean == 2.5).all())
    assert torch.allclose(rstd, torch.full_like(rstd, 1000.0), rtol=1e-5)
    y, _, _, rstd = salr.layer_norm(x.to(dev()), torch.ones(100, device=dev()), eps=0.0)
    assert bool(torch.isinf(rstd).all()) and bool(torch.isnan(y).all())


@pytest.mark.parametrize("K", [300, 4096])
def test_rows_do_not_touch_each_other(salr, K):
    s = _inputs(9, K, torch.bfloat16, torch.float32)
    clean = _forward(salr, s, True, True)
    bad = dict(s, x=s["x"].clone())
    bad["x"][2, 5], bad["x"][6, 0] = float("nan"), float("inf")
    got = _forward(salr, bad, True, True)
    rows = [0, 1, 3, 4, 5, 7, 8]
    for a, b in zip(clean, got):
        assert torch.equal(a[rows], b[rows])
    assert bool(torch.isnan(got[0][2]).all()) and bool(torch.isnan(got[0][6]).all())
    d = {k: t.to(dev()) for k, t in s.items()}
    dy = d["dy"].clone()
    dy[4, 3] = float("inf")
    one = salr.layer_norm_backward(d["dy"], clean[1], d["weight"], clean[2], clean[3])[0]
    two = salr.layer_norm_backward(dy, clean[1], d["weight"], clean[2], clean[3])[0]
    rows = [0, 1, 2, 3, 5, 6, 7, 8]
    # (both sums of that row are infinite: minus infinity where they agree, NaN where they do not)
    assert torch.equal(one[rows], two[rows]) and not bool(torch.isfinite(two[4]).any())


def test_in_place(salr):
    s = _inputs(37, 1031, torch.bfloat16, torch.bfloat16)
    y, total, mean, rstd = _forward(salr, s, True, True)
    for y_at, sum_at in (("x", "residual"), ("residual", "x"), ("x", None), (None, "residual")):
        d = {k: t.to(dev()) for k, t in s.items()}
        y2, sum2 = (torch.empty_like(d["x"]) if at is None else d[at] for at in (y_at, sum_at))
        salr.salr_layer_norm(d["x"], d["residual"], d["weight"], d["bias"], 1e-5, y2, sum2, None, None)
        assert torch.equal(y2, y) and torch.equal(sum2, total)
    d = {k: t.to(dev()) for k, t in s.items()}
    dx, dw, db = salr.layer_norm_backward(d["dy"], total, d["weight"], mean, rstd, dsum=d["dsum"], need_dw=True, need_db=True)
    for at in ("dy", "x", "dsum"):
        d = {k: t.to(dev()) for k, t in s.items()}
        d["x"] = total.clone()
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        ws = torch.empty(salr.salr_layer_norm_backward_workspace_bytes(37, 1031, True), dtype=torch.uint8, device=dev())
        salr.salr_layer_norm_backward(d["dy"], d["x"], d["weight"], mean, rstd, d["dsum"], d[at], dw2, db2, ws)
        assert torch.equal(d[at], dx) and torch.equal(dw2, dw) and torch.equal(db2, db)


@pytest.mark.parametrize("T,K", [(255, 264), (256, 1031), (257, 1031), (256, 16384), (511, 515), (512, 4096), (513, 4096), (40, 32768)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_backward_about_few_rows(salr, T, K, dtype):
    """The numbers of rows between which the sums of dw and db move into the launch that forms dx; dx apart, in dy's place and in x's."""
    s = _inputs(T, K, dtype, torch.float32, 11)
    x = s["x"].double()
    mean = x.mean(1).float()
    rstd = (x.var(1, unbiased=False) + 1e-5).rsqrt().float()
    want, tol = ref.layer_norm_backward(s["dy"], s["x"], s["weight"], mean, rstd, s["dsum"])
    ws = torch.empty(salr.salr_layer_norm_backward_workspace_bytes(T, K, True), dtype=torch.uint8, device=dev())
    for at in (None, "dy", "x"):
        d = {k: t.to(dev()) for k, t in s.items()}
        dx = torch.empty_like(d["x"]) if at is None else d[at]
        dw, db = torch.empty(K, device=dev()), torch.empty(K, device=dev())
        salr.salr_layer_norm_backward(d["dy"], d["x"], d["weight"], mean.to(dev()), rstd.to(dev()), d["dsum"], dx, dw, db, ws)
        ref.close(dx, want[0], tol[0], dtype)
        ref.close(dw, want[1], tol[1], torch.float32)
        ref.close(db, want[2], tol[2], torch.float32)


@pytest.mark.parametrize("K", [9, 515, 4099])
def test_neighbours_stay(salr, K):
    s = _inputs(5, K, torch.bfloat16, torch.float32)
    want = _forward(salr, s, False, False)
    n = 5 * K
    buf = torch.full((2 * n + 64,), 3.0, dtype=torch.bfloat16, device=dev())
    x, y = buf[3:3 + n].view(5, K), buf[n + 30:2 * n + 30].view(5, K)   # element addresses, no vector's
    x.copy_(s["x"])
    salr.salr_layer_norm(x, None, s["weight"].to(dev()), None, 1e-5, y, None, None, None)
    assert torch.equal(y, want[0])
    assert bool((buf[:3] == 3).all()) and bool((buf[3 + n:n + 30] == 3).all()) and bool((buf[2 * n + 30:] == 3).all())
    dx = salr.layer_norm_backward(s["dy"].to(dev()), x, s["weight"].to(dev()), want[2], want[3])[0]
    salr.salr_layer_norm_backward(s["dy"].to(dev()), x, s["weight"].to(dev()), want[2], want[3], None, y, None, None, None)
    assert torch.equal(y, dx)
    assert bool((buf[:3] == 3).all()) and bool((buf[3 + n:n + 30] == 3).all()) and bool((buf[2 * n + 30:] == 3).all())


def test_empty(salr):
    w = torch.ones(16, device=dev())
    x = torch.empty(0, 16, device=dev())
    y, total, mean, rstd = salr.layer_norm(x, w)
    assert y.shape == (0, 16) and total is None and mean.numel() == 0
    dx, dw, db = salr.layer_norm_backward(x, x, w, mean, rstd, need_dw=True, need_db=True)
    assert dx.shape == (0, 16) and bool((dw == 0).all()) and bool((db == 0).all())


def test_captured(salr):
    s = _inputs(200, 777, torch.bfloat16, torch.float32)
    d = {k: t.to(dev()) for k, t in s.items()}
    y, total = torch.empty_like(d["x"]), torch.empty_like(d["x"])
    mean, rstd = torch.empty(200, device=dev()), torch.empty(200, device=dev())
    dx, dw, db = torch.empty_like(d["x"]), torch.empty_like(d["weight"]), torch.empty_like(d["weight"])
    ws = torch.empty(salr.salr_layer_norm_backward_workspace_bytes(200, 777, True), dtype=torch.uint8, device=dev())

    def step():
        salr.salr_layer_norm(d["x"], d["residual"], d["weight"], d["bias"], 1e-5, y, total, mean, rstd)
        salr.salr_layer_norm_backward(d["dy"], total, d["weight"], mean, rstd, d["dsum"], dx, dw, db, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        d["x"].copy_(_inputs(200, 777, torch.bfloat16, torch.float32, 50 + i)["x"])
        graph.replay()
        got = [t.clone() for t in (y, total, mean, rstd, dx, dw, db)]
        ws.fill_(255)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, total, mean, rstd, dx, dw, db))), i


def test_streams(salr):
    s = _inputs(500, 4096, torch.bfloat16, torch.float32)
    want = _forward(salr, s, True, True)
    d = {k: t.to(dev()) for k, t in s.items()}
    grads = salr.layer_norm_backward(d["dy"], want[1], d["weight"], want[2], want[3], need_dw=True, need_db=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = salr.layer_norm(d["x"], d["weight"], d["bias"], residual=d["residual"], stream=side)
    grads2 = salr.layer_norm_backward(d["dy"], got[1], d["weight"], got[2], got[3], need_dw=True, need_db=True, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want + grads, got + grads2))


def test_refusals(salr):
    x = torch.randn(4, 32, device=dev())
    w = torch.ones(32, device=dev())
    stats = torch.ones(4, device=dev())
    for bad in (dict(x=x.half()), dict(x=x.cpu()), dict(x=x.t()), dict(weight=w.half()), dict(weight=None), dict(bias=w.bfloat16()), dict(residual=x.bfloat16())):
        with pytest.raises(TypeError):
            salr.layer_norm(**{"x": x, "weight": w, **bad})
    for bad in (dict(x=x[0]), dict(weight=w[:16]), dict(bias=w[:16]), dict(residual=x[:2])):
        with pytest.raises(ValueError):
            salr.layer_norm(**{"x": x, "weight": w, **bad})
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(salr.SalrError):
            salr.layer_norm(x, w, eps=eps)
    with pytest.raises(salr.SalrError):
        salr.layer_norm(torch.zeros(1, 32769, device=dev()), torch.zeros(32769, device=dev()))
    for bad in (dict(mean=stats.double()), dict(rstd=None), dict(dsum=x.bfloat16()), dict(dy=None)):
        with pytest.raises(TypeError):
            salr.layer_norm_backward(**{"dy": x, "x": x, "weight": w, "mean": stats, "rstd": stats, **bad})
    for bad in (dict(mean=stats[:2]), dict(dy=x[:2])):
        with pytest.raises(ValueError):
            salr.layer_norm_backward(**{"dy": x, "x": x, "weight": w, "mean": stats, "rstd": stats, **bad})
    with pytest.raises(salr.SalrError):   # a workspace that is too small
        salr.layer_norm_backward(x, x, w, stats, stats, need_dw=True, workspace=torch.empty(16, dtype=torch.uint8, device=dev()))
    with pytest.raises(salr.SalrError):   # in part
        salr.salr_layer_norm(x[:3], None, w, None, 1e-5, x[1:], None, None, None)
    with pytest.raises(salr.SalrError):   # y is sum
        y = torch.empty_like(x)
        salr.salr_layer_norm(x, x.clone(), w, None, 1e-5, y, y, None, None)
