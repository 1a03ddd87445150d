"""GPU tests of salr_dropout: the mask bit for bit against Philox on the CPU, values against 64 bits (tests/beside_ref.py has the tolerances)."""
import pytest
import torch

import beside_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    return salr


def _made(shape, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=gen).to(dtype), torch.randn(shape, generator=gen).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5), (48, 512), (111, 271), (2049, 1023), (4200, 4111)])
def test_against_the_counter(salr, shape, dtype):
    x, r = _made(shape, dtype, 1)
    for p, residual in ((0.1, None), (0.35, r), (0.0, r)):
        got = salr.dropout(x.to(dev()), p, 0x123456789ABCDEF, 77, residual=None if residual is None else residual.to(dev()))
        want, tol = ref.dropout(x, p, 0x123456789ABCDEF, 77, residual)
        assert got.dtype == dtype and got.shape == x.shape
        ref.close(got, want, tol, dtype)
        if residual is None:
            assert torch.equal(got.cpu() != 0, (want != 0) & (got.cpu() != 0))
            assert torch.equal(got.cpu() == 0, (want == 0) | (x == 0))


def test_seeds_and_offsets(salr):
    x = torch.ones(100000, device=dev())
    first = salr.dropout(x, 0.5, 3, 0)
    assert torch.equal(first, salr.dropout(x, 0.5, 3, 0))
    for seed, offset in ((4, 0), (3, 1), (-3, 0), (2 ** 62, 0), (3, 2 ** 40)):
        other = salr.dropout(x, 0.5, seed, offset)
        assert torch.equal(other.cpu() != 0, ref.keep_mask(100000, 0.5, seed, offset))
        same = float((other == first).float().mean())
        assert abs(same - 0.5) < 6 * 0.5 / 100000 ** 0.5   # six standard deviations
    share = float((salr.dropout(x, 0.25, 9) != 0).float().mean())
    assert abs(share - 0.75) < 6 * (0.1875 / 100000) ** 0.5
    assert torch.equal(salr.dropout(x, 0.0, 9), x)
    assert float(salr.dropout(x, 65535 / 65536, 9).max()) == 65536.0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_is_dropped_may_be_anything(salr, dtype):
    x, _ = _made((1000,), dtype, 3)
    keep = ref.keep_mask(1000, 0.5, 11, 0)
    x[~keep] = float("nan")
    x[torch.nonzero(~keep)[::3, 0]] = float("inf")
    got = salr.dropout(x.to(dev()), 0.5, 11).cpu()
    assert bool(torch.isfinite(got).all()) and bool((got[~keep] == 0).all())


def test_gradient_is_the_same_call(salr):
    """y is linear in x: its differences are the mask, and the gradient of sum(y dy) is the call on dy."""
    x, dy = _made((33, 77), torch.float32, 4)
    e = torch.zeros_like(x)
    e[::2, ::3] = 1.0
    args = (0.3, 21, 5)
    moved = salr.dropout((x + e).to(dev()), *args) - salr.dropout(x.to(dev()), *args)
    grad = salr.dropout(dy.to(dev()), *args)
    lhs, rhs = float((moved.cpu().double() * dy).sum()), float((grad.cpu().double() * ((x + e) - x).double()).sum())
    room = 4 * ref.U * float(((x.abs() + 1) * 2 * dy.abs() / 0.7).double().sum())
    assert abs(lhs - rhs) <= room


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_place_and_neighbours(salr, dtype):
    x, r = _made((1001,), dtype, 5)
    want = salr.dropout(x.to(dev()), 0.2, 6, residual=r.to(dev()))
    for place in ("x", "residual", "apart"):
        buf = torch.full((3 * 1024,), 7.0, dtype=dtype, device=dev())
        xs, rs, ys = buf[1:1002], buf[1025:2026], buf[2050:3051]   # element addresses, no vector's
        xs.copy_(x)
        rs.copy_(r)
        y = {"x": xs, "residual": rs, "apart": ys}[place]
        salr.salr_dropout(xs, rs, 0.2, 6, 0, y)
        assert torch.equal(y, want)
        rest = torch.ones(3 * 1024, dtype=torch.bool, device=dev())
        for s in (slice(1, 1002), slice(1025, 2026), slice(2050, 3051)):
            rest[s] = False
        assert bool((buf[rest] == 7.0).all())


def test_captured_with_a_seed_on_the_device(salr):
    x = torch.randn(5000, device=dev())
    seed, y = torch.tensor([5], device=dev()), torch.empty(5000, device=dev())
    salr.salr_dropout(x, None, 0.5, seed, 0, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        salr.salr_dropout(x, None, 0.5, seed, 0, y)
    for step in range(5):
        seed.fill_(100 + step)
        graph.replay()
        assert torch.equal(y, salr.dropout(x, 0.5, 100 + step)), step
        torch.cuda.synchronize()


def test_streams(salr):
    x = torch.randn(1 << 20, device=dev())
    want = salr.dropout(x, 0.5, 1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = salr.dropout(x, 0.5, 1, stream=side)
    out = torch.empty_like(x)
    salr.salr_dropout(x, None, 0.5, 1, 0, out, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(out, want)


def test_more_than_the_grid(salr):
    """70 M elements: the grid's threads go round four times."""
    n = 70_000_003
    x = torch.ones(n, dtype=torch.bfloat16, device=dev())
    got = salr.dropout(x, 0.5, 12, 3) != 0
    for start in (0, 16 * 1024 * 1024 - 8, 4 * 8192 * 2048 - 64, n - 1003):
        start = start // 8 * 8
        block = torch.arange(start // 8, start // 8 + 125).numpy().astype("uint64")
        words = ref.philox([block, block * 0, block * 0 + 3, block * 0], [12, 0])
        bits = torch.stack([torch.from_numpy(h.astype("int64")) for w in words for h in (w & 0xFFFF, w >> 16)], dim=1).reshape(-1)
        here = min(1000, n - start)
        assert torch.equal(got[start:start + here].cpu(), (bits >= 32768)[:here])


def test_empty(salr):
    assert salr.dropout(torch.empty(0, 5, device=dev()), 0.1, 1).shape == (0, 5)


def test_refusals(salr):
    x = torch.randn(64, device=dev())
    with pytest.raises(TypeError):
        salr.dropout(x.half(), 0.1, 1)
    with pytest.raises(TypeError):
        salr.dropout(x.view(8, 8).t(), 0.1, 1)
    with pytest.raises(TypeError):
        salr.dropout(x.cpu(), 0.1, 1)
    with pytest.raises(TypeError):
        salr.dropout(x, 0.1, 1, residual=x.bfloat16())
    with pytest.raises(ValueError):
        salr.dropout(x, 0.1, 1, residual=x[:32])
    with pytest.raises(ValueError):
        salr.dropout(x, 0.1, torch.zeros(2, dtype=torch.int64, device=dev()))
    with pytest.raises(TypeError):
        salr.dropout(x, 0.1, torch.zeros(1, dtype=torch.int32, device=dev()))
    for p in (-0.1, 1.0, 1.5, float("nan"), 1 - 2.0 ** -18):
        with pytest.raises(salr.SalrError):
            salr.dropout(x, p, 1)
    with pytest.raises(salr.SalrError):
        salr.salr_dropout(x[:40], None, 0.1, 1, 0, x[8:48])
