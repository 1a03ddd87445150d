"""GPU tests of norm, shared layer, dropout and adapters as they are used together, forward and backward, against 64 bits, and of the example that trains so.

Tolerance of a chain: every stage rounds to bf16 once, by 2^-8 of each value at most, and passes on what it was given; the maps have a norm of about one (the
weights are scaled for that), so n stages leave n 2^-8 of a result's norm.
"""
import importlib.util
import os

import pytest
import torch

import beside_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("finetune_tenants", os.path.join(ROOT, "examples", "finetune_tenants.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    return salr


def _close(got, want, stages):
    off = float((got.detach().cpu().double() - want).norm() / want.norm())
    assert off <= stages * 2.0 ** -8, off


def _dense(salr, block, K):
    return salr.decode(*block.weight, K, K).view(torch.bfloat16).cpu().double()


def test_a_block_forward_and_backward(salr):
    """One block of the example between a given stream and a given gradient: what it adds, the stream's gradient, and every weight's."""
    T, K, n = 192, 256, 3
    gen = torch.Generator(device="cuda").manual_seed(3)
    block = _example().Block(K, [8, 24, 13], 0.2, 7, gen)
    for m, c in zip(block.master[n:], block.copy[n:]):
        c.copy_(m.normal_(0.0, 0.2, generator=gen))
    block.norm[0].normal_(1.0, 0.2, generator=gen)
    block.norm[1].normal_(0.0, 0.2, generator=gen)
    h, add, dy = (torch.randn(T, K, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(3))
    ids = torch.randint(-1, n, (T,), device="cuda", generator=gen, dtype=torch.int32)
    stream, out = block.forward(h, add, ids, 5)
    dh = block.backward(dy)

    leaf = lambda t: t.detach().cpu().double().requires_grad_()   # noqa: E731
    a, b = [leaf(c) for c in block.copy[:n]], [leaf(c) for c in block.copy[n:]]
    w, bias, s = leaf(block.norm[0]), leaf(block.norm[1]), leaf(stream)
    assert torch.equal(stream.cpu(), (h.float() + add.float()).to(torch.bfloat16).cpu())
    d = s - s.mean(1, keepdim=True)
    x = d * (d.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w + bias
    keep = ref.keep_mask(T * K, 0.2, 5, 7).view(T, K)
    xd = x * keep / (1 - int(0.2 * 65536 + 0.5) / 65536)
    y = x @ _dense(salr, block, K).t()
    where = ids.cpu()
    delta = torch.zeros_like(y)
    for i in range(n):
        rows = torch.nonzero(where == i)[:, 0]
        delta = delta.index_add(0, rows, xd[rows] @ a[i] @ b[i])
    total = s + y + delta
    (total * dy.cpu().double()).sum().backward()
    _close(out, (y + delta).detach(), 4)          # norm, dropout, layer, sum
    _close(dh, s.grad, 8)                         # four stages back through four
    _close(block.norm_grad[0], w.grad, 7)
    _close(block.norm_grad[1], bias.grad, 7)
    for i in range(n):
        _close(block.grad[i], a[i].grad, 6)       # dy is exact; x two stages, its product, the result
        _close(block.grad[n + i], b[i].grad, 6)


def test_set_linear_is_layer_and_adapters(salr):
    """AdapterSet.linear: the layer's output with every token's adapter added; one adapter for all tokens is what ``linear`` does with it."""
    T, K = 100, 512
    gen = torch.Generator(device="cuda").manual_seed(4)
    block = _example().Block(K, [16, 8], 0.0, 0, gen)
    for c in block.copy[2:]:
        c.normal_(0.0, 0.2, generator=gen)
    x = torch.randn(T, K, device="cuda", generator=gen).to(torch.bfloat16)
    ids = torch.randint(-1, 2, (T,), device="cuda", generator=gen, dtype=torch.int32)
    got = block.adapters.linear(x, *block.weight, ids)
    base = salr.linear(x, *block.weight, None, None)
    want, tol = ref.adapters(x.cpu(), ids.cpu(), [c.cpu() for c in block.copy[:2]], [c.cpu() for c in block.copy[2:]], base.cpu())
    ref.close(got, want, tol, torch.bfloat16)
    one = block.adapters.linear(x, *block.weight, torch.zeros_like(ids))
    _close(one, salr.linear(x, *block.weight, block.copy[0], block.copy[2]).cpu().double(), 3)


def test_gradients_of_the_example_against_differences(salr):
    """The example's step on a model small enough for 64-bit differences along a direction in each kind of weight."""
    T, K, V, n = 96, 128, 150, 2
    gen = torch.Generator(device="cuda").manual_seed(6)
    model = _example().Model(K, V, [8, 16], 1, 0.1, gen)
    block = model.blocks[0]
    for m, c in zip(block.master[n:], block.copy[n:]):
        c.copy_(m.normal_(0.0, 0.3, generator=gen))
    tokens = torch.randint(0, 64, (T,), device="cuda", generator=gen)
    targets = torch.randint(0, V, (T,), device="cuda", generator=gen)
    targets[:12] = -100
    ids = torch.sort(torch.randint(0, n, (T,), device="cuda", generator=gen, dtype=torch.int32)).values
    loss = model.step(tokens, targets, ids, 9)
    dense = _dense(salr, block, K)
    keep = ref.keep_mask(T * K, 0.1, 9, 0).view(T, K).double() / (1 - int(0.1 * 65536 + 0.5) / 65536)
    weights = [c.cpu().double() for c in block.copy] + [p.cpu().double() for p in block.norm]
    h, head, goal, where = model.embedding[tokens].cpu().double(), model.head.cpu().double(), targets.cpu(), ids.cpu().long()

    def value(weights):
        a, b, (w, bias) = weights[:n], weights[n:2 * n], weights[2 * n:]
        y, _, _ = ref.layer_norm(h, w, bias, 1e-5)[0]
        delta = torch.stack([((y * keep) @ a[i]) @ b[i] for i in range(n)])[where, torch.arange(T)]
        z = (h + y @ dense.t() + delta) @ head.t()
        live = goal >= 0
        return float((torch.logsumexp(z[live], 1) - z[live, goal[live]]).mean())

    assert abs(float(loss) - value(weights)) <= 6 * 2.0 ** -8 * value(weights)
    cpu = torch.Generator().manual_seed(2)
    for k, grad in enumerate(block.grad + block.norm_grad):
        g = grad.cpu().double()
        e = torch.randn(g.shape, generator=cpu, dtype=torch.float64)
        e = e / e.norm() + g / g.norm()   # (a direction in which the loss moves)
        step = 1e-4
        up, down = [value([w + (s * step * e if i == k else 0) for i, w in enumerate(weights)]) for s in (1, -1)]
        slope = (up - down) / (2 * step)
        assert abs(slope - float((g * e).sum())) <= 8 * 2.0 ** -8 * float(g.norm() * e.norm()), k


def test_the_example_runs_and_repeats():
    train = _example().train
    one = train(steps=4, T=200, log=None)
    assert len(one) == 4 and all(0 <= x < 30 for x in one) and one == train(steps=4, T=200, log=None)


def test_a_captured_step_of_a_block(salr):
    """Norm, dropout with its seed on the device, and adapters, forward and backward, in one graph that is replayed."""
    T, K, N = 160, 320, 488
    gen = torch.Generator(device="cuda").manual_seed(8)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(torch.bfloat16)   # noqa: E731
    a, b = [normal(K, r) / K ** 0.5 for r in (4, 16)], [normal(r, N) for r in (4, 16)]
    adapters = salr.AdapterSet(a, b, [torch.empty_like(t) for t in a], [torch.empty_like(t) for t in b])
    h, add, dy, w = normal(T, K), normal(T, K), normal(T, N), torch.ones(K, device="cuda")
    ids, seed = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.tensor([1], device="cuda")
    y, total, xd, out, dx = (torch.empty_like(t) for t in (h, h, h, dy, h))
    mean, rstd, dw = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(K, device="cuda")
    need = max(adapters.workspace_bytes(T), adapters.backward_workspace_bytes(T), salr.salr_layer_norm_backward_workspace_bytes(T, K, True))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        salr.salr_layer_norm(h, add, w, None, 1e-5, y, total, mean, rstd)
        salr.salr_dropout(y, None, 0.1, seed, 3, xd)
        adapters.add(xd, ids, None, out=out, workspace=ws)
        adapters.backward(dy, xd, ids, None, dx=dx, workspace=ws)
        salr.salr_dropout(dx, None, 0.1, seed, 3, dx)
        salr.salr_layer_norm_backward(dx, total, w, mean, rstd, None, dx, dw, None, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    outputs = [y, total, xd, out, dx, dw, *adapters.da, *adapters.db]
    for i in range(4):
        seed.fill_(50 + i)
        ids.copy_(torch.randint(-1, 2, (T,), device="cuda", generator=gen))
        h.normal_(generator=gen)
        graph.replay()
        got = [t.clone() for t in outputs]
        torch.cuda.synchronize()
        step()
        assert all(torch.equal(p, q) for p, q in zip(got, outputs)), i


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="one GPU only")
def test_on_a_gpu_that_is_not_current(salr):
    def run(d):
        gen = torch.Generator().manual_seed(1)
        x, r = (torch.randn(30, 64, generator=gen).bfloat16().to(d) for _ in range(2))
        w = torch.ones(64, device=d)
        y, total, mean, rstd = salr.layer_norm(x, w, residual=r)
        dx, dw, _ = salr.layer_norm_backward(y, total, w, mean, rstd, need_dw=True)
        a, b = torch.randn(64, 8, generator=gen).bfloat16().to(d), torch.randn(8, 96, generator=gen).bfloat16().to(d)
        adapters = salr.AdapterSet([a], [b], [torch.empty_like(a)], [torch.empty_like(b)])
        ids = torch.zeros(30, dtype=torch.int32, device=d)
        out = adapters.add(salr.dropout(y, 0.3, 4), ids)
        back = adapters.backward(out, y, ids)[0]
        torch.cuda.synchronize(d)
        return [t.cpu() for t in (y, total, mean, rstd, dx, dw, out, back, *adapters.da, *adapters.db)]
    here, there = run("cuda:0"), run("cuda:1")
    assert all(torch.equal(p, q) for p, q in zip(here, there))
    x = torch.ones(8, 8, device="cuda:0")
    for call in (lambda: salr.dropout(x, 0.1, 1, residual=x.to("cuda:1")), lambda: salr.layer_norm(x, torch.ones(8, device="cuda:1"))):
        with pytest.raises(ValueError, match="different devices"):
            call()
    with pytest.raises(ValueError, match="another device"):
        salr.dropout(x, 0.1, 1, stream=torch.cuda.Stream("cuda:1"))
