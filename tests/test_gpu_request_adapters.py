"""GPU tests of the adapters of many requests, forward and backward, against 64 bits (tests/beside_ref.py derives the tolerances)."""
import pytest
import torch

import beside_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    return salr


RANKS = [16, 1, 13, 64, 0, 8, 33, 4]


def _ids(kind, T, n, gen):
    if kind == "one":
        return torch.full((T,), n - 1, dtype=torch.int32)
    if kind == "none":
        return torch.full((T,), -1, dtype=torch.int32)
    if kind == "mixed":   # with tokens of no adapter, and of ids that are none
        ids = torch.randint(-2, n, (T,), generator=gen, dtype=torch.int32)
        if T > 4:
            ids[T // 2], ids[T // 3] = n, 2 ** 31 - 1
            ids[T // 4] = -2 ** 31
        return ids
    cuts = torch.sort(torch.randint(-1, n, (T,), generator=gen, dtype=torch.int32)).values   # "prompts": one request behind the other
    return cuts


def _made(T, K, N, ranks, kind, seed=0):
    gen = torch.Generator().manual_seed(seed + 31 * T + K + N)
    normal = lambda *shape: torch.randn(*shape, generator=gen).to(torch.bfloat16)   # noqa: E731
    n = len(ranks)
    return {"x": normal(T, K), "dy": normal(T, N), "base": normal(T, N), "dx_base": normal(T, K), "ids": _ids(kind, T, n, gen),
            "a": [(torch.randn(K, r, generator=gen) / K ** 0.5).to(torch.bfloat16) for r in ranks], "b": [normal(r, N) for r in ranks]}


def _dev(s, *names):
    return [[t.to(dev()) for t in s[k]] if isinstance(s[k], list) else s[k].to(dev()) for k in names]


def _set(salr, s, train=False):
    a, b = _dev(s, "a", "b")
    return salr.AdapterSet(a, b, *([[torch.full_like(t, 9.0) for t in l] for l in (a, b)] if train else []))


SIZES = [(1, 64, 96), (1, 4096, 4096), (2, 33, 8), (5, 8, 65), (3, 9, 11), (16, 512, 256), (17, 2720, 2731), (63, 100, 517), (64, 1030, 1024), (65, 64, 64), (127, 48, 1000), (128, 300, 72), (129, 40, 520), (130, 261, 300),
         (300, 2720, 2731), (1000, 96, 4099), (700, 1600, 40)]


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("kind", ["one", "mixed", "prompts", "none"])
def test_add(salr, T, K, N, kind):
    s = _made(T, K, N, RANKS, kind)
    x, ids, base = _dev(s, "x", "ids", "base")
    adapters = _set(salr, s)
    want, tol = ref.adapters(s["x"], s["ids"], s["a"], s["b"], s["base"])
    got = adapters.add(x, ids, base)
    ref.close(got, want, tol, torch.bfloat16)
    assert torch.equal(base.cpu(), s["base"])
    without = s["ids"] < 0
    assert torch.equal(got.cpu()[without], s["base"][without])
    again = base.clone()
    assert adapters.add(x, ids, again, out=again) is again
    assert torch.equal(again.view(torch.int16), got.view(torch.int16))
    want, tol = ref.adapters(s["x"], s["ids"], s["a"], s["b"], None)
    ref.close(adapters.add(x, ids), want, tol, torch.bfloat16)


@pytest.mark.parametrize("ranks", [[256], [100, 7], [128, 65, 17], [0], [0, 3], [2] * 70, [16] * 130])
@pytest.mark.parametrize("T", [3, 40, 200])
def test_ranks_and_counts(salr, ranks, T):
    s = _made(T, 544, 203, ranks, "mixed")
    want, tol = ref.adapters(s["x"], s["ids"], s["a"], s["b"], s["base"])
    ref.close(_set(salr, s).add(*_dev(s, "x", "ids", "base")), want, tol, torch.bfloat16)
    _backward(salr, s)


@pytest.mark.parametrize("ranks", [[16], [13, 5], [32], [31, 20], [64], [61, 4], [128, 9]])
@pytest.mark.parametrize("T,K,N", [(1, 1031, 96), (7, 517, 331), (100, 264, 1031), (150, 517, 331), (150, 1031, 96), (150, 1024, 331)])
def test_lengths_and_ranks(salr, T, K, N, ranks):
    """Every form of the products (how many tokens, the largest rank of the set) with lengths and ranks of whole vectors and of others."""
    s = _made(T, K, N, ranks, "prompts", 14)
    s["ids"][0] = 0
    want, tol = ref.adapters(s["x"], s["ids"], s["a"], s["b"], s["base"])
    ref.close(_set(salr, s).add(*_dev(s, "x", "ids", "base")), want, tol, torch.bfloat16)
    _backward(salr, s)


def _backward(salr, s, with_base=True):
    x, dy, ids, dx_base = _dev(s, "x", "dy", "ids", "dx_base")
    adapters = _set(salr, s, train=True)
    (want, tol), da, db = ref.adapters_backward(s["dy"], s["x"], s["ids"], s["a"], s["b"], s["dx_base"] if with_base else None)
    dx, got_a, got_b = adapters.backward(dy, x, ids, dx_base if with_base else None)
    ref.close(dx, want, tol, torch.bfloat16)
    for got, (w, t) in zip(got_a + got_b, da + db):
        ref.close(got, w, t, torch.bfloat16)
    return adapters, dx, [t.clone() for t in got_a + got_b]


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("kind", ["one", "mixed", "prompts", "none"])
def test_backward(salr, T, K, N, kind):
    s = _made(T, K, N, RANKS, kind, 3)
    adapters, dx, grads = _backward(salr, s)
    x, dy, ids, dx_base = _dev(s, "x", "dy", "ids", "dx_base")
    # in place, without the gradients, and only they
    place = dx_base.clone()
    got, da, db = adapters.backward(dy, None, ids, place, dx=place, need_gradients=False)
    assert da is None and db is None and torch.equal(got.view(torch.int16), dx.view(torch.int16)) and got.data_ptr() == place.data_ptr()
    for t in adapters.da + adapters.db:
        t.fill_(5.0)
    assert adapters.backward(dy, x, ids, need_dx=False)[0] is None
    assert all(torch.equal(a, b) for a, b in zip(adapters.da + adapters.db, grads))
    _backward(salr, s, with_base=False)


@pytest.mark.parametrize("T,K,N,ranks", [(257, 64, 96, [16]), (1030, 40, 72, [13, 4]), (2100, 136, 60, [33]), (2600, 100, 4000, [8, 16, 5]), (5000, 264, 1160, [64, 1]), (9000, 72, 640, [4] * 100)])
def test_many_tokens_of_one_adapter(salr, T, K, N, ranks):
    """Gradients whose sums are joined: chunks that are full, all but empty, and an adapter beside them that has one."""
    s = _made(T, K, N, ranks, "one", 11)
    s["ids"][: T // 20] = 0
    s["ids"][T // 3] = -1
    _, dx, grads = _backward(salr, s)
    _, dx2, again = _backward(salr, s)
    assert torch.equal(dx, dx2) and all(torch.equal(p, q) for p, q in zip(grads, again))
    x, dy, ids, dx_base = _dev(s, "x", "dy", "ids", "dx_base")
    a, b = _dev(s, "a", "b")
    only = [torch.empty_like(t) for t in b]
    salr.AdapterSet(a, b, None, only).backward(dy, x, ids)
    assert all(torch.equal(p, q) for p, q in zip(only, grads[len(a):]))


def test_adjoint(salr):
    """(x A) B is linear in x, in A and in B: <dy, y> is <dx, x>, <dA, A> and <dB, B>, as differences along each of them would be."""
    s = _made(150, 320, 512, [16, 13, 64], "prompts", 8)
    (dx, dx_tol), da, db = ref.adapters_backward(s["dy"], s["x"], s["ids"], s["a"], s["b"], None)
    y_tol = ref.adapters(s["x"], s["ids"], s["a"], s["b"], None)[1]
    y = _set(salr, s).add(*_dev(s, "x", "ids")).cpu().double()
    adapters, got_dx, grads = _backward(salr, s, with_base=False)
    step = ref.half(torch.bfloat16) * 1.01
    dyd, xd = s["dy"].double(), s["x"].double()
    left, room = float((dyd * y).sum()), float((dyd.abs() * (y_tol + step * y.abs())).sum())
    for got, tol, at in ((got_dx.cpu().double(), dx_tol, xd), (torch.cat([t.cpu().double().reshape(-1) for t in grads[:3]]),
                         torch.cat([t.reshape(-1) for _, t in da]), torch.cat([t.double().reshape(-1) for t in s["a"]])),
                         (torch.cat([t.cpu().double().reshape(-1) for t in grads[3:]]), torch.cat([t.reshape(-1) for _, t in db]),
                          torch.cat([t.double().reshape(-1) for t in s["b"]]))):
        assert abs(float((got * at).sum()) - left) <= room + float((at.abs() * (tol + step * got.abs())).sum())


def test_tokens_and_adapters_do_not_touch_each_other(salr):
    """NaN and infinities of one token, or of one adapter, stay with its own; an infinity in x is not NaN where the formula has none."""
    for T in (40, 100, 200):
        s = _made(T, 96, 130, [5, 16, 20], "mixed", 2)
        s["ids"] = torch.arange(T, dtype=torch.int32) % 4 - 1
        x, ids, base, dy = _dev(s, "x", "ids", "base", "dy")
        clean_set, clean_dx, clean_grads = _backward(salr, s)
        clean = clean_set.add(x, ids, base)
        bad = x.clone()
        bad[8] = float("nan")             # without an adapter
        bad[9] = float("nan")             # adapter 0
        bad[10, 4] = float("inf")         # adapter 1
        got = clean_set.add(bad, ids, base)
        others = [t for t in range(T) if t not in (9, 10)]
        assert torch.equal(got[others], clean[others]) and bool(torch.isnan(got[9]).all())
        t = s["a"][1][4].double() * float("inf")
        assert torch.equal(torch.isnan(got[10].cpu()), torch.isnan((t[:, None] * s["b"][1].double()).sum(0)))
        clean_set.backward(dy, bad, ids)
        assert torch.equal(clean_set.da[2], clean_grads[2]) and torch.equal(clean_set.db[2], clean_grads[5])
        assert bool(torch.isnan(clean_set.da[0]).all()) and bool(torch.isnan(clean_set.db[0]).all())
        a, b = _dev(s, "a", "b")
        a[2][:, 19], b[2][3] = float("inf"), float("nan")
        got = salr.AdapterSet(a, b).add(x, ids, base)
        others = [t for t in range(T) if s["ids"][t] != 2]
        assert torch.equal(got[others], clean[others])
        bad_dy = dy.clone()
        bad_dy[8], bad_dy[11] = float("nan"), float("nan")   # no adapter; adapter 2
        dx, _, _ = clean_set.backward(bad_dy, x, ids, s["dx_base"].to(dev()))
        others = [t for t in range(T) if t != 11]
        assert torch.equal(dx[others], clean_dx[others])
        assert torch.equal(clean_set.da[1], clean_grads[1]) and torch.equal(clean_set.db[1], clean_grads[4])


def test_a_token_does_not_depend_on_the_others(salr):
    """The same sizes, other fellows: the same bits."""
    for T in (60, 120, 500):
        s = _made(T, 500, 300, RANKS, "mixed", 6)
        adapters = _set(salr, s)
        x, ids, base = _dev(s, "x", "ids", "base")
        one = adapters.add(x, ids, base)
        turn = torch.randperm(T, generator=torch.Generator().manual_seed(1)).to(dev())
        two = adapters.add(x[turn].contiguous(), ids[turn].contiguous(), base[turn].contiguous())
        assert torch.equal(one[turn].view(torch.int16), two.view(torch.int16))


def test_neighbours_stay(salr):
    """Outputs at element addresses inside larger buffers, gradients between guards."""
    for T in (7, 90):
        s = _made(T, 65, 67, [3, 17], "mixed", 4)
        x, ids, base, dy, dx_base = _dev(s, "x", "ids", "base", "dy", "dx_base")
        want = _set(salr, s).add(x, ids, base)
        buf = torch.full((T * 67 + 40,), 3.0, dtype=torch.bfloat16, device=dev())
        out = buf[5:5 + T * 67].view(T, 67)
        _set(salr, s).add(x, ids, base, out=out)
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and bool((buf[:5] == 3).all()) and bool((buf[5 + T * 67:] == 3).all())
        a, b = _dev(s, "a", "b")
        whole = torch.full((20000,), 3.0, dtype=torch.bfloat16, device=dev())
        used, places, at = torch.zeros(20000, dtype=torch.bool, device=dev()), [], 8
        for t in a + b:
            places.append(whole[at:at + t.numel()].view(t.shape))
            used[at:at + t.numel()] = True
            at += (t.numel() + 15) // 8 * 8
        salr.AdapterSet(a, b, places[:2], places[2:]).backward(dy, x, ids, dx_base)
        _, _, grads = _backward(salr, s)
        assert all(torch.equal(p, g) for p, g in zip(places, grads)) and bool((whole[~used] == 3).all())


def test_frozen_pairs_and_one_factor(salr):
    s = _made(100, 128, 160, [8, 16, 24], "prompts", 5)
    x, dy, ids, dx_base = _dev(s, "x", "dy", "ids", "dx_base")
    _, dx, grads = _backward(salr, s)
    a, b = _dev(s, "a", "b")
    da, db = [None, torch.empty_like(a[1]), None], [torch.empty_like(b[0]), None, None]
    got, _, _ = salr.AdapterSet(a, b, da, db).backward(dy, x, ids, dx_base)
    assert torch.equal(got, dx) and torch.equal(da[1], grads[1]) and torch.equal(db[0], grads[3])
    only = [torch.empty_like(t) for t in b]
    salr.AdapterSet(a, b, None, only).backward(dy, x, ids)
    assert all(torch.equal(p, g) for p, g in zip(only, grads[3:]))


def test_no_tokens(salr):
    s = _made(0, 64, 96, [4, 16], "mixed")
    adapters, dx, grads = _backward(salr, s)
    assert dx.shape == (0, 64) and all(bool((g == 0).all()) for g in grads)
    assert adapters.add(*_dev(s, "x", "ids", "base")).shape == (0, 96)


@pytest.mark.parametrize("T", [20, 110, 300])
def test_captured(salr, T):
    """Ids and inputs change between the replays; what is left in the workspace does not matter."""
    s = _made(T, 416, 600, RANKS, "mixed", 7)
    x, ids, base, dy, dx_base = _dev(s, "x", "ids", "base", "dy", "dx_base")
    adapters = _set(salr, s, train=True)
    ws = torch.empty(max(adapters.workspace_bytes(T), adapters.backward_workspace_bytes(T)), dtype=torch.uint8, device=dev())
    y, dx = torch.empty_like(base), torch.empty_like(x)

    def step():
        adapters.add(x, ids, base, out=y, workspace=ws)
        adapters.backward(dy, x, ids, dx_base, dx=dx, workspace=ws)
        return [t.clone() for t in (y, dx, *adapters.da, *adapters.db)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        adapters.add(x, ids, base, out=y, workspace=ws)
        adapters.backward(dy, x, ids, dx_base, dx=dx, workspace=ws)
    gen = torch.Generator().manual_seed(4)
    for i in range(4):
        ids.copy_(_ids(["prompts", "mixed", "one", "none"][i], T, len(RANKS), gen))
        x.copy_(torch.randn(T, 416, generator=gen))
        ws.fill_(255)
        graph.replay()
        got = [t.clone() for t in (y, dx, *adapters.da, *adapters.db)]
        ws.fill_(127)
        want = step()
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, want)), i
        torch.cuda.synchronize()


def test_streams(salr):
    s = _made(500, 1024, 1200, RANKS, "prompts", 9)
    x, ids, base, dy, dx_base = _dev(s, "x", "ids", "base", "dy", "dx_base")
    adapters, dx, grads = _backward(salr, s)
    y = adapters.add(x, ids, base)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y2 = adapters.add(x, ids, base, stream=side)
    dx2, da, db = adapters.backward(dy, x, ids, dx_base, stream=side)
    side.synchronize()
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and all(torch.equal(p, g) for p, g in zip(da + db, grads))
    # two calls at once, a workspace each (allocated)
    other = torch.cuda.Stream()
    y3, y4 = adapters.add(x, ids, base, stream=side), adapters.add(x, ids, base, stream=other)
    side.synchronize()
    other.synchronize()
    assert torch.equal(y, y3) and torch.equal(y, y4)


def test_far_rows(salr):
    """Rows behind 2^31 elements."""
    T, K, N = 600_000, 8, 4100
    a, b = [torch.randn(K, 2, device=dev()).bfloat16()], [torch.randn(2, N, device=dev()).bfloat16()]
    x = torch.randn(T, K, device=dev()).bfloat16()
    ids = torch.full((T,), -1, dtype=torch.int32, device=dev())
    rows = [0, 300_000, 524_287, 524_288, 599_999]
    ids[rows] = 0
    adapters = salr.AdapterSet(a, b)
    y = adapters.add(x, ids)
    want, tol = ref.adapters(x[rows].cpu(), torch.zeros(5, dtype=torch.int32), [a[0].cpu()], [b[0].cpu()], None)
    ref.close(y[rows], want, tol, torch.bfloat16)
    y[rows] = 0
    assert not bool(y.any())


def test_values_may_change_but_not_places(salr):
    s = _made(10, 64, 64, [8, 8], "mixed")
    x, ids, base = _dev(s, "x", "ids", "base")
    a, b = _dev(s, "a", "b")
    adapters = salr.AdapterSet(a, b, [torch.zeros_like(t) for t in a], [torch.zeros_like(t) for t in b])
    a[0].mul_(2)
    s["a"][0] = s["a"][0] * 2
    want, tol = ref.adapters(s["x"], s["ids"], s["a"], s["b"], s["base"])
    ref.close(adapters.add(x, ids, base), want, tol, torch.bfloat16)
    version = adapters.da[0]._version
    adapters.backward(s["dy"].to(dev()), x, ids)
    assert adapters.da[0]._version > version
    a[0].data = a[0].clone()
    with pytest.raises(ValueError):
        adapters.add(x, ids, base)


def test_refusals(salr):
    s = _made(6, 64, 96, [4, 8], "mixed")
    x, ids, base, dy, a, b = _dev(s, "x", "ids", "base", "dy", "a", "b")
    adapters = salr.AdapterSet(a, b)
    for bad in (dict(x=x.float()), dict(x=None), dict(x=x.cpu()), dict(ids=ids.long()), dict(ids=ids.cpu()), dict(base=base.float())):
        with pytest.raises(TypeError):
            adapters.add(**{"x": x, "ids": ids, "base": base, **bad})
    for bad in (dict(x=x[:5]), dict(x=x[:, :32].contiguous()), dict(ids=ids[:5]), dict(ids=None), dict(base=base[:, :32].contiguous()), dict(out=x)):
        with pytest.raises(ValueError):
            adapters.add(**{"x": x, "ids": ids, "base": base, **bad})
    with pytest.raises(salr.SalrError):
        adapters.add(x, ids, base, workspace=torch.empty(16, dtype=torch.uint8, device=dev()))
    with pytest.raises(ValueError):
        adapters.backward(dy, x, ids)
    for args in (([], []), (a, b[:1]), (a[0], b[0]), ([a[0]], [b[1]]), ([a[0], a[1][:32].contiguous()], b)):
        with pytest.raises((ValueError, TypeError)):
            salr.AdapterSet(*args)
    with pytest.raises(TypeError):
        salr.AdapterSet([t.float() for t in a], b)
    with pytest.raises(TypeError):
        salr.AdapterSet([a[0].t().contiguous().t(), a[1]], b)
    with pytest.raises(ValueError):   # gradients in the same memory
        salr.AdapterSet(a, b, [a[0], torch.empty_like(a[1])])
    g = torch.empty_like(a[0])
    with pytest.raises(ValueError):
        salr.AdapterSet([a[0], a[0]], [b[0], b[0]], [g, g])
    with pytest.raises(salr.SalrError):   # fewer than eight features
        salr.AdapterSet([a[0][:7].contiguous()], [b[0]])
    with pytest.raises(salr.SalrError):   # a rank above 256
        salr.AdapterSet([torch.zeros(64, 257, dtype=torch.bfloat16, device=dev())], [torch.zeros(257, 64, dtype=torch.bfloat16, device=dev())])
    square = salr.AdapterSet([torch.zeros(64, 4, dtype=torch.bfloat16, device=dev())], [torch.zeros(4, 64, dtype=torch.bfloat16, device=dev())])
    buf = torch.zeros(10, 64, dtype=torch.bfloat16, device=dev())
    with pytest.raises(salr.SalrError):
        square.add(buf[:6], ids, out=buf[:6])
    with pytest.raises(salr.SalrError):
        square.add(x, ids, buf[:6], out=buf[2:8])
