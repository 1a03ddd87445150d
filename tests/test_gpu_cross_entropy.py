"""GPU tests of salr_linear_cross_entropy against a plain 64-bit implementation.

Tolerances, from the number formats (u = 2^-24, the rounding of fp32; bf16 has 8 significant bits and rounds to 2^-8):
  logit   K products summed in fp32: |dl| <= (K + 8) u sum_k |h_k w_k|, L the largest of a token's; lse and loss move by at most that each,
          and by a few roundings of their own and of the vocabulary's sum: L (twice for the loss) + (16 + tiles) u (1 + |lse| + |l|)
  dh      G is off by a factor 1 + 2 L + 2^-8 (its rounding to bf16), the sum over the vocabulary by (V + 8) u, the result is rounded
          to bf16.  Where dw is not asked for, the target's own part is no rounded operand.
  dw      the same with the sum over the tokens
"""
import pytest
import torch

import finetune_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _inputs(T, K, V, seed, std_w=0.1, sure=16.0, masked=True):
    gen = torch.Generator().manual_seed(seed)
    w = (torch.randn(V, K, generator=gen) * std_w).bfloat16()
    t = torch.randint(0, V, (T,), generator=gen)
    lift = torch.rand(T, 1, generator=gen) * sure / (std_w * std_w * K)
    h = (torch.randn(T, K, generator=gen) + w[t].float() * lift).bfloat16()
    if masked and T > 1:
        t[1::4] = -100
        h[1::4] = float("nan")
        h[1::8] = float("inf")
    g = torch.rand(T, generator=gen) * 2 - 0.5
    return h, w, t, g


def _run(h, w, t, g, need_dh, need_dw, workspace=None):
    import paper_2601_16991_amd as salr
    got = salr.linear_cross_entropy(h.to(dev()), w.to(dev()), t.to(dev()), None if g is None else g.to(dev()), need_dh=need_dh, need_dw=need_dw,
                                    workspace=workspace)
    torch.cuda.synchronize()
    return [None if x is None else x.cpu() for x in got]


def _check(h, w, t, g, got, need_dh, need_dw):
    T, K = h.shape
    V = w.shape[0]
    loss, lse, dh, dw, G = ref.cross_entropy(h, w, t, torch.ones(T) if g is None else g)
    live = t >= 0
    x = torch.where(live[:, None], h.double(), 0.0)
    L = (K + 8) * U * (x.abs() @ w.double().abs().t()).amax(1)
    own = (16 + (V + 255) // 256) * U * (2 + lse.abs() + (lse - loss).abs())
    assert got[0].dtype == got[1].dtype == torch.float32
    assert ((got[1].double() - lse).abs() <= L + own).all()
    assert ((got[0].double() - loss).abs() <= 2 * L + own).all()
    assert (got[0][~live] == 0).all() and (got[1][~live] == 0).all()
    assert (got[2] is not None) == need_dh and (got[3] is not None) == need_dw
    A = G.abs()
    if need_dh:
        factor = (2 * L + (V + 8) * U)[:, None]
        rounded = A.clone()
        if not need_dw:
            rounded.scatter_(1, t.clamp(min=0)[:, None], 0.0)
        tol = factor * (A @ w.double().abs()) + 2.0 ** -8 * (rounded @ w.double().abs()) + 2.0 ** -8 * dh.abs() + 1e-36
        assert got[2].dtype == torch.bfloat16
        assert ((got[2].double() - dh).abs() <= tol).all()
        assert (got[2][~live] == 0).all()
    if need_dw:
        factor = (2 * L + (T + 8) * U + 2.0 ** -8)[:, None]
        tol = (A * factor).t() @ x.abs() + 2.0 ** -8 * dw.abs() + 1e-36
        assert ((got[3].double() - dw).abs() <= tol).all()


@pytest.mark.parametrize("need_dh,need_dw", [(False, False), (True, False), (True, True), (False, True)])
@pytest.mark.parametrize("T,K,V", [
    (1, 8, 1), (1, 64, 256), (2, 24, 255), (15, 72, 257), (16, 512, 4099), (17, 128, 1000), (31, 200, 513), (33, 64, 5000), (64, 136, 1031),
    (65, 256, 300), (128, 1000, 777), (129, 64, 2049), (255, 96, 3001), (257, 512, 1537), (300, 2720, 2731), (513, 320, 5003),
])
def test_against_64_bits(T, K, V, need_dh, need_dw):
    h, w, t, g = _inputs(T, K, V, 1000 * T + V)
    print(f"[ce] T{T} K{K} V{V} {need_dh} {need_dw}", flush=True)
    _check(h, w, t, g, _run(h, w, t, g, need_dh, need_dw), need_dh, need_dw)


@pytest.mark.parametrize("need_dw", [False, True])
def test_several_pieces_of_the_vocabulary(need_dw):
    """The running maximum grows from piece to piece and falls behind in others."""
    T, K, V = 520, 64, 70001
    h, w, t, g = _inputs(T, K, V, 5)
    w[:, 0] = (torch.arange(V) // 9000 % 3 - 1).bfloat16() * 8   # pieces with logits far up or down
    h[0::4, 0] = 6.0
    h[2::4, 0] = -6.0
    _check(h, w, t, g, _run(h, w, t, g, True, need_dw), True, need_dw)


@pytest.mark.parametrize("need_dw", [False, True])
@pytest.mark.parametrize("T,V", [(2100, 70001), (5000, 30011)])
def test_more_logits_than_a_piece_holds(T, V, need_dw):
    """More than 128 M logits: two pieces, the running maximum a step up in the second for some tokens and in the first for others."""
    import paper_2601_16991_amd as salr
    K = 32
    assert T * V > 1 << 27
    h, w, t, g = _inputs(T, K, V, 23)
    w[:, 0] = 0.0
    w[: V // 7, 0] = 60.0
    w[-V // 9:, 0] = -60.0
    h[0::4, 0] = 1.0
    h[2::4, 0] = -1.0
    h[1::4, 0] = 0.0
    h[3::4, 0] = 0.25
    h, w, t, g = [x.to(dev()) for x in (h, w, t, g)]
    got = salr.linear_cross_entropy(h, w, t, g, need_dh=True, need_dw=need_dw)
    _check(h, w, t, g, got, True, need_dw)


@pytest.mark.parametrize("T", [1, 40, 300])
def test_no_gradient_of_the_loss_means_ones(T):
    h, w, t, _ = _inputs(T, 64, 900, 3)
    _check(h, w, t, None, _run(h, w, t, None, True, True), True, True)


def test_all_tokens_masked():
    h, w, t, g = _inputs(70, 64, 900, 4)
    t[:] = -1
    h[:] = float("nan")
    for need_dw in (False, True):
        for x in _run(h, w, t, g, True, need_dw):
            assert x is None or (x == 0).all()


@pytest.mark.parametrize("shift", [-3000.0, 3000.0, 60000.0])
def test_logits_far_from_zero(shift):
    """A common shift of a token's logits changes nothing but lse."""
    T, K, V = 40, 64, 1300
    h, w, t, g = _inputs(T, K, V, 6, masked=False)
    h[:, 0] = 1.0
    w[:, 0] = shift
    _check(h, w, t, g, _run(h, w, t, g, True, False), True, False)
    _check(h, w, t, g, _run(h, w, t, g, True, True), True, True)


@pytest.mark.parametrize("logit", [-500.0, -90.0, 0.0, 90.0, 500.0, 2.0 ** 20])
def test_a_vocabulary_of_one_word(logit):
    T, K = 20, 8
    h, w = torch.zeros(T, K).bfloat16(), torch.zeros(1, K).bfloat16()
    h[:, 0], w[:, 0] = 1.0, logit
    t, g = torch.zeros(T, dtype=torch.int64), torch.ones(T)
    _check(h, w, t, g, _run(h, w, t, g, True, False), True, False)
    _check(h, w, t, g, _run(h, w, t, g, True, True), True, True)


@pytest.mark.parametrize("need_dw", [False, True])
@pytest.mark.parametrize("low,high", [(-62.0, 44.0), (-300.0, 44.0), (-44.0, 100.0), (-1000.0, 1000.0), (-46.0, -43.0), (43.0, 46.0)])
def test_logits_of_a_row_far_apart(low, high, need_dw):
    """Every fifth word at `high`, the others at `low`, in whole tiles and within them; targets of both kinds."""
    T, K, V = 40, 64, 1300
    h, w, t, g = _inputs(T, K, V, 21, masked=False, std_w=0.01, sure=0.0)
    v = torch.arange(V)
    top = torch.where(v < 700, v // 64 % 5 == 1, v % 5 == 1)
    h[:, 0] = 1.0
    w[:, 0] = torch.where(top, high, low).bfloat16()
    t[: T // 2] = torch.nonzero(top)[: T // 2, 0]
    _check(h, w, t, g, _run(h, w, t, g, True, need_dw), True, need_dw)


def test_many_rows_with_references_of_two_kinds():
    """Tokens of which each has one tile far above the others: every E of the rest is brought in line."""
    T, K, V = 300, 64, 5000
    h, w, t, g = _inputs(T, K, V, 22, masked=False, std_w=0.05, sure=0.0)
    w[2000:2100, 0] = 60.0
    h[:, 0] = 1.0
    h[::3, 0] = 0.25
    _check(h, w, t, g, _run(h, w, t, g, True, False), True, False)


def test_well_predicted_tokens_keep_their_gradient():
    """1 - p of 1e-9 and less: the gradient is that small and right to bf16, not the difference of rounded probabilities."""
    T, K, V = 64, 128, 2000
    h, w, t, g = _inputs(T, K, V, 7, masked=False, sure=0.0)
    h = (w[t].float() * 30.0).bfloat16()   # logits of the target about 38, of the others about 0
    loss, _, dh, _, _ = ref.cross_entropy(h, w, t, g)
    assert 0 < loss.max() < 1e-6
    got = _run(h, w, t, g, True, False)
    _check(h, w, t, g, got, True, False)
    assert ((got[0].double() - loss).abs() <= 1e-3 * loss).all()
    assert (got[2].double() - dh).norm() <= 5e-3 * dh.norm()


@pytest.mark.parametrize("T", [3, 200])
def test_minus_infinite_logits_and_their_targets(T):
    """A row of the head that pushes its logit to -infinity: probability 0, and a token that wants it has an infinite loss or NaN."""
    K, V = 64, 700
    h, w, t, g = _inputs(T, K, V, 8, masked=False)
    h = h.abs() + 1
    w[5] = -3e38
    w[300] = -3e38
    t[t == 5] = 6
    t[t == 300] = 6
    loss, lse, _, _, _ = ref.cross_entropy(h, w.float().clamp(min=-1e30), t, g)
    got = _run(h, w, t, g, True, False)
    assert torch.isfinite(got[0]).all() and torch.isfinite(got[1]).all() and torch.isfinite(got[2].float()).all()
    assert (got[0].double() - loss).abs().max() < 1e-3 and (got[1].double() - lse).abs().max() < 1e-3


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("T", [5, 90, 400])
def test_not_finite_values_stay_in_their_token(T, bad):
    K, V = 64, 900
    h, w, t, g = _inputs(T, K, V, 9)
    w[:, 3] = w[:, 3].abs() + 0.01
    clean = _run(h, w, t, g, True, False)
    h2 = h.clone()
    h2[2, 3] = bad
    got = _run(h2, w, t, g, True, False)
    rest = torch.arange(T) != 2
    for a, b in zip(got, clean):
        if a is not None:
            assert torch.isnan(a[2].float()).all()
            assert torch.equal(a[rest], b[rest])


def test_target_past_the_vocabulary():
    T, K, V = 70, 64, 900
    h, w, t, g = _inputs(T, K, V, 10)
    clean = _run(h, w, t, g, True, False)
    t[4] = V
    t[6] = 2 ** 40
    got = _run(h, w, t, g, True, False)
    rest = (torch.arange(T) != 4) & (torch.arange(T) != 6)
    for a, b in zip(got, clean):
        if a is not None:
            assert torch.isnan(a[4].float()).all() and torch.isnan(a[6].float()).all()
            assert torch.equal(a[rest], b[rest])


@pytest.mark.parametrize("T,K,V,need_dw", [(20, 64, 900, False), (300, 256, 5003, False), (300, 256, 5003, True)])
def test_same_bits_whatever_the_workspace_held(T, K, V, need_dw):
    import paper_2601_16991_amd as salr
    h, w, t, g = _inputs(T, K, V, 11)
    first = _run(h, w, t, g, True, need_dw)
    need = salr.salr_linear_cross_entropy_workspace_bytes(T, K, V, True, need_dw)
    for fill in (0, 255):
        ws = torch.full((need,), fill, dtype=torch.uint8, device=dev())
        for a, b in zip(_run(h, w, t, g, True, need_dw, ws), first):
            assert a is None or torch.equal(a, b)


def test_gradient_against_differences():
    """(loss(h + d) - loss(h - d)) / 2 along d, in fp32 from the kernel itself.  h and d on a grid of 2^-6 below 2, so that both sums are
    exact in bf16.  Third order: a logit moves by a = max |d w| (in 64 bits), the loss's third derivative is at most 2 a^3: / 6.  The
    losses' own error enters over 2, twice."""
    T, K, V = 64, 64, 500
    gen = torch.Generator().manual_seed(12)
    h = (torch.randint(-64, 65, (T, K), generator=gen) / 64.0).bfloat16()
    w = (torch.randn(V, K, generator=gen) * 0.3).bfloat16()
    t = torch.randint(0, V, (T,), generator=gen)
    d = (torch.randint(0, 2, (T, K), generator=gen) * 2 - 1) / 64.0
    up, down = (h.float() + d).bfloat16(), (h.float() - d).bfloat16()
    assert torch.equal(up.float() - h.float(), d) and torch.equal(h.float() - down.float(), d)
    slope = (_run(up, w, t, None, False, False)[0].double() - _run(down, w, t, None, False, False)[0].double()) / 2
    dh = _run(h, w, t, None, True, False)[2].double()
    along = (dh * d.double()).sum(1)
    a = (d.double() @ w.double().t()).abs().amax(1)
    L = (K + 8) * U * (up.double().abs() @ w.double().abs().t()).amax(1)
    G = ref.cross_entropy(h, w, t, torch.ones(T))[4].abs()
    tol = a ** 3 / 3 + 2 * L + 64 * U * 16 + 2.0 ** -8 * ((G @ w.double().abs()) * d.abs().double()).sum(1)
    assert ((slope - along).abs() <= tol).all()
    assert tol.median() < 0.3 * along.abs().median()


def test_head_gradient_against_differences():
    """The same for dw: along one direction of the whole head."""
    T, K, V = 32, 64, 300
    gen = torch.Generator().manual_seed(13)
    h = torch.randn(T, K, generator=gen).bfloat16()
    w = (torch.randint(-64, 65, (V, K), generator=gen) / 128.0).bfloat16()
    t = torch.randint(0, V, (T,), generator=gen)
    d = (torch.randint(0, 2, (V, K), generator=gen) * 2 - 1) / 128.0
    up, down = (w.float() + d).bfloat16(), (w.float() - d).bfloat16()
    assert torch.equal(up.float() - w.float(), d) and torch.equal(w.float() - down.float(), d)
    slope = (_run(h, up, t, None, False, False)[0].double().sum() - _run(h, down, t, None, False, False)[0].double().sum()) / 2
    dw = _run(h, w, t, None, False, True)[3].double()
    a = (h.double() @ d.double().t()).abs().amax(1)
    L = (K + 8) * U * (h.double().abs() @ up.double().abs().t()).amax(1)
    G = ref.cross_entropy(h, w, t, torch.ones(T))[4].abs()
    tol = (a ** 3 / 3 + 2 * L + 64 * U * 16).sum() + 2.0 ** -8 * ((G.t() @ h.double().abs()) * d.abs().double()).sum()
    assert abs(slope - (dw * d.double()).sum()) <= tol


def test_on_another_stream_and_in_a_graph():
    import paper_2601_16991_amd as salr
    T, K, V = 150, 128, 3000
    h, w, t, g = _inputs(T, K, V, 14)
    first = _run(h, w, t, g, True, True)
    d = [x.to(dev()) for x in (h, w, t, g)]
    loss, lse = torch.empty(T, device=dev()), torch.empty(T, device=dev())
    dh, dw = torch.empty_like(d[0]), torch.empty_like(d[1])
    ws = torch.empty(salr.salr_linear_cross_entropy_workspace_bytes(T, K, V, True, True), dtype=torch.uint8, device=dev())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    salr.salr_linear_cross_entropy(*d, loss, lse, dh, dw, ws, stream=side)
    side.synchronize()
    for a, b in zip((loss, lse, dh, dw), first):
        assert torch.equal(a.cpu(), b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        salr.salr_linear_cross_entropy(*d, loss, lse, dh, dw, ws)
    for _ in range(3):
        for x in (loss, lse, dh, dw, ws):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((loss, lse, dh, dw), first):
            assert torch.equal(a.cpu(), b)


def test_offsets_past_32_bits():
    """A head of 5.4 GB: rows whose byte offset passes 2^32 are the ones that count."""
    T, K, V = 3, 8192, 330000
    gen = torch.Generator(device=dev()).manual_seed(15)
    w = torch.empty(V, K, dtype=torch.bfloat16, device=dev()).normal_(0.0, 0.02, generator=gen)
    h = torch.randn(T, K, device=dev(), generator=gen).bfloat16()
    t = torch.tensor([V - 1, 7, V - 200], device=dev())
    import paper_2601_16991_amd as salr
    loss, lse, dh, _ = salr.linear_cross_entropy(h, w, t)
    z = torch.cat([h.double() @ w[i:i + 30000].double().t() for i in range(0, V, 30000)], 1)
    G = torch.softmax(z, 1)
    want = torch.logsumexp(z, 1) - z.gather(1, t[:, None])[:, 0]
    G[torch.arange(T, device=dev()), t] -= 1.0
    dref = sum(G[:, i:i + 30000] @ w[i:i + 30000].double() for i in range(0, V, 30000))
    assert (loss.double() - want).abs().max() < 1e-4
    assert (dh.double() - dref).norm() < 5e-3 * dref.norm()


def test_no_hidden_size():
    """An empty contraction: all logits are 0."""
    import paper_2601_16991_amd as salr
    h, w = torch.empty(5, 0, dtype=torch.bfloat16, device=dev()), torch.empty(700, 0, dtype=torch.bfloat16, device=dev())
    t = torch.tensor([0, 699, -1, 300, 700], device=dev())
    loss, lse, dh, dw = salr.linear_cross_entropy(h, w, t, need_dw=True)
    want = torch.log(torch.tensor(700.0)).item()
    for x in (loss.cpu(), lse.cpu()):
        assert torch.allclose(x[[0, 1, 3]], torch.full((3,), want), rtol=1e-6) and x[2] == 0 and torch.isnan(x[4])
    assert dh.shape == (5, 0) and dw.shape == (700, 0)


@pytest.mark.parametrize("need_dw", [False, True])
def test_more_tokens_than_a_grid_dimension(need_dw):
    T, K, V = 70001, 32, 300
    h, w, t, g = _inputs(T, K, V, 17, std_w=0.3, sure=4.0)
    _check(h, w, t, g, _run(h, w, t, g, True, need_dw), True, need_dw)


def test_no_tokens():
    import paper_2601_16991_amd as salr
    h, w = torch.empty(0, 64, dtype=torch.bfloat16, device=dev()), torch.ones(300, 64, dtype=torch.bfloat16, device=dev())
    t = torch.empty(0, dtype=torch.int64, device=dev())
    loss, lse, dh, dw = salr.linear_cross_entropy(h, w, t, need_dw=True)
    assert loss.shape == lse.shape == (0,) and dh.shape == (0, 64) and (dw == 0).all()


def test_refusals():
    import paper_2601_16991_amd as salr
    h, w, t, g = [x.to(dev()) for x in _inputs(8, 64, 100, 16)]
    with pytest.raises(ValueError):
        salr.linear_cross_entropy(h, w[:, :32].contiguous(), t)
    with pytest.raises(ValueError):
        salr.linear_cross_entropy(h, w, t[:4])
    with pytest.raises(ValueError):
        salr.linear_cross_entropy(h, w, t, g[:4])
    with pytest.raises(TypeError):
        salr.linear_cross_entropy(h.float(), w, t)
    with pytest.raises(TypeError):
        salr.linear_cross_entropy(h, w, t.int())
    with pytest.raises(TypeError):
        salr.linear_cross_entropy(h[:, ::2], w[:, ::2], t)
    with pytest.raises(TypeError):
        salr.linear_cross_entropy(h.cpu(), w, t)
    for bad in (h[:, :60].contiguous(), ):   # K % 8
        with pytest.raises(salr.SalrError) as e:
            salr.linear_cross_entropy(bad, w[:, :60].contiguous(), t)
        assert e.value.status == salr.SALR_ERR_SHAPE
    with pytest.raises(salr.SalrError) as e:
        salr.linear_cross_entropy(h, w, t, workspace=torch.empty(256, dtype=torch.uint8, device=dev()))
    assert e.value.status == salr.SALR_ERR_CAPACITY
    shifted = torch.empty(8 * 64 + 8, dtype=torch.bfloat16, device=dev())[1:8 * 64 + 1].view(8, 64)
    with pytest.raises(salr.SalrError) as e:
        salr.linear_cross_entropy(shifted, w, t)
    assert e.value.status == salr.SALR_ERR_INVALID_ARG
