"""GPU tests of salr_linear_cross_entropy where its references (whole powers of two that E is kept relative to) differ from what most
calls see: masked tokens with logits far below zero, several pieces of the vocabulary, targets far above everything else, logits whose
references fp32 cannot hold as multiples of 128.  Tolerances are those of test_gpu_cross_entropy.py."""
import math

import pytest
import torch

import test_gpu_cross_entropy as base
from gpu_util import dev

pytestmark = pytest.mark.gpu


def _on_device(need_dw, *tensors):
    import paper_2601_16991_amd as salr
    return salr.linear_cross_entropy(*tensors, need_dh=True, need_dw=need_dw)


@pytest.mark.parametrize("shift", [-60.0, -200.0, -3000.0])
def test_masked_tokens_with_logits_far_below_zero(shift):
    """More than 128 M logits with both gradients.  Masked and live tokens alike have finite hidden states and all logits near `shift`,
    a few of either kind none of it."""
    T, K, V = 4200, 32, 32100
    assert T * V > 1 << 27
    h, w, t, g = base._inputs(T, K, V, 31, masked=False)
    w[:, 0] = shift
    h[:, 0] = 1.0
    h[5::16, 0] = 0.0
    h[2::16, 0] = 0.0
    t[1::4] = -100
    h, w, t, g = [x.to(dev()) for x in (h, w, t, g)]
    base._check(h, w, t, g, _on_device(True, h, w, t, g), True, True)


@pytest.mark.parametrize("need_dw", [False, True])
@pytest.mark.parametrize("others,target", [(44.0, 120.0), (44.0, 108.0), (30.0, 100.0)])
def test_targets_far_above_all_others(others, target, need_dw):
    """Targets 64 to 76 above: 1 - p between 1e-25 and 1e-30, which fp32 and bf16 hold, where 2^-126 times what is left of E does not."""
    T, K, V = 40, 64, 1300
    h, w, t, g = base._inputs(T, K, V, 41, masked=False, std_w=0.01, sure=0.0)
    t[:] = torch.arange(700, 740)   # each token is far above for its own target only
    h[:, 0] = 1.0
    w[:, 0] = others
    h[:, 1:41] = 0.0
    w[:, 1:41] = 0.0
    h[torch.arange(T), torch.arange(1, 41)] = 1.0
    w[t, torch.arange(1, 41)] = target - others
    base._check(h, w, t, g, base._run(h, w, t, g, True, need_dw), True, need_dw)


def test_targets_far_above_in_several_pieces():
    T, K, V = 4200, 32, 32100
    h, w, t, g = base._inputs(T, K, V, 42, masked=False, std_w=0.01, sure=0.0)
    h[:, 0] = 1.0
    w[:, 0] = 44.0
    h[:, 1] = 0.0
    h[::2, 1] = 1.0
    w[:, 1] = 0.0
    w[77, 1] = 76.0
    t[::2] = 77
    h, w, t, g = [x.to(dev()) for x in (h, w, t, g)]
    for need_dw in (False, True):
        base._check(h, w, t, g, _on_device(need_dw, h, w, t, g), True, need_dw)


@pytest.mark.parametrize("need_dw", [False, True])
@pytest.mark.parametrize("low", [-1e9, -1e10, -1e30, -1.5e38, -3e38])
@pytest.mark.parametrize("T", [40, 300])
def test_words_that_a_large_number_rules_out(T, low, need_dw):
    """The last words' logits are `low`, whole tiles of them: the result is that without these words."""
    K, V, real = 64, 1300, 700
    h, w, t, g = base._inputs(T, K, real, 43, masked=False)
    h[:, 0] = 1.0
    w[:, 0] = 0.0
    pad = torch.zeros(V - real, K).bfloat16()
    pad[:, 0] = low
    loss, lse, dh, dw = base._run(h, torch.cat([w, pad]), t, g, True, need_dw)
    base._check(h, w, t, g, (loss, lse, dh, dw[:real] if need_dw else None), True, need_dw)
    assert not need_dw or (dw[real:] == 0).all()


@pytest.mark.parametrize("large", [1e9, 1e10, 1e20, 1e30, 1.6e38])
def test_two_words_that_share_a_large_logit(large):
    """Both forms and several tokens: the two have one half each, whichever is the target, and a token that wants a third word gets the
    distance.  The logits are exact: one product that is not zero."""
    T, K, V = 60, 64, 1300
    w = torch.zeros(V, K).bfloat16()
    w[5, 0] = w[900, 0] = large
    w[900, 1], w[5, 2] = 3.0, 5.0
    h = torch.zeros(T, K).bfloat16()
    h[:, 0] = 1.0
    t = torch.full((T,), 5)
    t[20:40], t[40:] = 900, 33
    g = torch.linspace(0.5, 2, T)
    top = w[5, 0].double()
    for need_dw in (False, True):
        loss, lse, dh, dw = base._run(h, w, t, g, True, need_dw)
        assert ((loss[:40].double() - math.log(2)).abs() < 1e-6).all()
        assert ((loss[40:].double() / top - 1).abs() < 1e-6).all() and ((lse.double() / top - 1).abs() < 1e-6).all()
        half = w[5].double() * 0.5 + w[900].double() * 0.5
        want = g.double()[:, None] * (half - w[t].double())
        off = 2.0 ** -7 * g.double()[:, None] * (w[5].double().abs() + w[900].double().abs())
        assert ((dh.double() - want).abs() <= off + 1e-30).all()
        if need_dw:
            G = torch.zeros(T, V, dtype=torch.float64)
            G[:, 5] = G[:, 900] = 0.5
            G[torch.arange(T), t] -= 1.0
            G *= g.double()[:, None]
            assert ((dw.double() - G.t() @ h.double()).abs() <= 2.0 ** -7 * (G.abs().t() @ h.double().abs()) + 1e-30).all()


def test_large_logits_in_several_pieces():
    """Logits of 1e20 on one word in each piece, and a block of words ruled out by -1e30; both gradients."""
    T, K, V = 4200, 32, 32100
    h, w, t, g = base._inputs(T, K, V, 44, masked=False)
    h[:, 0:3] = 0.0
    w[:, 0:3] = 0.0
    h[:, 0] = 1.0
    w[20000:21000, 0] = -1e30
    w[5, 1] = w[30000, 1] = 1e20
    h[7, 1] = 1.0           # two words share this token
    t[t // 1000 == 20] = 3
    t[7] = 5
    live = torch.arange(V)[(torch.arange(V) < 20000) | (torch.arange(V) >= 21000)]
    h, w, t, g, live = [x.to(dev()) for x in (h, w, t, g, live)]
    rest = torch.arange(T, device=dev()) != 7
    where = torch.where(t >= 21000, t - 1000, t)
    for need_dw in (False, True):
        loss, lse, dh, dw = _on_device(need_dw, h, w, t, g)
        assert abs(float(loss[7]) - math.log(2)) < 1e-6 and abs(float(lse[7]) / 1e20 - 1) < 1e-2
        base._check(h[rest], w[live][:, :], where[rest], g[rest], (loss[rest], lse[rest], dh[rest], None), True, False) if not need_dw else None
        assert torch.isfinite(dh[rest].float()).all() and torch.isfinite(loss[rest]).all()
        if need_dw:
            G7 = torch.zeros(V, device=dev())
            G7[5], G7[30000] = -0.5, 0.5
            clean = _on_device(True, h[rest].contiguous(), w, t[rest].contiguous(), g[rest].contiguous())[3]
            want = clean.double() + (G7 * g[7]).double()[:, None] * h[7].double()[None]
            off = 2.0 ** -6 * ((G7.abs() * g[7].abs()).double()[:, None] * h[7].double().abs()[None] + clean.double().abs()) + 1e-4   # (fp32 sums of 4200 terms)
            assert ((dw.double() - want).abs() <= off).all()
            assert (dw[20000:21000] == 0).all()


@pytest.mark.parametrize("need_dw", [False, True])
def test_references_that_rise_and_fall_from_piece_to_piece(need_dw):
    """Three pieces of the vocabulary, in blocks of 50000 words whose logits lie near -60, 0 and 60 in turn, for other tokens near 60, 0 and
    -60: the running reference (-128, 0, 128) rises late, early or in between, and tiles fall behind it."""
    T, K, V = 1100, 32, 260003
    assert 2 * ((256 << 20) // (512 * T)) * 256 < V <= 3 * ((256 << 20) // (512 * T)) * 256
    h, w, t, g = base._inputs(T, K, V, 51)
    w[:, 0] = (torch.arange(V) // 50000 % 3 - 1).bfloat16()
    h[:, 0] = 0.0
    h[0::4, 0] = 60.0
    h[2::4, 0] = -60.0
    h, w, t, g = [x.to(dev()) for x in (h, w, t, g)]
    base._check(h, w, t, g, _on_device(need_dw, h, w, t, g), True, need_dw)


@pytest.mark.parametrize("T,V,block", [(300, 26003, 5000), (1100, 260003, 50000)])
@pytest.mark.parametrize("high", [40.0, 50.0, 60.0])
def test_words_that_are_unlikely_for_every_token_get_their_gradient(high, T, V, block):
    """A third of the words has probabilities of 1e-17 to 1e-30 where one of h's components is not zero: dw of that component is the sum of these, which
    bf16 and fp32 hold."""
    K = 32
    h, w, t, g = base._inputs(T, K, V, 51)
    w[:, 0] = (torch.arange(V) // block % 3 - 1).bfloat16()
    h[:, 0] = 0.0
    h[0::4, 0] = high
    h[2::4, 0] = -high
    h, w, t, g = [x.to(dev()) for x in (h, w, t, g)]
    base._check(h, w, t, g, _on_device(True, h, w, t, g), True, True)
