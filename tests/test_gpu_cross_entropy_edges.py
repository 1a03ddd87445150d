"""GPU tests of salr_linear_cross_entropy where its references (whole powers of two that E is kept relative to) differ from what most
calls see: masked tokens with logits far below zero, several pieces of the vocabulary, targets far above everything else, logits whose
references fp32 cannot hold as multiples of 128.  Tolerances are those of test_gpu_cross_entropy.py."""
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
