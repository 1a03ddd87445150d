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
