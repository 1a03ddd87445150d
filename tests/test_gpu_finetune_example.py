"""GPU test of the fine-tuning example: layers, loss, clipping and optimiser together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("finetune_adapters", os.path.join(ROOT, "examples", "finetune_adapters.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("bits", [32, 8])
def test_the_loss_falls(bits):
    """64 tokens to map to followers: from about log V = 8.3 (more by the random logits) to a small part of it."""
    losses = _example().train(steps=120, bits=bits, log=None)
    assert all(0 <= x < 20 for x in losses)
    assert losses[0] > 7 and sum(losses[-5:]) / 5 < 0.25 * losses[0]


def test_same_steps_same_losses():
    train = _example().train
    assert train(steps=5, T=128, bits=8, log=None) == train(steps=5, T=128, bits=8, log=None)
