"""The fine-tuning operators on a GPU that is not the current one, and their refusal of tensors of several.  Needs two GPUs."""
import pytest
import torch

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(torch.cuda.device_count() < 2, reason="one GPU only")]


def _loss_inputs(device):
    gen = torch.Generator().manual_seed(1)
    h, w = torch.randn(20, 64, generator=gen).bfloat16(), (torch.randn(500, 64, generator=gen) * 0.1).bfloat16()
    return [x.to(device) for x in (h, w, torch.arange(20), torch.ones(20))]


def test_loss_on_a_gpu_that_is_not_current():
    import paper_2601_16991_amd as salr
    here, there = [salr.linear_cross_entropy(*_loss_inputs(d), need_dw=True) for d in ("cuda:0", "cuda:1")]
    torch.cuda.synchronize(1)
    assert all(b.device.index == 1 and torch.equal(a.cpu(), b.cpu()) for a, b in zip(here, there))


@pytest.mark.parametrize("which", [1, 2, 3])
def test_loss_refuses_tensors_of_two_gpus(which):
    import paper_2601_16991_amd as salr
    x = _loss_inputs("cuda:0")
    x[which] = x[which].to("cuda:1")
    with pytest.raises(ValueError, match="different devices"):
        salr.linear_cross_entropy(*x)
    f = torch.empty(20, device="cuda:0")
    with pytest.raises(ValueError, match="different devices"):
        salr.salr_linear_cross_entropy(*x, f, f.clone(), None, None, torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0"))


def test_step_and_norm_on_a_gpu_that_is_not_current():
    import paper_2601_16991_amd as salr
    got = []
    for d in ("cuda:0", "cuda:1"):
        gen = torch.Generator().manual_seed(2)
        p, g = torch.randn(3000, generator=gen).to(d), torch.randn(3000, generator=gen).to(d)
        opt = salr.AdamW([p], [g])
        norm = opt.grad_norm(0.5)
        opt.step(lr=1e-2, step=1, grad_scale=norm[1:])
        torch.cuda.synchronize(d)
        assert norm.device == p.device
        got.append((p.cpu(), norm.cpu()))
        other = torch.ones(1, device="cuda:0" if d == "cuda:1" else "cuda:1")
        with pytest.raises(ValueError, match="different devices"):
            opt.step(lr=1e-2, step=2, grad_scale=other)
        with pytest.raises(ValueError, match="another device"):
            opt.grad_norm(1.0, stream=torch.cuda.Stream(other.device))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
