"""GPU tests of the optimiser step's defaults and of what its list of tensors may hold."""
import pytest
import torch

import finetune_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu


def test_eight_bit_averages_follow_slow_changes_without_a_seed():
    """sqrt(v) falls by 0.05 % a step where the gradients end, less than a spacing of its 8-bit values: only where every step draws other
    random numbers does its mean follow.  No seed is given.  (Sizes and tolerance as where every step is given one: the mean of 127 x 64
    values has a standard deviation of 0.14 %, 1 % is allowed.)"""
    import paper_2601_16991_amd as salr
    blocks = 64
    n = 128 * blocks
    p, g = torch.zeros(n, device=dev()), torch.zeros(n, device=dev())
    m, v, s = salr.adamw_states([p], 8)
    start = torch.full((n,), 100.0)
    start[::128] = 448.0
    v[0].copy_(start.to(torch.float8_e4m3fn))
    s[0][:, 1] = 1e-3
    opt = salr.AdamW([p], [g], m, v, scales=s)
    k = 400
    for i in range(1, k + 1):
        g[::128] = 0.448   # keeps the large one where it is
        opt.step(lr=0.0, step=i, beta2=0.999)
    got = (v[0].float().view(-1, 128) * s[0][:, 1:])[:, 1:]
    want = float(start.to(torch.float8_e4m3fn).float()[1]) * 1e-3 * 0.999 ** (k / 2)
    assert abs(float(got.mean()) / want - 1) < 0.01


def test_no_seed_means_the_number_of_the_step():
    import paper_2601_16991_amd as salr

    def go(**seed):
        gen = torch.Generator().manual_seed(4)
        g = [torch.randn(n, generator=gen).to(dev()) for n in (3000, 129)]
        opt = salr.AdamW([torch.zeros_like(x) for x in g], g, bits=8)
        for k in (3, 4):
            opt.step(lr=1e-3, step=k, **({"seed": k} if seed.get("own") else seed))
        return torch.cat([x.view(torch.uint8).cpu() for x in opt.exp_avg_sq])
    assert torch.equal(go(), go(own=True))
    assert torch.equal(go(seed=0), go(seed=0)) and not torch.equal(go(), go(seed=0))


def test_a_list_outlives_its_owner_until_its_stream_is_done():
    """An object that is dropped right after its call on a side stream: its memory is not handed to the other stream's tensors while the
    call waits there.  (They are only allocated here, never written.)"""
    import paper_2601_16991_amd as salr
    grads = [torch.full((5000,), 2.0, device=dev()), torch.full((20000,), 2.0, device=dev())]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    norm = salr.GradNorm(grads)
    opt = salr.AdamW([torch.zeros_like(g) for g in grads], grads)
    params = opt.params
    held = {norm._list.plan.data_ptr(), norm._workspace.data_ptr(), opt._list.plan.data_ptr(), *(x.data_ptr() for x in opt.exp_avg + opt.exp_avg_sq)}
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        got = norm(1.0)
    opt.step(lr=0.5, step=1, stream=side)
    del norm, opt
    taken = [torch.empty(n, dtype=torch.uint8, device=dev()) for n in (64, 256, 512, 8192, 20000, 80000) for _ in range(64)]
    busy = not side.query()
    assert not held & {x.data_ptr() for x in taken}
    side.synchronize()
    assert busy and ref.close(float(got[0]), (4.0 * 25000) ** 0.5) and all(bool((p < -0.49).all()) for p in params)


def test_memory_that_would_be_written_twice_is_refused():
    """A tied weight, a slice of another tensor, one tensor in two roles.  Gradients are only read: they may be the same."""
    import paper_2601_16991_amd as salr
    flat = torch.zeros(4096, device=dev())
    p, q, g = flat[:1024], flat[1024:2048], torch.ones(1024, device=dev())
    new = lambda: torch.zeros(1024, device=dev())
    for params, grads, kw in (
        ([p, p], [g, g.clone()], {}),                                              # tied
        ([flat[:1024], flat[1020:2044]], [g, g.clone()], {}),                      # the last four of one, the first four of the other
        ([flat[:2048], flat[1024:1032]], [torch.ones(2048, device=dev()), g[:8]], {}),   # one inside the other
        ([p], [p], {}),                                                            # its own gradient
        ([p], [g], {"exp_avg": [q], "exp_avg_sq": [q]}),
        ([p, q], [g, g], {"exp_avg": [new(), p], "exp_avg_sq": [new(), new()]}),
        ([p], [g], {"copies": [p.view(torch.bfloat16)[:1024]]}),
        ([p, q], [g, new()], {"exp_avg": [new(), new()], "exp_avg_sq": [new(), g]}),    # a state that is a gradient
    ):
        with pytest.raises(ValueError, match="shares memory with another tensor"):
            salr.AdamW(params, grads, **kw)
    salr.AdamW([p, q, flat[2048:2056]], [g, g, g[:8]]).step(lr=1.0, step=1)
    salr.AdamW([p, flat[:0], q], [g, g[:0], g]).step(lr=1.0, step=1)
    assert float(salr.GradNorm([g, g])(1.0)[0]) == float(torch.tensor(2048.0).sqrt())   # fp32's
    torch.cuda.synchronize()
    assert (flat[2056:] == 0).all() and (flat[:2056] != 0).all()


def test_autograd_sees_that_a_step_changed_what_it_saved():
    import paper_2601_16991_amd as salr
    p = torch.ones(300, device=dev(), requires_grad=True)
    g, copy = torch.ones(300, device=dev()), torch.empty(300, dtype=torch.bfloat16, device=dev())
    opt = salr.AdamW([p], [g], copies=[copy])
    before = [x._version for x in (p, copy, g)]
    loss = (p * p).sum()
    opt.step(lr=1e-2, step=1)
    assert [x._version - b for x, b in zip((p, copy, g), before)] == [1, 1, 0]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    opt.grad_norm(1.0)
    assert p._version == before[0] + 1
    with torch.inference_mode():
        q = torch.ones(300, device=dev())
        salr.AdamW([q], [g.clone()]).step(lr=1e-2, step=1)
        assert (q != 1).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_more_records_than_a_launch_has_threads_for(bits):
    """2^22 records and some, all of them empty (64 zero bytes) but the first, those around 2^22 and the last."""
    import paper_2601_16991_amd as salr
    at = [0, 4194302, 4194303, 4194304, 4194400]
    gen = torch.Generator().manual_seed(8)
    grads = [torch.randn(500 + i, generator=gen).to(dev()) for i in range(len(at))]
    few = salr.AdamW([torch.ones_like(g) for g in grads], grads, bits=bits)
    many = salr.AdamW([torch.ones_like(g) for g in grads], grads, bits=bits)
    plan = torch.zeros(at[-1] + 1, 64, dtype=torch.uint8, device=dev())
    plan[at] = many._list.plan[:64 * len(at)].view(len(at), 64)
    few.step(lr=1e-2, step=1)
    l = many._list
    assert salr.lib().salr_adamw_step(plan.data_ptr(), at[-1] + 1, l.param_type, l.grad_type, l.state_bits, 1e-2, 0.9, 0.999, 1e-8, 0.0, 1, 1, None,
                                      None) == salr.SALR_OK
    ws, out = torch.zeros(salr.GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=dev()), torch.empty(2, device=dev())
    assert salr.lib().salr_grad_norm(plan.data_ptr(), at[-1] + 1, l.grad_type, 1.0, out.data_ptr(), ws.data_ptr(), ws.numel(), None) == salr.SALR_OK
    torch.cuda.synchronize()
    for a, b in zip(few.params + few.exp_avg + few.exp_avg_sq, many.params + many.exp_avg + many.exp_avg_sq):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    want = float(torch.sqrt(sum(g.double().square().sum() for g in grads)))
    assert abs(float(out[0]) / want - 1) < 2.0 ** -23
