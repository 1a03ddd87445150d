"""GPU tests of the norm's gradient and the adapters' gradients with rows behind 2^31 elements, on some rows against 64 bits."""
import pytest
import torch

import beside_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu


def test_norm():
    import paper_2601_16991_amd as salr
    T, K = 140_000, 16_384
    rows = [0, 131_071, 131_072, 139_999]
    x = torch.empty(T, K, dtype=torch.bfloat16, device=dev()).normal_()
    w = torch.ones(K, device=dev()) * 1.5
    y, _, mean, rstd = salr.layer_norm(x, w)
    for got, want, tol, kind in zip((y[rows], mean[rows], rstd[rows]), *ref.layer_norm(x[rows].cpu(), w.cpu(), None, 1e-5), (torch.bfloat16, torch.float32, torch.float32)):
        ref.close(got, want, tol, kind)
    dx, _, db = salr.layer_norm_backward(y, x, w, mean, rstd, need_db=True)
    want, tol = ref.layer_norm_backward(y[rows].cpu(), x[rows].cpu(), w.cpu(), mean[rows].cpu(), rstd[rows].cpu(), None)
    ref.close(dx[rows], want[0], tol[0], torch.bfloat16)
    # db of all rows: a workgroup adds T / 256 of them, then the workgroups' sums are added
    total, size = y.sum(0, dtype=torch.float64).cpu(), sum(part.double().abs().sum(0).cpu() for part in y.split(20_000))
    assert bool(((db.cpu().double() - total).abs() <= (T / 256 + 50) * ref.U * size).all())


def test_adapters_gradients():
    import paper_2601_16991_amd as salr
    T, K, N = 600_000, 8, 4100
    gen = torch.Generator(device="cuda").manual_seed(2)
    half = lambda *s: torch.randn(*s, device=dev(), generator=gen).bfloat16()   # noqa: E731
    a, b, x, dy = [half(K, 2)], [half(2, N)], half(T, K), half(T, N)
    rows = [0, 300_000, 524_287, 524_288, 599_999]
    ids = torch.full((T,), -1, dtype=torch.int32, device=dev())
    ids[rows] = 0
    adapters = salr.AdapterSet(a, b, [torch.empty_like(a[0])], [torch.empty_like(b[0])])
    dx, da, db = adapters.backward(dy, x, ids)
    (want, tol), want_a, want_b = ref.adapters_backward(dy[rows].cpu(), x[rows].cpu(), torch.zeros(5, dtype=torch.int32), [a[0].cpu()], [b[0].cpu()], None)
    ref.close(dx[rows], want, tol, torch.bfloat16)
    ref.close(da[0], *want_a[0], torch.bfloat16)
    ref.close(db[0], *want_b[0], torch.bfloat16)
    dx[rows] = 0
    assert not bool(dx.any())
