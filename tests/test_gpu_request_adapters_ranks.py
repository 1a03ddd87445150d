"""GPU tests of the calls on a list whose records have larger ranks than the call names: those ranks are not looked at, through the C boundary, against 64 bits."""
import ctypes

import pytest
import torch

import beside_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,K,N", [(1, 264, 520), (4, 203, 96), (100, 130, 331), (300, 264, 96), (1500, 136, 72)])
@pytest.mark.parametrize("most", [0, 5, 16, 17, 33, 64])
def test_ranks_above_the_largest(T, K, N, most):
    import paper_2601_16991_amd as salr
    lib, ranks = salr.lib(), [40, 8, 23, 100, 64]
    n = len(ranks)
    gen = torch.Generator().manual_seed(T + most)
    normal = lambda *s: torch.randn(*s, generator=gen).bfloat16()   # noqa: E731
    a, b = [(normal(K, r) / K ** 0.5) for r in ranks], [normal(r, N) for r in ranks]
    x, base, dy, dx_base = normal(T, K), normal(T, N), normal(T, N), normal(T, K)
    ids = torch.randint(-1, n, (T,), generator=gen, dtype=torch.int32)
    ids[: T // 2 + 1] = 3   # enough of one for sums in chunks
    da, db, xd, based, dyd, dx_based, idsd = [t.to(dev()) for t in a], [t.to(dev()) for t in b], x.to(dev()), base.to(dev()), dy.to(dev()), dx_base.to(dev()), ids.to(dev())
    ga, gb = [torch.full_like(t, 9.0) for t in da], [torch.full_like(t, 9.0) for t in db]
    table = (salr.Adapter * n)(*[salr.Adapter(*[t[i].data_ptr() for t in (da, db, ga, gb)], ranks[i]) for i in range(n)])
    records = torch.frombuffer(bytearray(bytes(table)), dtype=torch.uint8).to(dev())
    y, dx = torch.empty_like(based), torch.empty_like(xd)
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    need = max(salr.salr_adapters_add_workspace_bytes(T, K, N, n, most), salr.salr_adapters_backward_workspace_bytes(T, K, N, n, most, True))
    ws = torch.empty(need, dtype=torch.uint8, device=dev())
    assert lib.salr_adapters_add(records.data_ptr(), n, most, xd.data_ptr(), T, K, N, idsd.data_ptr(), based.data_ptr(), y.data_ptr(), ws.data_ptr(), need, stream) == salr.SALR_OK
    assert lib.salr_adapters_backward(records.data_ptr(), n, most, xd.data_ptr(), dyd.data_ptr(), T, K, N, idsd.data_ptr(), dx_based.data_ptr(), dx.data_ptr(), 1, ws.data_ptr(),
                                      need, stream) == salr.SALR_OK
    short_a, short_b = [t[:, :most].contiguous() for t in a], [t[:most].contiguous() for t in b]
    want, tol = ref.adapters(x, ids, short_a, short_b, base)
    ref.close(y, want, tol, torch.bfloat16)
    (want, tol), want_a, want_b = ref.adapters_backward(dy, x, ids, short_a, short_b, dx_base)
    ref.close(dx, want, tol, torch.bfloat16)
    for got, (w, t) in zip(ga, want_a):
        ref.close(got[:, :most], w, t, torch.bfloat16)
        assert bool((got[:, most:] == 9).all())
    for got, (w, t) in zip(gb, want_b):
        ref.close(got[:most], w, t, torch.bfloat16)
        assert bool((got[most:] == 9).all())
