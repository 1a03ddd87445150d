"""GPU tests of the forms that adapters of many requests take for up to 128 tokens, against 64 bits: all in one launch (a workgroup is a token and up to 512 columns) on
both sides of where that ends, and in two.  Which it was is seen from the workspace, which one launch leaves alone.  Tolerances: tests/beside_ref.py, whose second
rounding of x A the one launch does not have.
"""
import pytest
import torch

import beside_ref as ref
from gpu_util import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    return salr


def _run(salr, T, K, N, ranks, one_launch):
    gen = torch.Generator().manual_seed(7 * T + K + N + sum(ranks))
    normal = lambda *shape: torch.randn(*shape, generator=gen)   # noqa: E731
    n = len(ranks)
    a, b = [(normal(K, r) / K ** 0.5).bfloat16() for r in ranks], [normal(r, N).bfloat16() for r in ranks]
    x, base = normal(T, K).bfloat16(), normal(T, N).bfloat16()
    adapters = salr.AdapterSet([t.to(dev()) for t in a], [t.to(dev()) for t in b])
    ws = torch.empty(adapters.workspace_bytes(T), dtype=torch.uint8, device=dev())
    buf = torch.full((T * N + 40,), 3.0, dtype=torch.bfloat16, device=dev())
    kinds = [torch.arange(T, dtype=torch.int32) % n, torch.full((T,), n - 1, dtype=torch.int32), torch.full((T,), -1, dtype=torch.int32), torch.full((T,), n, dtype=torch.int32),
             torch.randint(-1, n + 1, (T,), generator=gen, dtype=torch.int32)]
    for ids in kinds:
        for with_base in (True, False):
            want, tol = ref.adapters(x, ids, a, b, base if with_base else None)
            ws.fill_(255)
            got = adapters.add(x.to(dev()), ids.to(dev()), base.to(dev()) if with_base else None, workspace=ws)
            live = bool(((ids >= 0) & (ids < n)).any())
            assert bool((ws == 255).all()) == (one_launch or not live)
            ref.close(got, want, tol, torch.bfloat16)
        # in place, at an element's address between guards
        buf.fill_(3.0)
        out = buf[5:5 + T * N].view(T, N)
        out.copy_(base)
        want, tol = ref.adapters(x, ids, a, b, base)
        adapters.add(x.to(dev()), ids.to(dev()), out, out=out, workspace=ws)
        ref.close(out, want, tol, torch.bfloat16)
        assert torch.equal(out.cpu()[ids < 0], base[ids < 0])
        assert bool((buf[:5] == 3).all()) and bool((buf[5 + T * N:] == 3).all())


@pytest.mark.parametrize("T,K,N,ranks", [(1, 4096, 4096, [16]), (1, 4096, 4096, [13, 5]), (1, 2048, 8191, [32]), (1, 2048, 8192, [20, 7]), (1, 1024, 4099, [64]), (1, 1024, 4096, [41, 64]),
                                         (3, 512, 1031, [33, 64, 1]), (2, 1031, 4096, [16, 3]), (4, 700, 1537, [8, 24]), (16, 512, 512, [16, 2, 9]), (16, 512, 77, [50]), (1, 8, 8, [1]),
                                         (5, 9, 513, [64, 0, 17])])
def test_one_launch(salr, T, K, N, ranks):
    _run(salr, T, K, N, ranks, True)


@pytest.mark.parametrize("T,K,N,ranks", [(1, 4097, 64, [16]), (1, 2056, 64, [17]), (1, 512, 8193, [16]), (17, 64, 96, [16]), (9, 64, 600, [8, 16]), (1, 64, 96, [65]),
                                         (100, 517, 331, [16]), (100, 517, 331, [13, 5]), (20, 1031, 704, [16, 1]), (100, 517, 331, [32]), (128, 523, 704, [31, 20]), (100, 517, 331, [64]),
                                         (33, 1031, 264, [61, 4]), (40, 520, 331, [16]), (40, 520, 331, [32]), (70, 517, 331, [128, 9]), (18, 9, 9, [16, 250])])
def test_two_launches(salr, T, K, N, ranks):
    _run(salr, T, K, N, ranks, False)
