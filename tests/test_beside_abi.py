"""salr_dropout, salr_layer_norm, salr_adapters_add and their gradients refuse what does not fit on the host, before any launch; the mask's generator
against published values.  No GPU needed: no call here reaches a kernel."""
import ctypes

import numpy as np
import pytest

import beside_ref as ref

FAKE = 0x10000000   # never dereferenced
FAR = 1 << 40       # apart from FAKE by more than any size here


def at(i, off=0):
    return FAKE + i * FAR + off


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    salr.lib()
    return salr


def test_philox_known_answers():
    """The test vectors published with the generator (zeros, ones, digits of pi)."""
    for counter, key, want in (([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
                               ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
                               ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0], [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])):
        assert [int(w) for w in ref.philox(counter, key)] == want
    assert ref.keep_mask(13, 0.0, 5, 6).all() and len(ref.keep_mask(13, 0.5, 5, 6)) == 13
    assert np.array_equal(ref.keep_mask(64, 0.5, -1, 0).numpy(), ref.keep_mask(64, 0.5, 2 ** 64 - 1, 0).numpy())


def _dropout(salr, **kw):
    a = dict(x=at(0), residual=at(1), count=1000, type=0, p=0.1, seed_device=at(2), y=at(3)) | kw
    return salr.lib().salr_dropout(a["x"], a["residual"], a["count"], a["type"], a["p"], 1, a["seed_device"], 0, a["y"], None)


def test_dropout_arguments(salr):
    for bad in (dict(x=None), dict(y=None), dict(count=-1), dict(type=2), dict(p=-0.1), dict(p=1.0), dict(p=float("nan")), dict(p=1 - 2.0 ** -18), dict(x=at(0, 2)),
                dict(type=1, x=at(0, 1)), dict(residual=at(1, 2)), dict(y=at(3, 1)), dict(seed_device=at(2, 4)), dict(y=at(0, 4)), dict(y=at(1, 3996)),
                dict(y=at(0, -3996))):
        assert _dropout(salr, **bad) == salr.SALR_ERR_INVALID_ARG, bad
    assert _dropout(salr, count=(1 << 42) + 1) == salr.SALR_ERR_SHAPE
    assert _dropout(salr, count=0, x=None, y=None) == salr.SALR_OK


def _norm(salr, T=8, K=100, **kw):
    a = dict(x=at(0), residual=at(1), weight=at(2), bias=at(3), type=0, wtype=0, eps=1e-5, y=at(4), sum=at(5), mean=at(6), rstd=at(7)) | kw
    return salr.lib().salr_layer_norm(a["x"], a["residual"], a["weight"], a["bias"], T, K, a["type"], a["wtype"], a["eps"], a["y"], a["sum"], a["mean"], a["rstd"],
                                      None)


def test_layer_norm_arguments(salr):
    for bad in (dict(x=None), dict(weight=None), dict(y=None), dict(residual=None), dict(sum=None), dict(T=-1), dict(K=-1), dict(type=5), dict(wtype=-1),
                dict(eps=-1e-9), dict(eps=float("inf")), dict(eps=float("nan")), dict(x=at(0, 2)), dict(weight=at(2, 1)), dict(mean=at(6, 2)), dict(y=at(0, 4)),
                dict(y=at(1, 400)), dict(y=at(5)), dict(sum=at(0, 396)), dict(y=at(2, 4)), dict(mean=at(7)), dict(mean=at(0)), dict(rstd=at(4, 64)), dict(rstd=at(3))):
        assert _norm(salr, **bad) == salr.SALR_ERR_INVALID_ARG, bad
    for size in (dict(K=32769), dict(T=1 << 22), dict(K=0)):
        assert _norm(salr, **size) == salr.SALR_ERR_SHAPE
    assert _norm(salr, T=0, x=None) == salr.SALR_OK and _norm(salr, T=0, K=0, y=None) == salr.SALR_OK


def _norm_grad(salr, T=8, K=100, **kw):
    a = dict(dy=at(0), x=at(1), weight=at(2), mean=at(3), rstd=at(4), dsum=at(5), type=0, wtype=0, dx=at(6), dw=at(7), db=at(8), ws=at(9), bytes=1 << 30) | kw
    return salr.lib().salr_layer_norm_backward(a["dy"], a["x"], a["weight"], a["mean"], a["rstd"], a["dsum"], T, K, a["type"], a["wtype"], a["dx"], a["dw"], a["db"],
                                               a["ws"], a["bytes"], None)


def test_layer_norm_backward_arguments(salr):
    for bad in (dict(dy=None), dict(x=None), dict(weight=None), dict(mean=None), dict(rstd=None), dict(T=-1), dict(type=2), dict(wtype=3), dict(ws=None), dict(ws=at(9, 8)),
                dict(dy=at(0, 2)), dict(dw=at(7, 2)), dict(dx=at(0, 4)), dict(dx=at(1, -4)), dict(dx=at(5, 400)), dict(dx=at(2)), dict(dw=at(8, 4)), dict(db=at(6, 4)),
                dict(dw=at(2)), dict(db=at(3)), dict(dx=at(4))):
        assert _norm_grad(salr, **bad) == salr.SALR_ERR_INVALID_ARG, bad
    for size in (dict(K=32769), dict(T=1 << 22), dict(K=0)):
        assert _norm_grad(salr, **size) == salr.SALR_ERR_SHAPE
    need = salr.salr_layer_norm_backward_workspace_bytes(8, 100, True)
    assert need > 0 and salr.salr_layer_norm_backward_workspace_bytes(8, 100, False) == 0
    assert salr.salr_layer_norm_backward_workspace_bytes(8, 32769, True) == 0
    assert _norm_grad(salr, bytes=need - 1) == salr.SALR_ERR_CAPACITY
    assert _norm_grad(salr, dx=None, dw=None, db=None, dy=None) == salr.SALR_OK
    assert _norm_grad(salr, T=0, dw=None, db=None, dy=None) == salr.SALR_OK and _norm_grad(salr, T=0, K=0, dy=None) == salr.SALR_OK


def test_adapter_list(salr):
    def check(*adapters):
        n, most = len(adapters), ctypes.c_int64(-1)
        table = (salr.Adapter * max(n, 1))(*[salr.Adapter(*a) for a in adapters])
        return salr.lib().salr_adapter_list_check(table, n, ctypes.byref(most)), most.value
    fine = (at(0), at(1), at(2), at(3), 16)
    assert check(fine, (None, None, None, None, 0), fine[:4] + (256,)) == (salr.SALR_OK, 256)
    assert check() == (salr.SALR_OK, 0)
    for bad in ((None,) + fine[1:], (at(0), None, at(2), at(3), 1), fine[:4] + (-1,), (at(0, 8),) + fine[1:], (at(0), at(1, 2), at(2), at(3), 1), (at(0), at(1), at(2, 4), at(3), 1)):
        assert check(fine, bad)[0] == salr.SALR_ERR_INVALID_ARG, bad
    assert check(fine[:4] + (257,))[0] == salr.SALR_ERR_UNSUPPORTED
    assert salr.lib().salr_adapter_list_check(None, 2, ctypes.byref(ctypes.c_int64())) == salr.SALR_ERR_INVALID_ARG
    assert salr.lib().salr_adapter_list_check((salr.Adapter * 4097)(), 4097, ctypes.byref(ctypes.c_int64())) == salr.SALR_ERR_SHAPE


def _add(salr, T=8, K=64, N=96, n=3, rank=16, **kw):
    a = dict(list=at(0), x=at(1), ids=at(2), base=at(3), y=at(4), ws=at(5), bytes=1 << 40) | kw
    return salr.lib().salr_adapters_add(a["list"], n, rank, a["x"], T, K, N, a["ids"], a["base"], a["y"], a["ws"], a["bytes"], None)


def _grad(salr, T=8, K=64, N=96, n=3, rank=16, want=1, **kw):
    a = dict(list=at(0), x=at(1), ids=at(2), dy=at(3), dx_base=at(4), dx=at(5), ws=at(6), bytes=1 << 40) | kw
    return salr.lib().salr_adapters_backward(a["list"], n, rank, a["x"], a["dy"], T, K, N, a["ids"], a["dx_base"], a["dx"], want, a["ws"], a["bytes"], None)


def test_adapters_arguments(salr):
    sizes = (dict(T=-1), dict(K=-1), dict(N=-1), dict(n=0), dict(n=-2), dict(rank=-1), dict(rank=257))
    for bad in sizes + (dict(list=None), dict(x=None), dict(ids=None), dict(y=None), dict(ws=None), dict(list=at(0, 4)), dict(x=at(1, 1)), dict(ids=at(2, 2)),
                        dict(base=at(3, 1)), dict(y=at(4, 1)), dict(ws=at(5, 128)), dict(y=at(3, 192)), dict(y=at(1, 2)), dict(y=at(2, 2))):
        assert _add(salr, **bad) == salr.SALR_ERR_INVALID_ARG, bad
    for bad in sizes + (dict(list=None), dict(x=None), dict(ids=None), dict(dy=None), dict(ws=None), dict(list=at(0, 4)), dict(dy=at(3, 1)), dict(dx_base=at(4, 1)),
                        dict(dx=at(5, 1)), dict(dx=at(4, 2)), dict(dx=at(1)), dict(dx=at(3, -2)), dict(dx=at(2))):
        assert _grad(salr, **bad) == salr.SALR_ERR_INVALID_ARG, bad
    for size in (dict(T=1 << 28), dict(K=(1 << 22) + 1), dict(N=(1 << 22) + 1), dict(n=4097), dict(K=1 << 21, N=1 << 21, n=129), dict(T=(1 << 28) - 1, rank=256), dict(K=7), dict(N=7), dict(K=0), dict(N=0)):
        assert _add(salr, **size) == salr.SALR_ERR_SHAPE and _grad(salr, **size) == salr.SALR_ERR_SHAPE, size
    for T in (8, 300):
        need = salr.salr_adapters_add_workspace_bytes(T, 64, 96, 3, 16)
        assert need > 0 and _add(salr, T=T, bytes=need - 1) == salr.SALR_ERR_CAPACITY
        need = salr.salr_adapters_backward_workspace_bytes(T, 64, 96, 3, 16, True)
        assert need > salr.salr_adapters_backward_workspace_bytes(T, 64, 96, 3, 16, False) > 0
        assert _grad(salr, T=T, bytes=need - 1) == salr.SALR_ERR_CAPACITY
    assert salr.salr_adapters_add_workspace_bytes(8, 64, 96, 0, 16) == 0 and salr.salr_adapters_backward_workspace_bytes(1 << 28, 64, 96, 1, 16, True) == 0
    assert _add(salr, T=0, x=None) == salr.SALR_OK
    assert _grad(salr, want=0, dx=None, dy=None) == salr.SALR_OK and _grad(salr, want=0, T=0, dy=None) == salr.SALR_OK


def test_workspaces_and_inputs_that_share_memory(salr):
    """A workspace over a tensor of the call, results over the list or the seed: refused."""
    assert _dropout(salr, seed_device=at(3, 8)) == salr.SALR_ERR_INVALID_ARG
    for i in range(9):
        assert _norm_grad(salr, ws=at(i)) == salr.SALR_ERR_INVALID_ARG, i
    for i in range(5):
        assert _add(salr, ws=at(i)) == salr.SALR_ERR_INVALID_ARG, i
    for i in range(6):
        assert _grad(salr, ws=at(i)) == salr.SALR_ERR_INVALID_ARG, i
    assert _add(salr, y=at(0, 48)) == salr.SALR_ERR_INVALID_ARG and _grad(salr, dx=at(0, 48)) == salr.SALR_ERR_INVALID_ARG
