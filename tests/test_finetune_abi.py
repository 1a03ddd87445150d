"""salr_linear_cross_entropy, salr_step_plan, salr_adamw_step and salr_grad_norm refuse what does not fit on the host, before any launch.
No GPU needed: no call here reaches a kernel."""
import ctypes

import pytest

FAKE = 0x10000   # never dereferenced


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    salr.lib()
    return salr


def _ce(salr, T=8, K=64, V=100, **kw):
    a = dict(h=FAKE, w=FAKE, targets=FAKE, grad_loss=FAKE, loss=FAKE, lse=FAKE, dh=FAKE, dw=FAKE, ws=FAKE, bytes=1 << 40) | kw
    return salr.lib().salr_linear_cross_entropy(a["h"], T, K, a["w"], V, a["targets"], a["grad_loss"], a["loss"], a["lse"], a["dh"], a["dw"], a["ws"],
                                                a["bytes"], None)


def test_cross_entropy_arguments(salr):
    for null in ("h", "w", "targets", "loss", "lse", "ws"):
        assert _ce(salr, **{null: None}) == salr.SALR_ERR_INVALID_ARG, null
    for size in (dict(T=-1), dict(K=-8), dict(V=-1)):
        assert _ce(salr, **size) == salr.SALR_ERR_INVALID_ARG
    for name, off in (("h", 2), ("w", 8), ("dh", 2), ("dw", 2), ("ws", 16), ("targets", 4), ("grad_loss", 2), ("loss", 2), ("lse", 1)):
        assert _ce(salr, **{name: FAKE + off}) == salr.SALR_ERR_INVALID_ARG, name
    for size in (dict(K=60), dict(K=(1 << 22) + 8), dict(V=0), dict(V=1 << 31), dict(T=1 << 31), dict(T=1 << 30, V=1 << 30)):
        assert _ce(salr, **size) == salr.SALR_ERR_SHAPE, size
    need = salr.salr_linear_cross_entropy_workspace_bytes(8, 64, 100, True, True)
    assert need > 0 and _ce(salr, bytes=need - 1) == salr.SALR_ERR_CAPACITY
    assert _ce(salr, T=0, dw=None) == salr.SALR_OK
    assert _ce(salr, T=0, V=0) == salr.SALR_OK


def test_cross_entropy_workspace_never_holds_the_logits(salr):
    assert salr.salr_linear_cross_entropy_workspace_bytes(8, 60, 100, True, True) == 0
    for T, K, V in ((4096, 4096, 131072), (16384, 8192, 131072), (1, 4096, 131072)):
        plain = salr.salr_linear_cross_entropy_workspace_bytes(T, K, V, False, False)
        full = salr.salr_linear_cross_entropy_workspace_bytes(T, K, V, True, True)
        assert plain < full <= (160 << 20) + 8 * T * V // 256 + 32 * T + max(16 * T * K, 16 << 20) + 65536


def _plan(salr, tensors, bits=32, param=0, grad=0, room=None):
    n = len(tensors)
    table = (salr.StepTensor * max(n, 1))(*tensors)
    counts = (ctypes.c_int64 * max(n, 1))(*[t.count for t in tensors])
    need = salr.lib().salr_step_plan_bytes(counts, n)
    out = (ctypes.c_uint8 * max(need if need < 1 << 30 else 1, 1))()
    chunks = ctypes.c_int64(-5)
    st = salr.lib().salr_step_plan(table, n, param, grad, bits, out, need if room is None else room, ctypes.byref(chunks))
    return st, need, chunks.value, out


def _tensor(salr, count=1000, **kw):
    a = dict(param=FAKE, copy=None, grad=FAKE, exp_avg=FAKE, exp_avg_sq=FAKE, scales=None, count=count) | kw
    return salr.StepTensor(*[a[k] for k in ("param", "copy", "grad", "exp_avg", "exp_avg_sq", "scales", "count")])


def test_plan(salr):
    st, need, chunks, out = _plan(salr, [_tensor(salr), _tensor(salr, 8192), _tensor(salr, 0, grad=None), _tensor(salr, 8193, param=FAKE * 2)])
    assert st == salr.SALR_OK and chunks == 4 and need == 4 * 64
    words = memoryview(out).cast("B").cast("Q")
    assert [words[8 * i] for i in range(4)] == [FAKE, FAKE, FAKE * 2, FAKE * 2 + 8192 * 4]
    counts = memoryview(out).cast("B").cast("i")
    assert [counts[16 * i + 12] for i in range(4)] == [1000, 8192, 8192, 1]
    assert [counts[16 * i + 13] for i in range(4)] == [0, 1024, 1024 + 8192, 1024 + 2 * 8192]   # whole blocks of 128


def test_plan_refusals(salr):
    bad = salr.SALR_ERR_INVALID_ARG
    assert _plan(salr, [_tensor(salr, grad=None)])[0] == bad
    assert _plan(salr, [_tensor(salr, param=None)])[0] == bad
    assert _plan(salr, [_tensor(salr, exp_avg=None)])[0] == bad
    assert _plan(salr, [_tensor(salr, exp_avg_sq=None)])[0] == bad
    assert _plan(salr, [_tensor(salr)], bits=8)[0] == bad                      # no scales
    assert _plan(salr, [_tensor(salr)], bits=16)[0] == bad
    assert _plan(salr, [_tensor(salr)], param=2)[0] == bad
    assert _plan(salr, [_tensor(salr)], grad=-1)[0] == bad
    assert _plan(salr, [_tensor(salr, copy=FAKE)], param=1)[0] == bad          # a copy of bf16
    for name, off in (("param", 8), ("grad", 2), ("exp_avg", 4), ("exp_avg_sq", 1), ("copy", 2)):
        assert _plan(salr, [_tensor(salr, **{name: FAKE + off})])[0] == bad, name
    assert _plan(salr, [_tensor(salr, scales=FAKE + 4)], bits=8)[0] == bad
    assert _plan(salr, [_tensor(salr, -1)], room=64)[0] == bad
    assert _plan(salr, [_tensor(salr, 1 << 43)], room=64)[0] == salr.SALR_ERR_SHAPE
    assert _plan(salr, [_tensor(salr, 9000)], room=64)[0] == salr.SALR_ERR_CAPACITY
    assert _plan(salr, [_tensor(salr, param=None, exp_avg=None, exp_avg_sq=None)], bits=0)[0] == salr.SALR_OK
    L = salr.lib()
    assert L.salr_step_plan_bytes(None, 3) == ctypes.c_size_t(-1).value
    assert L.salr_step_plan_bytes(None, -1) == ctypes.c_size_t(-1).value
    assert L.salr_step_plan_bytes((ctypes.c_int64 * 1)(-3), 1) == ctypes.c_size_t(-1).value
    assert L.salr_step_plan_bytes(None, 0) == 0


def test_step_and_norm_refusals(salr):
    L = salr.lib()

    def step(plan=FAKE, chunks=1, pt=0, gt=0, bits=32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, decay=0.0, number=1, scale=None):
        return L.salr_adamw_step(plan, chunks, pt, gt, bits, lr, b1, b2, eps, decay, number, 0, scale, None)

    nan, inf = float("nan"), float("inf")
    for kw in (dict(plan=None), dict(chunks=-1), dict(pt=2), dict(gt=7), dict(bits=0), dict(bits=16), dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(b1=1.0),
               dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=-1e-9), dict(decay=inf), dict(number=0), dict(plan=FAKE + 8), dict(scale=FAKE + 2)):
        assert step(**kw) == salr.SALR_ERR_INVALID_ARG, kw
    assert step(chunks=1 << 31) == salr.SALR_ERR_SHAPE
    assert step(plan=None, chunks=0) == salr.SALR_OK

    def norm(plan=FAKE, chunks=1, gt=0, most=1.0, out=FAKE, ws=FAKE, size=salr.GRAD_NORM_WORKSPACE_BYTES):
        return L.salr_grad_norm(plan, chunks, gt, most, out, ws, size, None)

    for kw in (dict(plan=None), dict(chunks=-1), dict(gt=2), dict(most=-1.0), dict(most=nan), dict(out=None), dict(ws=None), dict(out=FAKE + 1),
               dict(ws=FAKE + 4)):
        assert norm(**kw) == salr.SALR_ERR_INVALID_ARG, kw
    assert norm(chunks=1 << 31) == salr.SALR_ERR_SHAPE
    assert norm(size=salr.GRAD_NORM_WORKSPACE_BYTES - 1) == salr.SALR_ERR_CAPACITY
