"""GPU tests that autograd sees what the calls beside a layer write into a caller's tensors."""
import pytest
import torch

from gpu_util import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def salr():
    import paper_2601_16991_amd as salr
    return salr


def _calls(salr):
    """(name, what the call writes, what it reads, the call) for every call that takes a place for its results."""
    normal = lambda *s: torch.randn(*s, device=dev())   # noqa: E731
    half = lambda *s: normal(*s).bfloat16()             # noqa: E731
    x, residual, y, total, dy, dx = (normal(20, 64) for _ in range(6))
    w, b, dw, db = (normal(64) for _ in range(4))
    mean, rstd = normal(20), normal(20).abs()
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=dev())
    pairs = [half(64, 8)], [half(8, 96)]
    adapters = salr.AdapterSet(*pairs, [torch.empty_like(pairs[0][0])], [torch.empty_like(pairs[1][0])])
    hx, base, out, hdy, dx_base, hdx = half(20, 64), half(20, 96), half(20, 96), half(20, 96), half(20, 64), half(20, 64)
    ids = torch.zeros(20, dtype=torch.int32, device=dev())
    return [("dropout", [y], [x, residual], lambda: salr.salr_dropout(x, residual, 0.5, 1, 0, y)),
            ("norm", [y, total, mean, rstd], [x, residual, w, b], lambda: salr.salr_layer_norm(x, residual, w, b, 1e-5, y, total, mean, rstd)),
            ("norm, in place", [residual, x], [w, b, mean, rstd], lambda: salr.salr_layer_norm(x, residual, w, b, 1e-5, residual, x, None, None)),
            ("norm's gradient", [dx, dw, db], [dy, x, w, mean, rstd, total], lambda: salr.salr_layer_norm_backward(dy, x, w, mean, rstd, total, dx, dw, db, ws)),
            ("dx of it alone, in place", [dy], [x, w, mean, rstd, dw, db], lambda: salr.salr_layer_norm_backward(dy, x, w, mean, rstd, None, dy, None, None, None)),
            ("adapters", [out], [hx, base, ids, *adapters.a, *adapters.b, *adapters.da], lambda: adapters.add(hx, ids, base, out=out)),
            ("adapters, in place", [base], [hx, ids], lambda: adapters.add(hx, ids, base, out=base)),
            ("adapters' gradients", [hdx, *adapters.da, *adapters.db], [hx, hdy, ids, dx_base, *adapters.a], lambda: adapters.backward(hdy, hx, ids, dx_base, dx=hdx)),
            ("adapters' dx alone", [dx_base], [hx, hdy, *adapters.da], lambda: adapters.backward(hdy, None, ids, dx_base, dx=dx_base, need_gradients=False))]


def test_versions_of_what_is_written_rise_and_of_what_is_read_do_not(salr):
    for name, out, read, call in _calls(salr):
        before = [t._version for t in out + read]
        call()
        assert [t._version - b for t, b in zip(out + read, before)] == [1] * len(out) + [0] * len(read), name


def test_new_results_start_at_zero(salr):
    x, w = torch.randn(20, 64, device=dev()), torch.ones(64, device=dev())
    y, _, mean, rstd = salr.layer_norm(x, w)
    for t in (y, mean, rstd, salr.dropout(x, 0.5, 1), *salr.layer_norm_backward(x, y, w, mean, rstd, need_dw=True, need_db=True)):
        assert t._version == 0


def test_autograd_refuses_a_saved_value_that_was_overwritten(salr):
    x = torch.randn(20, 64, device=dev())
    leaf = torch.randn(20, 64, device=dev(), requires_grad=True)
    saved = leaf.detach().clone()
    loss = (leaf * saved).sum()   # keeps `saved`
    salr.salr_dropout(x, None, 0.5, 1, 0, saved)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_tensors_of_inference_mode(salr):
    """They have no versions."""
    with torch.inference_mode():
        for _, _, _, call in _calls(salr):
            call()
