"""A workspace that is no contiguous memory of the call's own GPU is refused before anything is enqueued, by every entry point that takes one:
host memory, and a tensor with more elements than memory behind it."""
import pytest
import torch

from gpu_util import dev

pytestmark = pytest.mark.gpu

M, K, N, R = 8, 128, 64, 8


def _z(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device=dev())


def _entry_points():
    import paper_2601_16991_amd as salr
    x, y, a, b = _z(M, K), _z(M, N), _z(K, R), _z(R, N)
    w = _z(N, K)
    w[:, ::2] = 1.0   # two of four, K / 2 a row
    bm, v, ro = salr.encode(w)
    layer = (x, bm, v, ro, a, b)
    table = _z(N, 8, 2, dtype=torch.int32)
    salr.salr_build_slice_table(bm, ro, K, table)
    codes, scales = salr.nf4_quantize(v)
    coded = (x, bm, codes, scales, ro, v.numel(), a, b)
    t, f = _z(M, dtype=torch.int64), _z(M, dtype=torch.float32)
    return {
        "linear": lambda ws: salr.linear(*layer, workspace=ws),
        "linear_2of4": lambda ws: salr.linear_2of4(*layer, workspace=ws),
        "linear_prepared": lambda ws: salr.linear_prepared(x, bm, v, ro, table, a, b, workspace=ws),
        "salr_sparse_lowrank_linear": lambda ws: salr.salr_sparse_lowrank_linear(*layer, y, ws),
        "salr_sparse_lowrank_linear_2of4": lambda ws: salr.salr_sparse_lowrank_linear_2of4(*layer, y, ws),
        "salr_sparse_lowrank_linear_prepared": lambda ws: salr.salr_sparse_lowrank_linear_prepared(x, bm, v, ro, table, a, b, y, ws),
        "salr_qsalr_linear": lambda ws: salr.salr_qsalr_linear(*coded, y, ws),
        "PreparedLinear": lambda ws: salr.PreparedLinear(*layer, y, ws).run(),
        "PreparedQsalrLinear": lambda ws: salr.PreparedQsalrLinear(*coded, y, ws).run(),
        "salr_sparse_lowrank_linear_backward": lambda ws: salr.salr_sparse_lowrank_linear_backward(
            _z(32, K), _z(32, N), bm, v, ro, a, b, _z(32, K), _z(K, R), _z(R, N), ws),
        "salr_residual_adapter": lambda ws: salr.salr_residual_adapter(w, 8, 8, 1, _z(K, 16, dtype=torch.float32), a, b, None, ws),
        "linear_cross_entropy": lambda ws: salr.linear_cross_entropy(x, w, t, workspace=ws),
        "salr_linear_cross_entropy": lambda ws: salr.salr_linear_cross_entropy(x, w, t, None, f, f.clone(), x.clone(), None, ws),
    }


@pytest.mark.parametrize("name", ["linear", "linear_2of4", "linear_prepared", "salr_sparse_lowrank_linear", "salr_sparse_lowrank_linear_2of4",
                                  "salr_sparse_lowrank_linear_prepared", "salr_qsalr_linear", "PreparedLinear", "PreparedQsalrLinear",
                                  "salr_sparse_lowrank_linear_backward", "salr_residual_adapter", "linear_cross_entropy",
                                  "salr_linear_cross_entropy"])
def test_refused(name):
    call = _entry_points()[name]
    call(torch.empty(1 << 26, dtype=torch.uint8, device=dev()))
    torch.cuda.synchronize()
    with pytest.raises(TypeError, match="workspace must be a CUDA tensor"):
        call(torch.empty(1 << 26, dtype=torch.uint8))
    with pytest.raises(TypeError, match="workspace must be contiguous"):
        call(torch.empty(1, dtype=torch.uint8, device=dev()).expand(1 << 26))
