"""MI355X-native SALR linear layer: thin Python binding over the C boundary in ``include/salr.h``.

The three operations keep their C names (``salr_encode_bitmap``, ``salr_decode``,
``salr_sparse_lowrank_linear``); this module only marshals arguments: torch CUDA tensors supply
device memory and the current stream, every step of the computation runs in the HIP kernels of
``libsalr_hip.so``.  There is no CPU or PyTorch fallback: a missing library is an ImportError.  The layer's entry points
are marshalled in native code (``csrc/salr_binding.cpp``), the others through ctypes.

bf16 tensors may be given as ``torch.bfloat16`` or as their raw patterns (``torch.int16`` /
``torch.uint16``); bitmap and row offsets are ``torch.int32`` / ``torch.uint32``.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsalr_hip.so")

SALR_OK, SALR_ERR_INVALID_ARG, SALR_ERR_SHAPE, SALR_ERR_CAPACITY, SALR_ERR_UNSUPPORTED, SALR_ERR_HIP = range(6)

_lib = None
_binding = None
_vp = ctypes.c_void_p
_i64 = ctypes.c_int64


class StepTensor(ctypes.Structure):
    """salr_step_tensor_t of include/salr.h."""
    _fields_ = [("param", _vp), ("copy", _vp), ("grad", _vp), ("exp_avg", _vp), ("exp_avg_sq", _vp), ("scales", _vp), ("count", _i64)]


class Adapter(ctypes.Structure):
    """salr_adapter_t of include/salr.h."""
    _fields_ = [("a", _vp), ("b", _vp), ("da", _vp), ("db", _vp), ("rank", _i64)]


class SalrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        msg = lib().salr_status_string(status).decode()
        super().__init__(f"{where}: {msg} (status {status})")


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library.  Built by ``paper_2601_16991_amd/build.py`` (or __graft_entry__.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python paper_2601_16991_amd/build.py` first")
        L = ctypes.CDLL(LIB_PATH)
        L.salr_status_string.restype = ctypes.c_char_p
        L.salr_status_string.argtypes = [ctypes.c_int]
        L.salr_bitmap_words_per_row.restype = _i64
        L.salr_bitmap_words_per_row.argtypes = [_i64]
        L.salr_magnitude_mask_rows.restype = ctypes.c_int
        L.salr_magnitude_mask_rows.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp]
        L.salr_magnitude_mask_nm.restype = ctypes.c_int
        L.salr_magnitude_mask_nm.argtypes = [_vp, _i64, _i64, _i64, _i64, _vp, _vp]
        L.salr_encode_bitmap.restype = ctypes.c_int
        L.salr_encode_bitmap.argtypes = [_vp, _i64, _i64, _vp, _vp, _i64, _vp, _vp]
        L.salr_decode.restype = ctypes.c_int
        L.salr_decode.argtypes = [_vp, _vp, _vp, _i64, _i64, _vp, _vp]
        L.salr_linear_workspace_bytes.restype = ctypes.c_size_t
        L.salr_linear_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64]
        L.salr_linear_workspace_bytes_min.restype = ctypes.c_size_t
        L.salr_linear_workspace_bytes_min.argtypes = [_i64, _i64, _i64, _i64]
        L.salr_linear_workspace_bytes_fastest.restype = ctypes.c_size_t
        L.salr_linear_workspace_bytes_fastest.argtypes = [_i64, _i64, _i64, _i64]
        L.salr_sparse_lowrank_linear.restype = ctypes.c_int
        L.salr_sparse_lowrank_linear.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp,
                                                 ctypes.c_size_t, _vp]
        L.salr_slice_table_bytes.restype = ctypes.c_size_t
        L.salr_slice_table_bytes.argtypes = [_i64, _i64]
        L.salr_build_slice_table.restype = ctypes.c_int
        L.salr_build_slice_table.argtypes = [_vp, _vp, _i64, _i64, _vp, ctypes.c_size_t, _vp]
        L.salr_sparse_lowrank_linear_prepared.restype = ctypes.c_int
        L.salr_sparse_lowrank_linear_prepared.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp,
                                                          ctypes.c_size_t, _vp]
        L.salr_sparse_lowrank_linear_noalloc.restype = ctypes.c_int
        L.salr_sparse_lowrank_linear_noalloc.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp]
        L.salr_nf4_quantize_values.restype = ctypes.c_int
        L.salr_nf4_quantize_values.argtypes = [_vp, _i64, _vp, _vp, _vp]
        L.salr_nf4_dequantize_values.restype = ctypes.c_int
        L.salr_nf4_dequantize_values.argtypes = [_vp, _vp, _i64, _vp, _vp]
        L.salr_qsalr_linear_workspace_bytes.restype = ctypes.c_size_t
        L.salr_qsalr_linear_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, _i64]
        L.salr_qsalr_linear_workspace_bytes_fastest.restype = ctypes.c_size_t
        L.salr_qsalr_linear_workspace_bytes_fastest.argtypes = [_i64, _i64, _i64, _i64, _i64]
        L.salr_qsalr_linear.restype = ctypes.c_int
        L.salr_qsalr_linear.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _i64, _vp, _vp,
                                        ctypes.c_size_t, _vp]
        L.salr_bitmap_is_2of4.restype = ctypes.c_int
        L.salr_bitmap_is_2of4.argtypes = [_vp, _i64, _i64, _vp, _vp]
        L.salr_linear_2of4_workspace_bytes.restype = ctypes.c_size_t
        L.salr_linear_2of4_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64]
        L.salr_linear_2of4_workspace_bytes_fastest.restype = ctypes.c_size_t
        L.salr_linear_2of4_workspace_bytes_fastest.argtypes = [_i64, _i64, _i64, _i64]
        L.salr_sparse_lowrank_linear_2of4.restype = ctypes.c_int
        L.salr_sparse_lowrank_linear_2of4.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp,
                                                      ctypes.c_size_t, _vp]
        L.salr_residual.restype = ctypes.c_int
        L.salr_residual.argtypes = [_vp, _vp, _i64, _i64, _vp, _vp]
        L.salr_concat_adapters.restype = ctypes.c_int
        L.salr_concat_adapters.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_i64), _i64, _i64, _i64,
                                           _vp, _vp, _vp]
        L.salr_residual_adapter_workspace_bytes.restype = ctypes.c_size_t
        L.salr_residual_adapter_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64]
        L.salr_residual_adapter.restype = ctypes.c_int
        L.salr_residual_adapter.argtypes = [_vp, _i64, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        L.salr_linear_backward_workspace_bytes.restype = ctypes.c_size_t
        L.salr_linear_backward_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, ctypes.c_int, ctypes.c_int]
        L.salr_sparse_lowrank_linear_backward.restype = ctypes.c_int
        L.salr_sparse_lowrank_linear_backward.argtypes = [_vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _vp,
                                                          _vp, _vp, ctypes.c_size_t, _vp]
        L.salr_linear_cross_entropy_workspace_bytes.restype = ctypes.c_size_t
        L.salr_linear_cross_entropy_workspace_bytes.argtypes = [_i64, _i64, _i64, ctypes.c_int, ctypes.c_int]
        L.salr_linear_cross_entropy.restype = ctypes.c_int
        L.salr_linear_cross_entropy.argtypes = [_vp, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        L.salr_step_plan_bytes.restype = ctypes.c_size_t
        L.salr_step_plan_bytes.argtypes = [ctypes.POINTER(_i64), _i64]
        L.salr_step_plan.restype = ctypes.c_int
        L.salr_step_plan.argtypes = [ctypes.POINTER(StepTensor), _i64, ctypes.c_int, ctypes.c_int, ctypes.c_int, _vp, ctypes.c_size_t,
                                     ctypes.POINTER(_i64)]
        L.salr_adamw_step.restype = ctypes.c_int
        L.salr_adamw_step.argtypes = [_vp, _i64, ctypes.c_int, ctypes.c_int, ctypes.c_int, *[ctypes.c_double] * 5, _i64, _i64, _vp, _vp]
        L.salr_grad_norm.restype = ctypes.c_int
        L.salr_grad_norm.argtypes = [_vp, _i64, ctypes.c_int, ctypes.c_float, _vp, _vp, ctypes.c_size_t, _vp]
        L.salr_dropout.restype = ctypes.c_int
        L.salr_dropout.argtypes = [_vp, _vp, _i64, ctypes.c_int, ctypes.c_double, _i64, _vp, _i64, _vp, _vp]
        L.salr_layer_norm.restype = ctypes.c_int
        L.salr_layer_norm.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, ctypes.c_int, ctypes.c_int, ctypes.c_double, _vp, _vp, _vp, _vp, _vp]
        L.salr_layer_norm_backward_workspace_bytes.restype = ctypes.c_size_t
        L.salr_layer_norm_backward_workspace_bytes.argtypes = [_i64, _i64, ctypes.c_int]
        L.salr_layer_norm_backward.restype = ctypes.c_int
        L.salr_layer_norm_backward.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, ctypes.c_int, ctypes.c_int, _vp, _vp, _vp, _vp,
                                               ctypes.c_size_t, _vp]
        L.salr_adapter_list_check.restype = ctypes.c_int
        L.salr_adapter_list_check.argtypes = [ctypes.POINTER(Adapter), _i64, ctypes.POINTER(_i64)]
        L.salr_adapters_add_workspace_bytes.restype = ctypes.c_size_t
        L.salr_adapters_add_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, _i64]
        L.salr_adapters_add.restype = ctypes.c_int
        L.salr_adapters_add.argtypes = [_vp, _i64, _i64, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        L.salr_adapters_backward_workspace_bytes.restype = ctypes.c_size_t
        L.salr_adapters_backward_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, _i64, ctypes.c_int]
        L.salr_adapters_backward.restype = ctypes.c_int
        L.salr_adapters_backward.argtypes = [_vp, _i64, _i64, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, ctypes.c_int, _vp, ctypes.c_size_t, _vp]
        L.salr_set_kernel_timing_events.restype = None
        L.salr_set_kernel_timing_events.argtypes = [_vp, _vp]
        _lib = L
    return _lib


def _native():
    """The native half of this binding (built beside the library); its calls raise this module's SalrError."""
    global _binding
    if _binding is None:
        lib()
        from . import _salr_binding
        _salr_binding.set_error(SalrError)
        _binding = _salr_binding
    return _binding


_BF16_TYPES = (torch.bfloat16, torch.int16, torch.uint16)
_U32_TYPES = (torch.int32, torch.uint32)


def _ptr(t: Optional[torch.Tensor], kinds, name: str) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype not in kinds:
        raise TypeError(f"{name}: dtype {t.dtype} not in {kinds}")
    if not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    return t.data_ptr() if t.numel() > 0 else None


def _workspace(workspace: Optional[torch.Tensor], like: torch.Tensor) -> Tuple[Optional[int], int]:
    """Address and bytes of a caller's workspace (of any type, on the device of ``like``)."""
    if workspace is None:
        return None, 0
    if not workspace.is_cuda:
        raise TypeError("workspace must be a CUDA tensor")
    if not workspace.is_contiguous():
        raise TypeError("workspace must be contiguous")
    if like.is_cuda and workspace.device != like.device:
        raise ValueError("workspace: tensors on different devices")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _stream(stream) -> Optional[int]:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream or None


def _handle(stream) -> Optional[int]:
    """A stream argument for the native calls: None = the current stream, else the stream's handle."""
    return None if stream is None else stream.cuda_stream


def _on(stream, device):
    """The stream argument of a call on tensors of ``device``."""
    if stream.device != device:
        raise ValueError("stream: of another device than the tensors")
    return stream


def _check(status: int, where: str) -> None:
    if status != SALR_OK:
        raise SalrError(status, where)


def salr_bitmap_words_per_row(cols: int) -> int:
    return int(lib().salr_bitmap_words_per_row(cols))


def salr_magnitude_mask_rows(w: torch.Tensor, keep: int, w_hat: torch.Tensor, stream=None) -> None:
    """Enqueue the per-row magnitude mask: w_hat = w with all but the `keep` largest |w| of each row zeroed."""
    rows, cols = w.shape
    if tuple(w_hat.shape) != (rows, cols):
        raise ValueError("w_hat shape")
    st = lib().salr_magnitude_mask_rows(_ptr(w, _BF16_TYPES, "w"), rows, cols, keep,
                                        _ptr(w_hat, _BF16_TYPES, "w_hat"), _stream(stream))
    _check(st, "salr_magnitude_mask_rows")


def salr_magnitude_mask_nm(w: torch.Tensor, n_keep: int, m_group: int, w_hat: torch.Tensor, stream=None) -> None:
    """Enqueue the N:M mask: the n_keep largest |w| of every m_group consecutive columns survive."""
    rows, cols = w.shape
    if tuple(w_hat.shape) != (rows, cols):
        raise ValueError("w_hat shape")
    st = lib().salr_magnitude_mask_nm(_ptr(w, _BF16_TYPES, "w"), rows, cols, n_keep, m_group,
                                      _ptr(w_hat, _BF16_TYPES, "w_hat"), _stream(stream))
    _check(st, "salr_magnitude_mask_nm")


def salr_encode_bitmap(w_dense: torch.Tensor, bitmap: torch.Tensor, values: Optional[torch.Tensor],
                       row_offsets: torch.Tensor, stream=None) -> None:
    """Enqueue the encoder.  ``values`` None = count only; its length is the capacity."""
    rows, cols = w_dense.shape
    cap = 0 if values is None else values.numel()
    st = lib().salr_encode_bitmap(_ptr(w_dense, _BF16_TYPES, "w_dense"), rows, cols, _ptr(bitmap, _U32_TYPES, "bitmap"),
                                  _ptr(values, _BF16_TYPES, "values"), cap, _ptr(row_offsets, _U32_TYPES, "row_offsets"),
                                  _stream(stream))
    _check(st, "salr_encode_bitmap")


def salr_decode(bitmap: torch.Tensor, values: torch.Tensor, row_offsets: torch.Tensor, rows: int, cols: int,
                w_dense_out: torch.Tensor, stream=None) -> None:
    st = lib().salr_decode(_ptr(bitmap, _U32_TYPES, "bitmap"), _ptr(values, _BF16_TYPES, "values"),
                           _ptr(row_offsets, _U32_TYPES, "row_offsets"), rows, cols,
                           _ptr(w_dense_out, _BF16_TYPES, "w_dense_out"), _stream(stream))
    _check(st, "salr_decode")


def salr_linear_workspace_bytes(M: int, K: int, N: int, R: int) -> int:
    return int(lib().salr_linear_workspace_bytes(M, K, N, R))


def salr_linear_workspace_bytes_min(M: int, K: int, N: int, R: int) -> int:
    return int(lib().salr_linear_workspace_bytes_min(M, K, N, R))


def salr_linear_workspace_bytes_fastest(M: int, K: int, N: int, R: int) -> int:
    return int(lib().salr_linear_workspace_bytes_fastest(M, K, N, R))


def salr_sparse_lowrank_linear(x: torch.Tensor, bitmap: torch.Tensor, values: torch.Tensor,
                               row_offsets: torch.Tensor, a_cat: Optional[torch.Tensor],
                               b_cat: Optional[torch.Tensor], y: torch.Tensor,
                               workspace: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue Y = X What^T + (X A_cat) B_cat.  Shapes: x [M,K], bitmap [N,K/32], a_cat [K,R], b_cat [R,N], y [M,N]."""
    _native().linear(0, x, bitmap, values, row_offsets, None, a_cat, b_cat, y, workspace, _handle(stream))


def salr_slice_table_bytes(N: int, K: int) -> int:
    return int(lib().salr_slice_table_bytes(N, K))


def salr_build_slice_table(bitmap: torch.Tensor, row_offsets: torch.Tensor, K: int, slice_table: torch.Tensor,
                           stream=None) -> None:
    """Enqueue the layer's slice table: slice_table int32/uint32 [N, 8, 2] (see include/salr.h)."""
    N = bitmap.shape[0]
    _check(lib().salr_build_slice_table(_ptr(bitmap, _U32_TYPES, "bitmap"), _ptr(row_offsets, _U32_TYPES, "row_offsets"),
                                        N, K, _ptr(slice_table, _U32_TYPES, "slice_table"),
                                        slice_table.numel() * slice_table.element_size(), _stream(stream)),
           "salr_build_slice_table")


def salr_sparse_lowrank_linear_prepared(x: torch.Tensor, bitmap: torch.Tensor, values: torch.Tensor,
                                        row_offsets: torch.Tensor, slice_table: torch.Tensor,
                                        a_cat: Optional[torch.Tensor], b_cat: Optional[torch.Tensor], y: torch.Tensor,
                                        workspace: Optional[torch.Tensor], stream=None) -> None:
    """salr_sparse_lowrank_linear with the layer's slice table as one more input."""
    _native().linear(1, x, bitmap, values, row_offsets, slice_table, a_cat, b_cat, y, workspace, _handle(stream))


def salr_nf4_quantize_values(values: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """Enqueue QSALR's coding of the packed values: codes uint8 [ceil(n/2)], scales bf16 [ceil(n/64)]."""
    n = values.numel()
    if codes.dtype != torch.uint8 or codes.numel() < (n + 1) // 2 or scales.numel() < (n + 63) // 64:
        raise ValueError("codes must be uint8 [ceil(n/2)] and scales [ceil(n/64)]")
    _check(lib().salr_nf4_quantize_values(_ptr(values, _BF16_TYPES, "values"), n, _ptr(codes, (torch.uint8,), "codes"),
                                          _ptr(scales, _BF16_TYPES, "scales"), _stream(stream)), "salr_nf4_quantize_values")


def salr_nf4_dequantize_values(codes: torch.Tensor, scales: torch.Tensor, count: int, values_out: torch.Tensor,
                               stream=None) -> None:
    """Enqueue the inverse: values_out [count] bf16 (its storage padded to a multiple of 8 elements)."""
    if codes.numel() < (count + 1) // 2 or scales.numel() < (count + 63) // 64 or values_out.numel() < count:
        raise ValueError("buffers too short for count")
    _check(lib().salr_nf4_dequantize_values(_ptr(codes, (torch.uint8,), "codes"), _ptr(scales, _BF16_TYPES, "scales"), count,
                                            _ptr(values_out, _BF16_TYPES, "values_out"), _stream(stream)),
           "salr_nf4_dequantize_values")


def salr_qsalr_linear_workspace_bytes(M: int, K: int, N: int, R: int, nnz: int) -> int:
    return int(lib().salr_qsalr_linear_workspace_bytes(M, K, N, R, nnz))


def salr_qsalr_linear_workspace_bytes_fastest(M: int, K: int, N: int, R: int, nnz: int) -> int:
    return int(lib().salr_qsalr_linear_workspace_bytes_fastest(M, K, N, R, nnz))


def salr_qsalr_linear(x: torch.Tensor, bitmap: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                      row_offsets: torch.Tensor, nnz: int, a_cat: Optional[torch.Tensor], b_cat: Optional[torch.Tensor],
                      y: torch.Tensor, workspace: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue Y = X decode(bitmap, dequantised codes)^T + (X A_cat) B_cat."""
    _native().qsalr_linear(x, bitmap, codes, scales, row_offsets, nnz, a_cat, b_cat, y, workspace, _handle(stream))


def codes_alloc(count: int, device) -> torch.Tensor:
    """A buffer for the 4-bit codes of `count` values whose storage is whole 16-byte vectors (salr_qsalr_linear reads
    the codes with vector loads)."""
    nbytes = (count + 1) // 2
    return torch.empty(max((nbytes + 15) // 16 * 16, 16), dtype=torch.uint8, device=device)[:nbytes]


def nf4_quantize(values: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    n = values.numel()
    codes = codes_alloc(n, values.device)
    scales = torch.empty(max((n + 63) // 64, 1), dtype=torch.int16, device=values.device)[:(n + 63) // 64]
    salr_nf4_quantize_values(values, codes, scales)
    return codes, scales


def nf4_dequantize(codes: torch.Tensor, scales: torch.Tensor, count: int) -> torch.Tensor:
    out = values_alloc(count, codes.device)
    salr_nf4_dequantize_values(codes, scales, count, out)
    return out


def qsalr_linear(x, bitmap, codes, scales, row_offsets, nnz, a_cat, b_cat) -> torch.Tensor:
    return _native().qsalr_linear(x, bitmap, codes, scales, row_offsets, nnz, a_cat, b_cat, None, None, None)


NOALLOC_SCRATCH_BYTES = 16 * 1024 * 1024   # SALR_NOALLOC_SCRATCH_BYTES of include/salr.h


def salr_sparse_lowrank_linear_noalloc(x: torch.Tensor, bitmap: torch.Tensor, values: torch.Tensor,
                                       row_offsets: torch.Tensor, a_cat: Optional[torch.Tensor],
                                       b_cat: Optional[torch.Tensor], y: torch.Tensor, stream=None) -> None:
    """Enqueue Y = X What^T + (X A_cat) B_cat with the library's own fixed scratch array in place of a workspace."""
    M, K = x.shape
    N = y.shape[1]
    R = 0 if a_cat is None else a_cat.shape[1]
    if y.shape[0] != M or bitmap.shape[0] != N or row_offsets.numel() != N + 1:
        raise ValueError("inconsistent shapes")
    if R and (tuple(a_cat.shape) != (K, R) or tuple(b_cat.shape) != (R, N)):
        raise ValueError("adapter shapes")
    st = lib().salr_sparse_lowrank_linear_noalloc(_ptr(x, _BF16_TYPES, "x"), M, K, N, _ptr(bitmap, _U32_TYPES, "bitmap"),
                                                  _ptr(values, _BF16_TYPES, "values"),
                                                  _ptr(row_offsets, _U32_TYPES, "row_offsets"),
                                                  _ptr(a_cat, _BF16_TYPES, "a_cat"), _ptr(b_cat, _BF16_TYPES, "b_cat"), R,
                                                  _ptr(y, _BF16_TYPES, "y"), _stream(stream))
    _check(st, "salr_sparse_lowrank_linear_noalloc")


def salr_bitmap_is_2of4(bitmap: torch.Tensor, result: torch.Tensor, stream=None) -> None:
    """Enqueue the check: result[0] (one uint32 on the device) = 1 iff every aligned group of four columns has two set bits."""
    rows, wpr = bitmap.shape
    st = lib().salr_bitmap_is_2of4(_ptr(bitmap, _U32_TYPES, "bitmap"), rows, wpr * 32, _ptr(result, _U32_TYPES, "result"),
                                   _stream(stream))
    _check(st, "salr_bitmap_is_2of4")


def salr_linear_2of4_workspace_bytes(M: int, K: int, N: int, R: int) -> int:
    return int(lib().salr_linear_2of4_workspace_bytes(M, K, N, R))


def salr_linear_2of4_workspace_bytes_fastest(M: int, K: int, N: int, R: int) -> int:
    return int(lib().salr_linear_2of4_workspace_bytes_fastest(M, K, N, R))


def salr_sparse_lowrank_linear_2of4(x: torch.Tensor, bitmap: torch.Tensor, values: torch.Tensor,
                                    row_offsets: torch.Tensor, a_cat: Optional[torch.Tensor],
                                    b_cat: Optional[torch.Tensor], y: torch.Tensor,
                                    workspace: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue Y = X What^T + (X A_cat) B_cat for a weight that passes salr_bitmap_is_2of4 (not checked here)."""
    _native().linear(2, x, bitmap, values, row_offsets, None, a_cat, b_cat, y, workspace, _handle(stream))


def salr_linear_backward_workspace_bytes(M: int, K: int, N: int, R: int, want_dx: bool, want_dadb: bool) -> int:
    return int(lib().salr_linear_backward_workspace_bytes(M, K, N, R, int(want_dx), int(want_dadb)))


def salr_sparse_lowrank_linear_backward(x: Optional[torch.Tensor], dy: torch.Tensor, bitmap: torch.Tensor,
                                        values: torch.Tensor, row_offsets: torch.Tensor, a_cat: Optional[torch.Tensor],
                                        b_cat: Optional[torch.Tensor], dx: Optional[torch.Tensor],
                                        da: Optional[torch.Tensor], db: Optional[torch.Tensor],
                                        workspace: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue dX = dY What + (dY B_cat^T) A_cat^T, dA = X^T (dY B_cat^T), dB = (X A_cat)^T dY; None = not computed."""
    M, N = dy.shape
    K = bitmap.shape[1] * 32
    R = 0 if a_cat is None else a_cat.shape[1]
    if bitmap.shape[0] != N or row_offsets.numel() != N + 1:
        raise ValueError("inconsistent shapes")
    if R and (tuple(a_cat.shape) != (K, R) or tuple(b_cat.shape) != (R, N)):
        raise ValueError("adapter shapes")
    for name, t, shape in (("x", x, (M, K)), ("dx", dx, (M, K)), ("da", da, (K, R)), ("db", db, (R, N))):
        if t is not None and tuple(t.shape) != shape:
            raise ValueError(f"{name} must be {shape}")
    ws_ptr, ws_bytes = _workspace(workspace, dy)
    st = lib().salr_sparse_lowrank_linear_backward(
        _ptr(x, _BF16_TYPES, "x"), _ptr(dy, _BF16_TYPES, "dy"), M, K, N, _ptr(bitmap, _U32_TYPES, "bitmap"),
        _ptr(values, _BF16_TYPES, "values"), _ptr(row_offsets, _U32_TYPES, "row_offsets"),
        _ptr(a_cat, _BF16_TYPES, "a_cat"), _ptr(b_cat, _BF16_TYPES, "b_cat"), R, _ptr(dx, _BF16_TYPES, "dx"),
        _ptr(da, _BF16_TYPES, "da"), _ptr(db, _BF16_TYPES, "db"), ws_ptr, ws_bytes, _stream(stream))
    _check(st, "salr_sparse_lowrank_linear_backward")


def linear_backward(x, dy, bitmap, values, row_offsets, a_cat, b_cat, need_dx=True, need_dadb=True):
    """(dx, da, db); entries not asked for (or without adapters) are None."""
    return _native().linear_backward(x, dy, bitmap, values, row_offsets, a_cat, b_cat, need_dx, need_dadb)


class PreparedLinear:
    """The argument list of one salr_sparse_lowrank_linear call, marshalled once: ``run()`` is then a
    single foreign call on the stream that is current at that moment (for launch-bound loops)."""

    def __init__(self, x, bitmap, values, row_offsets, a_cat, b_cat, y, workspace, two_of_four=False, slice_table=None):
        M, K = x.shape
        N = y.shape[1]
        R = 0 if a_cat is None else a_cat.shape[1]
        if y.shape[0] != M or bitmap.shape[0] != N or row_offsets.numel() != N + 1:
            raise ValueError("inconsistent shapes")
        if R and (tuple(a_cat.shape) != (K, R) or tuple(b_cat.shape) != (R, N)):
            raise ValueError("adapter shapes")
        if slice_table is not None and (two_of_four or slice_table.numel() != N * 16):
            raise ValueError("slice table")
        self._keep = (x, bitmap, values, row_offsets, a_cat, b_cat, y, workspace, slice_table)
        ws_ptr, ws_bytes = _workspace(workspace, x)
        table = () if slice_table is None else (_ptr(slice_table, _U32_TYPES, "slice_table"),)
        self._args = (_ptr(x, _BF16_TYPES, "x"), M, K, N, _ptr(bitmap, _U32_TYPES, "bitmap"),
                      _ptr(values, _BF16_TYPES, "values"), _ptr(row_offsets, _U32_TYPES, "row_offsets")) + table + (
                      _ptr(a_cat, _BF16_TYPES, "a_cat"), _ptr(b_cat, _BF16_TYPES, "b_cat"), R,
                      _ptr(y, _BF16_TYPES, "y"), ws_ptr, ws_bytes)
        self._fn = (lib().salr_sparse_lowrank_linear_prepared if slice_table is not None else
                    lib().salr_sparse_lowrank_linear_2of4 if two_of_four else lib().salr_sparse_lowrank_linear)

    def run(self, stream_handle: Optional[int] = None) -> None:
        st = self._fn(*self._args, stream_handle)
        if st != SALR_OK:
            raise SalrError(st, "salr_sparse_lowrank_linear")


class PreparedQsalrLinear:
    """The argument list of one salr_qsalr_linear call, marshalled once (see PreparedLinear)."""

    def __init__(self, x, bitmap, codes, scales, row_offsets, nnz, a_cat, b_cat, y, workspace):
        M, K = x.shape
        N = y.shape[1]
        R = 0 if a_cat is None else a_cat.shape[1]
        if y.shape[0] != M or bitmap.shape[0] != N or row_offsets.numel() != N + 1:
            raise ValueError("inconsistent shapes")
        if R and (tuple(a_cat.shape) != (K, R) or tuple(b_cat.shape) != (R, N)):
            raise ValueError("adapter shapes")
        if codes.numel() != (nnz + 1) // 2 or scales.numel() != (nnz + 63) // 64:
            raise ValueError("codes / scales do not match nnz")
        self._keep = (x, bitmap, codes, scales, row_offsets, a_cat, b_cat, y, workspace)
        ws_ptr, ws_bytes = _workspace(workspace, x)
        self._args = (_ptr(x, _BF16_TYPES, "x"), M, K, N, _ptr(bitmap, _U32_TYPES, "bitmap"),
                      _ptr(codes, (torch.uint8,), "codes"), _ptr(scales, _BF16_TYPES, "scales"),
                      _ptr(row_offsets, _U32_TYPES, "row_offsets"), nnz, _ptr(a_cat, _BF16_TYPES, "a_cat"),
                      _ptr(b_cat, _BF16_TYPES, "b_cat"), R, _ptr(y, _BF16_TYPES, "y"), ws_ptr, ws_bytes)

    def run(self, stream_handle: Optional[int] = None) -> None:
        st = lib().salr_qsalr_linear(*self._args, stream_handle)
        if st != SALR_OK:
            raise SalrError(st, "salr_qsalr_linear")


def salr_set_kernel_timing_events(start_event: Optional[int], stop_event: Optional[int]) -> None:
    """Measurement hook: hipEvent_t handles (as integers) recorded around the fused kernel; None, None = off."""
    lib().salr_set_kernel_timing_events(start_event, stop_event)


# ---------------------------------------------------------------------------------------------------
# Convenience wrappers: allocate the outputs with torch, then call the entry points above.
# ---------------------------------------------------------------------------------------------------

def values_alloc(nnz: int, device) -> torch.Tensor:
    """A packed-values buffer of nnz elements whose storage is padded to a multiple of 16 bytes."""
    padded = (nnz + 7) // 8 * 8
    return torch.empty(max(padded, 8), dtype=torch.int16, device=device)[:nnz]


def mask_rows(w: torch.Tensor, keep: int) -> torch.Tensor:
    return _native().mask(w, keep, 0, True)


def mask_nm(w: torch.Tensor, n_keep: int, m_group: int) -> torch.Tensor:
    return _native().mask(w, n_keep, m_group, False)


def salr_residual(w: torch.Tensor, w_hat: torch.Tensor, e: torch.Tensor, stream=None) -> None:
    """Enqueue E = W - What (bf16, [rows, cols])."""
    if w.shape != w_hat.shape or w.shape != e.shape or w.dim() != 2:
        raise ValueError("w, w_hat and e must be matrices of one shape")
    rows, cols = w.shape
    _check(lib().salr_residual(_ptr(w, _BF16_TYPES, "w"), _ptr(w_hat, _BF16_TYPES, "w_hat"), rows, cols,
                               _ptr(e, _BF16_TYPES, "e"), _stream(stream)), "salr_residual")


def salr_concat_adapters(a_list: Sequence[torch.Tensor], b_list: Sequence[torch.Tensor], a_cat: torch.Tensor,
                         b_cat: torch.Tensor, stream=None) -> None:
    """Enqueue A_cat = [A_1 ... A_n] ([K, R]) and B_cat = [B_1; ...; B_n] ([R, N])."""
    n = len(a_list)
    if len(b_list) != n:
        raise ValueError("as many A_i as B_i")
    K, N = a_cat.shape[0], b_cat.shape[1]
    ranks = []
    for i, (a, b) in enumerate(zip(a_list, b_list)):
        if a.dim() != 2 or b.dim() != 2 or a.shape[0] != K or b.shape[1] != N or a.shape[1] != b.shape[0]:
            raise ValueError(f"adapter {i}: shapes {tuple(a.shape)} {tuple(b.shape)}")
        ranks.append(a.shape[1])
    if a_cat.shape[1] != sum(ranks) or b_cat.shape[0] != sum(ranks):
        raise ValueError("a_cat / b_cat do not have sum(ranks) columns / rows")
    pa = (_vp * max(n, 1))(*[_ptr(a, _BF16_TYPES, "A_i") for a in a_list])
    pb = (_vp * max(n, 1))(*[_ptr(b, _BF16_TYPES, "B_i") for b in b_list])
    rk = (_i64 * max(n, 1))(*ranks)
    _check(lib().salr_concat_adapters(pa, pb, rk, n, K, N, _ptr(a_cat, _BF16_TYPES, "a_cat"),
                                      _ptr(b_cat, _BF16_TYPES, "b_cat"), _stream(stream)), "salr_concat_adapters")


def salr_residual_adapter_workspace_bytes(N: int, K: int, r: int, oversample: int) -> int:
    return int(lib().salr_residual_adapter_workspace_bytes(N, K, r, oversample))


def salr_residual_adapter(e: torch.Tensor, r: int, oversample: int, power_iterations: int, omega: torch.Tensor,
                          a_res: torch.Tensor, b_res: torch.Tensor, sigma: Optional[torch.Tensor],
                          workspace: torch.Tensor, stream=None) -> None:
    """Enqueue the rank-r residual adapter of E [N, K]: a_res [K, r], b_res [r, N] (bf16), sigma [r] (fp32)."""
    N, K = e.shape
    if tuple(omega.shape) != (K, r + oversample) or omega.dtype != torch.float32 or not omega.is_contiguous():
        raise ValueError("omega must be a contiguous fp32 [K, r + oversample] tensor")
    if tuple(a_res.shape) != (K, r) or tuple(b_res.shape) != (r, N):
        raise ValueError("a_res must be [K, r] and b_res [r, N]")
    if sigma is not None and (sigma.dtype != torch.float32 or sigma.numel() != r):
        raise ValueError("sigma must hold r fp32 values")
    st = lib().salr_residual_adapter(_ptr(e, _BF16_TYPES, "e"), N, K, r, oversample, power_iterations,
                                     _ptr(omega, (torch.float32,), "omega"), _ptr(a_res, _BF16_TYPES, "a_res"),
                                     _ptr(b_res, _BF16_TYPES, "b_res"),
                                     None if sigma is None else _ptr(sigma, (torch.float32,), "sigma"),
                                     *_workspace(workspace, e), _stream(stream))
    _check(st, "salr_residual_adapter")


def residual_adapter(e: torch.Tensor, r: int, omega: torch.Tensor, power_iterations: int = 2):
    """(a_res, b_res, sigma) with oversample = omega.shape[1] - r."""
    N, K = e.shape
    oversample = omega.shape[1] - r
    need = salr_residual_adapter_workspace_bytes(N, K, r, oversample)
    if need == 0:
        raise ValueError("sizes not supported by salr_residual_adapter")
    ws = torch.empty(need, dtype=torch.uint8, device=e.device)
    a_res = torch.empty((K, r), dtype=e.dtype, device=e.device)
    b_res = torch.empty((r, N), dtype=e.dtype, device=e.device)
    sigma = torch.empty(r, dtype=torch.float32, device=e.device)
    salr_residual_adapter(e, r, oversample, power_iterations, omega, a_res, b_res, sigma, ws)
    return a_res, b_res, sigma


def residual(w: torch.Tensor, w_hat: torch.Tensor) -> torch.Tensor:
    e = torch.empty_like(w)
    salr_residual(w, w_hat, e)
    return e


def concat_adapters(a_list: Sequence[torch.Tensor], b_list: Sequence[torch.Tensor]) -> Tuple[torch.Tensor, torch.Tensor]:
    R = sum(a.shape[1] for a in a_list)
    a_cat = torch.empty((a_list[0].shape[0], R), dtype=a_list[0].dtype, device=a_list[0].device)
    b_cat = torch.empty((R, b_list[0].shape[1]), dtype=b_list[0].dtype, device=b_list[0].device)
    salr_concat_adapters(a_list, b_list, a_cat, b_cat)
    return a_cat, b_cat


def encode(w_dense: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(bitmap, values, row_offsets) of an already pruned dense matrix; one sync after the nonzeros are counted,
    to size ``values``."""
    return _native().encode(w_dense)


def decode(bitmap: torch.Tensor, values: torch.Tensor, row_offsets: torch.Tensor, rows: int, cols: int
           ) -> torch.Tensor:
    return _native().decode(bitmap, values, row_offsets, rows, cols)


def bitmap_is_2of4(bitmap: torch.Tensor) -> bool:
    """Check a layer once (synchronises): does every aligned group of four columns hold exactly two stored values?"""
    flag = torch.zeros(1, dtype=torch.int32, device=bitmap.device)
    salr_bitmap_is_2of4(bitmap, flag)
    return bool(int(flag.item()) == 1)


def linear_2of4(x, bitmap, values, row_offsets, a_cat, b_cat, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    return _native().linear(2, x, bitmap, values, row_offsets, None, a_cat, b_cat, None, workspace, None)


def build_slice_table(bitmap, row_offsets, K: int) -> torch.Tensor:
    N = bitmap.shape[0]
    table = torch.empty((N, 8, 2), dtype=torch.int32, device=bitmap.device)
    salr_build_slice_table(bitmap, row_offsets, K, table)
    return table


def linear_prepared(x, bitmap, values, row_offsets, slice_table, a_cat, b_cat,
                    workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    return _native().linear(1, x, bitmap, values, row_offsets, slice_table, a_cat, b_cat, None, workspace, None)


def linear(x, bitmap, values, row_offsets, a_cat, b_cat, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y = X What^T + (X A_cat) B_cat, newly allocated.  Where ``workspace`` is None, or holds what salr_linear_workspace_bytes
    tells but less than salr_linear_workspace_bytes_fastest, one of the fastest size comes from torch's allocator for the
    length of the call and the workspace that was handed over stays unused (large batches, most on layers with K % 64 == 32, whose
    decoded weight the told size does not contain; and up to 128 tokens where workgroups of 128 weight rows are faster and need
    room for partial outputs); where the allocator has no room for it the call runs on what it was given.  With the fastest size nothing but the result is
    allocated; salr_sparse_lowrank_linear, which takes y, never allocates.  linear_prepared and linear_2of4 alike."""
    return _native().linear(0, x, bitmap, values, row_offsets, None, a_cat, b_cat, None, workspace, None)


# ---- a fine-tuning step around the layers: the head's loss, the gradients' norm, the optimiser

def salr_linear_cross_entropy_workspace_bytes(T: int, K: int, V: int, want_dh: bool, want_dw: bool) -> int:
    return int(lib().salr_linear_cross_entropy_workspace_bytes(T, K, V, int(want_dh), int(want_dw)))


def salr_linear_cross_entropy(h: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, grad_loss: Optional[torch.Tensor],
                              loss: torch.Tensor, lse: torch.Tensor, dh: Optional[torch.Tensor], dw: Optional[torch.Tensor],
                              workspace: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue softmax cross entropy of the logits h w^T: loss, lse fp32 [T], dh bf16 [T, K], dw bf16 [V, K]; None = not computed."""
    T, K = h.shape
    V = w.shape[0]
    for name, t, shape in (("w", w, (V, K)), ("targets", targets, (T,)), ("grad_loss", grad_loss, (T,)), ("loss", loss, (T,)),
                           ("lse", lse, (T,)), ("dh", dh, (T, K)), ("dw", dw, (V, K))):
        if t is not None and tuple(t.shape) != shape:
            raise ValueError(f"{name} must be {shape}")
    args = (_ptr(h, _BF16_TYPES, "h"), T, K, _ptr(w, _BF16_TYPES, "w"), V, _ptr(targets, (torch.int64,), "targets"),
            _ptr(grad_loss, (torch.float32,), "grad_loss"), _ptr(loss, (torch.float32,), "loss"), _ptr(lse, (torch.float32,), "lse"),
            _ptr(dh, _BF16_TYPES, "dh"), _ptr(dw, _BF16_TYPES, "dw"), *_workspace(workspace, h))
    for name, t in (("w", w), ("targets", targets), ("grad_loss", grad_loss), ("loss", loss), ("lse", lse), ("dh", dh), ("dw", dw)):
        if t is not None and t.device != h.device:
            raise ValueError(f"{name}: tensors on different devices")
    with torch.cuda.device(h.device):
        _check(lib().salr_linear_cross_entropy(*args, _stream(None if stream is None else _on(stream, h.device))), "salr_linear_cross_entropy")


def linear_cross_entropy(h, w, targets, grad_loss=None, need_dh=True, need_dw=False, workspace=None):
    """(loss, lse, dh, dw) of softmax cross entropy on the logits h w^T, which are not stored; entries not asked for are None.  The workspace
    (allocated for the call where it is None) is small for the loss alone, with dh about 256 MiB at most, with dw up to 768 MiB, each with a few
    times the size of h: see salr_linear_cross_entropy_workspace_bytes.

    h [T, K] and w [V, K] bf16, targets [T] int64 (negative: the token is masked), grad_loss [T] fp32 (None: ones) the gradient of
    what is minimised with respect to each token's loss."""
    return _native().linear_cross_entropy(h, w, targets, grad_loss, need_dh, need_dw, workspace)


STEP_BLOCK = 128                                      # elements that share two scales of 8-bit states
GRAD_NORM_WORKSPACE_BYTES = 8192                      # SALR_GRAD_NORM_WORKSPACE_BYTES of include/salr.h


class _StepList:
    """The tensors of a step as salr_step_plan lays them out: checked and written once, copied to the device, read by every call.
    ``tensors`` holds them for the calls, which raise ValueError once one has other memory than it had (``p.data = ...``)."""

    def __init__(self, grads, params=None, copies=None, exp_avg=None, exp_avg_sq=None, scales=None):
        self.plan, self.chunks, self.param_type, self.grad_type, self.state_bits, self.tensors = _native().step_list(
            grads, params, copies, exp_avg, exp_avg_sq, scales)


class GradNorm:
    """The norm of many gradients at once: ``GradNorm(grads)(max_norm)`` is a tensor [norm, min(1, max_norm / (norm + 1e-6))], the second
    value NaN where the norm is not finite.  The tensors are read where they are at every call, on the stream that is current then; where one
    has other memory than when the object was made the call raises ValueError (making the list costs what ``AdamW`` tells).  An object has one
    workspace: calls on different streams that may overlap need an object each, or their sums are wrong."""

    def __init__(self, grads, _list=None):
        self._list = _list or _StepList(list(grads))
        # (copied, which is done on return: the first call may be on any stream)
        self._workspace = torch.zeros(GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8).to(self._list.plan.device)
        self._call = _native().grad_norm

    def __call__(self, max_norm: float = float("inf"), out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        l = self._list
        if stream is not None:
            _on(stream, l.plan.device)
            if out is None:
                with torch.cuda.stream(stream):
                    out = torch.empty(2, device=l.plan.device)
        got = self._call(l.plan, l.chunks, l.grad_type, max_norm, self._workspace, out, _handle(stream), l.tensors)
        return got if out is None else out


def adamw_states(params, bits: int = 32):
    """(exp_avg, exp_avg_sq, scales) for ``AdamW``, all zero: lists with one tensor a param, scales None for 32 bits."""
    if bits not in (8, 32):
        raise ValueError("bits must be 8 or 32")
    kind = torch.float32 if bits == 32 else torch.float8_e4m3fn
    m, v = ([torch.zeros(p.numel(), dtype=torch.uint8 if bits == 8 else kind, device=p.device).view(kind) for p in params] for _ in range(2))
    if bits == 32:
        return m, v, None
    return m, v, [torch.zeros((p.numel() + STEP_BLOCK - 1) // STEP_BLOCK, 2, device=p.device) for p in params]


class AdamW:
    """AdamW over many tensors in one launch a step.  The tensors keep their memory: a step raises ValueError where one has other memory
    than when the object was made.  Each is in the lists once (ValueError where memory that a step writes is another tensor's too): a weight that
    is used in several places is one tensor with the sum of its gradients.

    The list is laid out and copied to the GPU when the object is made: about 50 us on the host for 14 tensors and 150 for 448, against 4 and
    17 us for a step.  So gradients that stay (a backward pass that writes into them, ``zero_grad(set_to_none=False)``) cost nothing, while a
    program that has new ones every step makes an object every step, with the states of the last one.

    params        fp32 or bf16 tensors, updated in place
    grads         their gradients (fp32 or bf16), read where they are at every step: a backward pass writes into them
    exp_avg, exp_avg_sq   states: fp32, or ``torch.float8_e4m3fn`` with ``scales`` [ceil(n / 128), 2] fp32 each; None: zeros in
                  ``bits`` (``adamw_states``).  In 8 bits exp_avg_sq holds the square root.
    copies        bf16 tensors (or None) that receive the rounded params of fp32 params: what the layers read
    """

    def __init__(self, params, grads, exp_avg=None, exp_avg_sq=None, scales=None, copies=None, bits: int = 32):
        params, grads = list(params), list(grads)
        exp_avg, exp_avg_sq, scales, copies = (None if x is None else list(x) for x in (exp_avg, exp_avg_sq, scales, copies))
        if (exp_avg is None) != (exp_avg_sq is None):
            raise ValueError("exp_avg and exp_avg_sq go together")
        if exp_avg is None:
            exp_avg, exp_avg_sq, scales = adamw_states(params, bits)
        self.params, self.grads, self.exp_avg, self.exp_avg_sq, self.scales, self.copies = params, grads, exp_avg, exp_avg_sq, scales, copies
        self._list = _StepList(grads, params, copies, exp_avg, exp_avg_sq, scales)
        self._norm = GradNorm(None, self._list)
        self._call = _native().adamw_step

    def grad_norm(self, max_norm: float = float("inf"), stream=None) -> torch.Tensor:
        """[norm, factor] of the gradients (see ``GradNorm``); ``grad_norm(c)[1:]`` is a ``grad_scale`` for ``step``.  The object has one workspace
        for it: calls on different streams must not overlap (a ``GradNorm`` of its own for each stream can)."""
        return self._norm(max_norm, None, stream)

    def step(self, lr: float, step: int, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0,
             grad_scale: Optional[torch.Tensor] = None, seed: Optional[int] = None, stream=None) -> None:
        """Step number ``step`` (from 1 on).  ``grad_scale``: one fp32 on the device that the gradients are multiplied by; where it is
        not finite nothing changes.  ``seed``: of the random rounding of 8-bit states, None: ``step``.  A caller that gives one gives another
        one every step: with the same random bits step after step the averages would stay where they are.  (A captured graph replays the
        numbers of its capture.)"""
        l = self._list
        if seed is None:
            seed = step
        self._call(l.plan, l.chunks, l.param_type, l.grad_type, l.state_bits, lr, beta1, beta2, eps, weight_decay, step, seed, grad_scale,
                   None if stream is None else _on(stream, l.plan.device).cuda_stream, l.tensors)


# ---- on either side of a layer: dropout, layer norm, adapters of many requests

def _within(stream, device):
    """A stream argument for calls that allocate: that stream is the current one meanwhile."""
    return torch.cuda.stream(_on(stream, device))


def salr_dropout(x: torch.Tensor, residual: Optional[torch.Tensor], p: float, seed, offset: int, y: torch.Tensor, stream=None) -> None:
    """Enqueue y = dropout(x) (+ residual), fp32 or bf16; y may be x or residual."""
    if y is None:
        raise TypeError("y must be a tensor")
    _native().dropout(x, residual, p, seed, offset, y, None if stream is None else _on(stream, x.device).cuda_stream)


def dropout(x: torch.Tensor, p: float, seed, offset: int = 0, residual: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """residual + (keep ? x / (1 - p) : 0), newly allocated; x and residual fp32 or bf16, contiguous, of any shape.

    Which elements stay follows from their positions, ``seed`` and ``offset`` (Philox4x32-10; p is taken in steps of 2^-16): no mask is stored, and
    the gradient of x is ``dropout(dy, p, seed, offset)`` (with another gradient of x as ``residual`` where there is one).  ``seed``: a number, or an int64
    tensor of one on the GPU that is read when the kernel runs: a captured graph has other masks at every replay where that changes in between."""
    if stream is None:
        return _native().dropout(x, residual, p, seed, offset, None, None)
    with _within(stream, x.device):
        return _native().dropout(x, residual, p, seed, offset, None, None)


def salr_layer_norm(x: torch.Tensor, residual: Optional[torch.Tensor], weight: torch.Tensor, bias: Optional[torch.Tensor], eps: float, y: torch.Tensor,
                    sum: Optional[torch.Tensor], mean: Optional[torch.Tensor], rstd: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue the layer norm of x [T, K], or of sum = x + residual; mean, rstd fp32 [T] or None."""
    _native().layer_norm(x, residual, weight, bias, eps, y, sum, mean, rstd, None if stream is None else _on(stream, x.device).cuda_stream, False)


def layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, residual: Optional[torch.Tensor] = None,
               stream=None):
    """(y, sum, mean, rstd): the layer norm of every row of x [T, K], or of sum = x + residual (None without a residual), which the next residual and
    ``layer_norm_backward`` take.  x and residual fp32 or bf16, weight and bias [K] fp32 or bf16; K up to 32768."""
    if stream is None:
        return _native().layer_norm(x, residual, weight, bias, eps, None, None, None, None, None, True)
    with _within(stream, x.device):
        return _native().layer_norm(x, residual, weight, bias, eps, None, None, None, None, None, True)


def salr_layer_norm_backward_workspace_bytes(T: int, K: int, want_weights: bool) -> int:
    return int(lib().salr_layer_norm_backward_workspace_bytes(T, K, int(want_weights)))


def salr_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                             dsum: Optional[torch.Tensor], dx: Optional[torch.Tensor], dw: Optional[torch.Tensor], db: Optional[torch.Tensor],
                             workspace: Optional[torch.Tensor], stream=None) -> None:
    """Enqueue the gradient of the layer norm: dx [T, K] (may be dy, x or dsum), dw and db [K]; None = not computed."""
    for name, t in (("dx", dx), ("dw", dw), ("db", db)):
        if t is not None and not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a tensor")
    _native().layer_norm_backward(dy, x, weight, mean, rstd, dsum, dx, dw, db, workspace, None if stream is None else _on(stream, x.device).cuda_stream)


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        dsum: Optional[torch.Tensor] = None, need_dx: bool = True, need_dw: bool = False, need_db: bool = False,
                        workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, dw, db); entries not asked for are None.  x is what was normalised (``sum`` where there was a residual), mean and rstd as ``layer_norm`` gave
    them; ``dsum``: a gradient that reaches x past the norm, added to dx."""
    args = (dy, x, weight, mean, rstd, dsum, True if need_dx else None, True if need_dw else None, True if need_db else None, workspace, None)
    if stream is None:
        return _native().layer_norm_backward(*args)
    with _within(stream, x.device):
        return _native().layer_norm_backward(*args)


def salr_adapters_add_workspace_bytes(T: int, K: int, N: int, n: int, max_rank: int) -> int:
    return int(lib().salr_adapters_add_workspace_bytes(T, K, N, n, max_rank))


def salr_adapters_backward_workspace_bytes(T: int, K: int, N: int, n: int, max_rank: int, want_gradients: bool) -> int:
    return int(lib().salr_adapters_backward_workspace_bytes(T, K, N, n, max_rank, int(want_gradients)))


class AdapterSet:
    """Adapters of many requests beside one shared layer [K -> N]: a list of pairs A_i [K, r_i], B_i [r_i, N] (bf16, ranks up to 256, each its own), of
    which every token of a batch names one by its place in the list, or none by a negative id.  ``linear`` applies one pair to all tokens; here

        y[t] = base[t] + (x[t] A_i) B_i,  i = ids[t]

    Every call looks at all tensors of the set on the host, and beyond 128 tokens at all ids once for each adapter on the GPU.  Up to 64 adapters that takes no time
    that was seen (one token, 1024 x 1024, rank 16: 4.3 us, 6.0 with 512 adapters, 34 with 4096), so a set is for adapters that are in use; another adapter is
    another set.

    The set is laid out and copied to the GPU when the object is made.  The tensors keep their memory: a call raises ValueError where one has other
    memory than it had then; values may change (an optimiser's copies).  An id that is not below the number of adapters gives NaN in its token's row.

    da, db   bf16 tensors of the shapes of a and b (or None for a pair that is frozen) that ``backward`` writes, as ``AdamW`` reads gradients where
             they are.  None of them may share memory with another tensor of the set, which is checked, or of a call, which is not.
    """

    def __init__(self, a: Sequence[torch.Tensor], b: Sequence[torch.Tensor], da: Optional[Sequence[Optional[torch.Tensor]]] = None,
                 db: Optional[Sequence[Optional[torch.Tensor]]] = None):
        self.a, self.b = list(a), list(b)
        self.da, self.db = (None if x is None else list(x) for x in (da, db))
        got = _native().adapter_list(self.a, self.b, self.da, self.db)
        self._list, self.n, self.K, self.N, self.max_rank, self._tensors = got
        self._first = (self._list, self.n, self.K, self.N, self.max_rank, self._tensors)
        self._add, self._backward = _native().adapters_add, _native().adapters_backward

    def workspace_bytes(self, T: int) -> int:
        """Of a workspace for ``add`` on T tokens (more tokens can need less: take the largest of those that will come)."""
        return salr_adapters_add_workspace_bytes(T, self.K, self.N, self.n, self.max_rank)

    def backward_workspace_bytes(self, T: int) -> int:
        """Of a workspace for ``backward`` on T tokens (likewise)."""
        return salr_adapters_backward_workspace_bytes(T, self.K, self.N, self.n, self.max_rank, True)

    def add(self, x: torch.Tensor, ids: torch.Tensor, base: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
            workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """base + (x A_i) B_i for every token: x [T, K] bf16, ids [T] int32, base [T, N] bf16 (None: zeros).  ``out`` may be ``base``; None: allocated, as
        the workspace is."""
        if stream is None:
            got = self._add(*self._first, x, ids, base, out, workspace, None)
        else:
            with _within(stream, self._list.device):
                got = self._add(*self._first, x, ids, base, out, workspace, None)
        return got if out is None else out

    def linear(self, x: torch.Tensor, bitmap: torch.Tensor, values: torch.Tensor, row_offsets: torch.Tensor, ids: torch.Tensor,
               workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The shared SALR layer with every token's own adapter: x What^T + (x A_i) B_i.  ``workspace``: of the layer (see ``linear``)."""
        y = linear(x, bitmap, values, row_offsets, None, None, workspace)
        return self.add(x, ids, y, out=y)

    def backward(self, dy: torch.Tensor, x: Optional[torch.Tensor], ids: torch.Tensor, dx_base: Optional[torch.Tensor] = None,
                 dx: Optional[torch.Tensor] = None, need_dx: bool = True, need_gradients: bool = True, workspace: Optional[torch.Tensor] = None,
                 stream=None):
        """(dx, da, db): dx = dx_base + (dy B_i^T) A_i^T in ``dx`` (which may be ``dx_base``; None: allocated), the gradients in the tensors that the set was
        made with, those of an adapter without a token as zeros.  ``x``: what ``add`` had (None where only dx is asked for)."""
        if need_gradients and self.da is None and self.db is None:
            raise ValueError("a set made without da and db has no place for gradients")
        out = (True if dx is None else dx) if need_dx else None
        args = (*self._first, x, ids, dy, dx_base, out, need_gradients, workspace, None)
        if stream is None:
            got = self._backward(*args)
        else:
            with _within(stream, self._list.device):
                got = self._backward(*args)
        return got, self.da if need_gradients else None, self.db if need_gradients else None
