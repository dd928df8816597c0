"""ctypes binding over libdass.so -- argument marshalling only.

Every function here has the name of the C entry point it forwards to (minus the ``dass_`` prefix
where that reads better) and does nothing but check tensor devices/dtypes, allocate requested
outputs with torch, and pass raw pointers, sizes and the current CUDA stream across the C ABI
(``include/dass.h``).  There is no CPU or PyTorch fallback: if the library is missing or a call
fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Callable, Optional, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdass.so")

OK = 0
BF16, F32 = 0, 1
ACT_SILU, ACT_GELU_TANH, ACT_RELU, ACT_NONE = 0, 1, 2, 3      # ACT_NONE: linear() only
AXIS_ROWS, AXIS_COLS = 0, 1
ROUTE_CHOSEN, ROUTE_ALL = 0, 1
ACT_BY_NAME = {"silu": ACT_SILU, "gelu_tanh": ACT_GELU_TANH, "relu": ACT_RELU}

EXPORTS = (
    "dass_calib_workspace_bytes", "dass_calib_accumulate", "dass_calib_accumulate_static", "dass_calib_status",
    "dass_norm_finalize",
    "dass_score_nm", "dass_compress_nm", "dass_prune_nm", "dass_prune_status", "dass_select_workspace_bytes", "dass_select_unstructured",
    "dass_selftest_wait_timeout", "dass_feature_workspace_bytes", "dass_feature_sumsq",
    "dass_mlp_forward_workspace_bytes", "dass_mlp_forward",
    "dass_route_topk", "dass_route_topk_backward", "dass_expert_sort_workspace_bytes", "dass_expert_sort",
    "dass_expert_gather", "dass_expert_combine", "dass_expert_combine_backward", "dass_linear", "dass_linear_status",
    "dass_bounds_report", "dass_bounds_shrink_next",
    "dass_status_string", "dass_version",
)


class DassError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = int(code)
        super().__init__(f"{where}: {status_string(code)} (dass_status {int(code)})")


_lib = None


def load() -> ctypes.CDLL:
    """Loads libdass.so (built in-tree by ``python -m paper_2405_01943_b200.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2405_01943_b200.build` "
                           "(there is no fallback implementation)")
    _lib = _declare(ctypes.CDLL(LIB_PATH))
    return _lib


class library:
    """Context manager that routes every call of this module through another build of the library (the
    checked-access build, ``libdass_check.so``) and switches back on exit."""

    def __init__(self, path: str):
        self.path = path

    def __enter__(self):
        global _lib
        self._saved = _lib
        _lib = _declare(ctypes.CDLL(self.path))
        return _lib

    def __exit__(self, *exc):
        global _lib
        _lib = self._saved
        return False


def _declare(lib: ctypes.CDLL) -> ctypes.CDLL:
    i64, vp, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
    lib.dass_calib_workspace_bytes.restype = ctypes.c_int
    lib.dass_calib_workspace_bytes.argtypes = [i64, i64, i64, ctypes.c_int, ctypes.POINTER(sz)]
    lib.dass_calib_accumulate.restype = ctypes.c_int
    lib.dass_calib_accumulate.argtypes = [vp, i64, i64, vp, vp, i64, i64, i64, ctypes.c_int, ctypes.c_int,
                                          vp, vp, sz, vp]
    lib.dass_calib_accumulate_static.restype = ctypes.c_int
    lib.dass_calib_accumulate_static.argtypes = [vp, i64, i64, vp, vp, i64, i64, i64, ctypes.c_int, ctypes.c_int,
                                                 vp, ctypes.POINTER(ctypes.c_void_p), vp]
    lib.dass_calib_status.restype = ctypes.c_int
    lib.dass_calib_status.argtypes = [vp, vp]
    lib.dass_norm_finalize.restype = ctypes.c_int
    lib.dass_norm_finalize.argtypes = [vp, i64, vp, vp]
    lib.dass_score_nm.restype = ctypes.c_int
    lib.dass_score_nm.argtypes = [vp, i64, i64, i64, ctypes.c_int, vp, ctypes.c_int, ctypes.c_float,
                                  ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, vp, vp]
    lib.dass_compress_nm.restype = ctypes.c_int
    lib.dass_compress_nm.argtypes = [vp, vp, i64, i64, i64, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                     ctypes.c_int, vp, vp, vp]
    lib.dass_prune_nm.restype = ctypes.c_int
    lib.dass_prune_nm.argtypes = [vp, i64, i64, i64, ctypes.c_int, vp, ctypes.c_int, ctypes.c_float,
                                  ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, vp, vp, vp, vp]
    lib.dass_prune_status.restype = ctypes.c_int
    lib.dass_prune_status.argtypes = [vp]
    lib.dass_select_workspace_bytes.restype = ctypes.c_int
    lib.dass_select_workspace_bytes.argtypes = [i64, i64, ctypes.c_int, ctypes.POINTER(sz)]
    lib.dass_select_unstructured.restype = ctypes.c_int
    lib.dass_select_unstructured.argtypes = [vp, i64, i64, i64, ctypes.c_int, vp, ctypes.c_int, ctypes.c_float,
                                             ctypes.c_double, ctypes.c_int, vp, vp, vp, sz, vp]
    lib.dass_selftest_wait_timeout.restype = ctypes.c_int
    lib.dass_selftest_wait_timeout.argtypes = [vp, i64, vp]
    lib.dass_feature_workspace_bytes.restype = ctypes.c_int
    lib.dass_feature_workspace_bytes.argtypes = [i64, i64, ctypes.POINTER(sz)]
    lib.dass_feature_sumsq.restype = ctypes.c_int
    lib.dass_feature_sumsq.argtypes = [vp, i64, i64, i64, ctypes.c_int, vp, vp, sz, vp]
    lib.dass_mlp_forward_workspace_bytes.restype = ctypes.c_int
    lib.dass_mlp_forward_workspace_bytes.argtypes = [i64, i64, i64, ctypes.c_int, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    lib.dass_mlp_forward.restype = ctypes.c_int
    lib.dass_mlp_forward.argtypes = [vp, i64, i64, vp, vp, i64, i64, i64, vp, i64, ctypes.c_int, ctypes.c_int,
                                     vp, i64, vp, sz, vp]
    ci = ctypes.c_int
    lib.dass_route_topk.restype = ci
    lib.dass_route_topk.argtypes = [vp, i64, i64, i64, ci, ci, ci, vp, vp, vp]
    lib.dass_route_topk_backward.restype = ci
    lib.dass_route_topk_backward.argtypes = [vp, i64, i64, i64, ci, ci, ci, vp, vp, vp, i64, vp]
    lib.dass_expert_sort_workspace_bytes.restype = ci
    lib.dass_expert_sort_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
    lib.dass_expert_sort.restype = ci
    lib.dass_expert_sort.argtypes = [vp, i64, i64, i64, vp, vp, vp, vp, sz, vp]
    lib.dass_expert_gather.restype = ci
    lib.dass_expert_gather.argtypes = [vp, i64, i64, i64, ci, vp, i64, vp, vp, vp, i64, i64, vp]
    lib.dass_expert_combine.restype = ci
    lib.dass_expert_combine.argtypes = [vp, i64, i64, i64, ci, vp, i64, i64, vp, vp, i64, vp, i64, vp]
    lib.dass_expert_combine_backward.restype = ci
    lib.dass_expert_combine_backward.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, vp, i64, vp, vp, vp, i64, vp, vp]
    lib.dass_linear.restype = ci
    lib.dass_linear.argtypes = [vp, i64, i64, i64, vp, vp, i64, i64, i64, vp, vp, ci, vp, i64, vp, i64, ci, vp, i64, vp]
    lib.dass_linear_status.restype = ci
    lib.dass_linear_status.argtypes = [vp]
    lib.dass_status_string.restype = ctypes.c_char_p
    lib.dass_status_string.argtypes = [ctypes.c_int]
    lib.dass_version.restype = ctypes.c_int
    lib.dass_version.argtypes = []
    lib.dass_bounds_report.restype = ctypes.c_int
    lib.dass_bounds_report.argtypes = [ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_ulonglong),
                                       ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int), vp]
    lib.dass_bounds_shrink_next.restype = ctypes.c_int
    lib.dass_bounds_shrink_next.argtypes = [sz]
    return lib


def status_string(code: int) -> str:
    return load().dass_status_string(int(code)).decode()


def version() -> int:
    return int(load().dass_version())


def _check(code: int, where: str) -> None:
    if code != OK:
        raise DassError(code, where)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype}: the library takes bfloat16 or float32")


def _here(t: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> int:
    """The index of the tensor's device, which has to be the current one: that is where the library launches, and whose
    streams and records it uses."""
    device, current = t.get_device(), torch._C._cuda_getDevice()
    if device != current:
        raise ValueError(f"a tensor on cuda:{device} while cuda:{current} is current: make the tensor's device current (torch.cuda.device)")
    if stream is not None and stream.device_index != device:
        raise ValueError(f"a stream of cuda:{stream.device_index} for tensors on cuda:{device}")
    return device


def _matrix(t: torch.Tensor, name: str) -> Tuple[int, int, int]:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    _here(t)
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError(f"{name} must be a 2-D row-major tensor (unit stride along columns)")
    return t.shape[0], t.shape[1], t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


def _stream_of(t: torch.Tensor, stream: Optional[torch.cuda.Stream]) -> int:
    """The given stream, or the current one of the tensor's device (by its raw handle: building a Stream object costs as
    much as the launch of a small kernel)."""
    if stream is None:
        device = t.get_device()
        if device == torch._C._cuda_getDevice():
            return torch._C._cuda_getCurrentRawStream(device)
    _here(t, stream)
    return stream.cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _made(stream: Optional[torch.cuda.Stream], device: torch.device, make: Callable[[], torch.Tensor]) -> torch.Tensor:
    """make()'s tensor for a call on `stream`.

    Memory from the allocator belongs to the stream that was current: it may still be in use by that stream's earlier work,
    and once released it is handed to that stream's later work, whatever another stream does with it.  So the tensor comes
    from the pool of the stream that the call runs on (where it is filled, if it is), and is also kept until what the
    caller's current stream has queued by its release is done."""
    if stream is None:
        return make()
    here = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        out = make()
    if here != stream:
        out.record_stream(here)
    return out


def _new(t: torch.Tensor, stream: Optional[torch.cuda.Stream]) -> Callable[..., torch.Tensor]:
    """t.new_empty for a call on `stream`."""
    return t.new_empty if stream is None else lambda shape, dtype=None: _made(stream, t.device, lambda: t.new_empty(shape, dtype=dtype))


def _workspace(t: torch.Tensor, device: torch.device) -> None:
    """Checks a caller's workspace: kernels write to its address."""
    if not t.is_cuda or t.dtype != torch.uint8 or t.device != device or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {device}")


# ----------------------------------------------------------------------------- stage (a)

def calib_workspace_bytes(T: int, d: int, I: int, dtype: torch.dtype) -> int:
    out = ctypes.c_size_t(0)
    code = load().dass_calib_workspace_bytes(int(T), int(d), int(I), BF16 if dtype == torch.bfloat16 else F32,
                                             ctypes.byref(out))
    _check(code, "dass_calib_workspace_bytes")
    return int(out.value)


def calib_workspace(T: int, d: int, I: int, dtype: torch.dtype, device="cuda") -> torch.Tensor:
    """A uint8 tensor large (and aligned) enough to serve as workspace of calib_accumulate."""
    n = calib_workspace_bytes(T, d, I, dtype)
    buf = torch.empty(n + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf[off:off + n]


def calib_accumulate(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, act: int, sumsq: torch.Tensor,
                     workspace: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """sumsq[i] += sum_t (act(X Wg^T) * (X Wu^T))[t, i]^2 on the given (or current) stream."""
    T, d, ldx = _matrix(X, "X")
    I, d2, ldw = _matrix(Wg, "Wg")
    I3, d3, ldw3 = _matrix(Wu, "Wu")
    if (d2, I3, d3, ldw3) != (d, I, d, ldw) or Wg.dtype != X.dtype or Wu.dtype != X.dtype:
        raise ValueError("X [T x d], Wg [I x d], Wu [I x d] must agree in d, I, dtype and row pitch")
    if sumsq.dtype != torch.float64 or not sumsq.is_cuda or sumsq.numel() != I or not sumsq.is_contiguous():
        raise ValueError("sumsq must be a contiguous CUDA float64 tensor of I elements")
    if not workspace.is_cuda or workspace.dtype != torch.uint8:
        raise ValueError("workspace must be a CUDA uint8 tensor (see calib_workspace)")
    code = load().dass_calib_accumulate(X.data_ptr(), T, ldx, Wg.data_ptr(), Wu.data_ptr(), I, d, ldw,
                                        _dtype_code(X), int(act), sumsq.data_ptr(),
                                        workspace.data_ptr(), workspace.numel(), _stream(stream))
    _check(code, "dass_calib_accumulate")


STATIC_SCRATCH_BYTES = 16 << 20


def calib_accumulate_static(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, act: int, sumsq: torch.Tensor,
                            stream: Optional[torch.cuda.Stream] = None) -> int:
    """calib_accumulate for callers that must not allocate: the scratch is a fixed array inside the
    library (at most STATIC_SCRATCH_BYTES, shared by all calls on the device -- do not overlap calls).
    Returns the scratch's device address, which calib_status_at() accepts."""
    T, d, ldx = _matrix(X, "X")
    I, d2, ldw = _matrix(Wg, "Wg")
    I3, d3, ldw3 = _matrix(Wu, "Wu")
    if (d2, I3, d3, ldw3) != (d, I, d, ldw) or Wg.dtype != X.dtype or Wu.dtype != X.dtype:
        raise ValueError("X [T x d], Wg [I x d], Wu [I x d] must agree in d, I, dtype and row pitch")
    if sumsq.dtype != torch.float64 or not sumsq.is_cuda or sumsq.numel() != I or not sumsq.is_contiguous():
        raise ValueError("sumsq must be a contiguous CUDA float64 tensor of I elements")
    addr = ctypes.c_void_p(0)
    code = load().dass_calib_accumulate_static(X.data_ptr(), T, ldx, Wg.data_ptr(), Wu.data_ptr(), I, d, ldw,
                                               _dtype_code(X), int(act), sumsq.data_ptr(), ctypes.byref(addr),
                                               _stream(stream))
    _check(code, "dass_calib_accumulate_static")
    return int(addr.value)


def calib_status_at(address: int, stream: Optional[torch.cuda.Stream] = None) -> None:
    """calib_status for a raw device address (the one calib_accumulate_static returned)."""
    _check(load().dass_calib_status(int(address), _stream(stream)), "dass_calib_status")


def calib_status(workspace: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Waits for the stream and raises if the last calibration kernel reported a timed-out wait."""
    _check(load().dass_calib_status(workspace.data_ptr(), _stream(stream)), "dass_calib_status")


def norm_finalize(sumsq: torch.Tensor, norm: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """norm = float32(sqrt(sumsq))."""
    _here(sumsq, stream)
    if norm is None:
        norm = _new(sumsq, stream)(sumsq.numel(), dtype=torch.float32)
    code = load().dass_norm_finalize(sumsq.data_ptr(), sumsq.numel(), norm.data_ptr(), _stream(stream))
    _check(code, "dass_norm_finalize")
    return norm


# ----------------------------------------------------------------------------- stage (b)

def mask_words_per_row(cols: int) -> int:
    return (cols + 31) // 32


def score_nm(W: torch.Tensor, norm: torch.Tensor, norm_axis: int, alpha: float, n_keep: int, m: int,
             group_axis: int, mask_bits: Optional[torch.Tensor] = None, W_pruned: Optional[torch.Tensor] = None,
             want_mask: bool = True, want_pruned: bool = True,
             stream: Optional[torch.cuda.Stream] = None):
    """Eq. 4 / Eq. 5 score + N:M selection. Returns (mask_bits or None, W_pruned or None)."""
    rows, cols, ld = _matrix(W, "W")
    if norm.dtype != torch.float32 or not norm.is_cuda or not norm.is_contiguous():
        raise ValueError("norm must be a contiguous CUDA float32 tensor")
    if norm.numel() != (rows if norm_axis == AXIS_ROWS else cols):
        raise ValueError("norm has the wrong length for norm_axis")
    if mask_bits is None and want_mask:
        mask_bits = _new(W, stream)((rows, mask_words_per_row(cols)), dtype=torch.int32)
    if W_pruned is None and want_pruned:
        W_pruned = _made(stream, W.device, lambda: W.new_empty_strided((rows, cols), (ld, 1)))
    if W_pruned is not None:
        prow, pcol, pld = _matrix(W_pruned, "W_pruned")
        if (prow, pcol, pld) != (rows, cols, ld) or W_pruned.dtype != W.dtype:
            raise ValueError("W_pruned must have W's shape, dtype and row pitch")
    code = load().dass_score_nm(W.data_ptr(), rows, cols, ld, _dtype_code(W), norm.data_ptr(), int(norm_axis),
                                float(alpha), int(n_keep), int(m), int(group_axis),
                                _ptr(mask_bits), _ptr(W_pruned), _stream(stream))
    _check(code, "dass_score_nm")
    return mask_bits, W_pruned


def compress_shapes(rows: int, cols: int, n_keep: int, m: int, group_axis: int):
    """((value rows, value cols), (meta lines, meta words per line))."""
    bits = 4 if (n_keep == 2 and m == 4) else m
    fpw = 32 // bits
    if group_axis == AXIS_COLS:
        return (rows, cols // m * n_keep), (rows, (cols // m + fpw - 1) // fpw)
    return (rows // m * n_keep, cols), (rows // m, (cols + fpw - 1) // fpw)


def compress_nm(W: torch.Tensor, mask_bits: torch.Tensor, n_keep: int, m: int, group_axis: int,
                values: Optional[torch.Tensor] = None, meta: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None):
    """Compressed values + metadata of W under mask_bits. Returns (values, meta)."""
    rows, cols, ld = _matrix(W, "W")
    vshape, mshape = compress_shapes(rows, cols, n_keep, m, group_axis)
    if values is None:
        values = _new(W, stream)(vshape)
    if meta is None:
        meta = _new(W, stream)(mshape, dtype=torch.int32)
    if tuple(values.shape) != vshape or not values.is_contiguous() or values.dtype != W.dtype:
        raise ValueError(f"values must be a contiguous {vshape} tensor of W's dtype")
    if tuple(meta.shape) != mshape or not meta.is_contiguous() or meta.dtype != torch.int32:
        raise ValueError(f"meta must be a contiguous int32 {mshape} tensor")
    if mask_bits.dtype != torch.int32 or not mask_bits.is_contiguous() or \
            tuple(mask_bits.shape) != (rows, mask_words_per_row(cols)):
        raise ValueError("mask_bits must be the contiguous int32 [rows x ceil(cols/32)] tensor score_nm produced")
    code = load().dass_compress_nm(W.data_ptr(), mask_bits.data_ptr(), rows, cols, ld, _dtype_code(W),
                                   int(n_keep), int(m), int(group_axis), values.data_ptr(), meta.data_ptr(),
                                   _stream(stream))
    _check(code, "dass_compress_nm")
    return values, meta


def prune_nm(W: torch.Tensor, norm: torch.Tensor, norm_axis: int, alpha: float, n_keep: int, m: int,
             group_axis: int, mask_bits: Optional[torch.Tensor] = None, W_pruned: Optional[torch.Tensor] = None,
             values: Optional[torch.Tensor] = None, meta: Optional[torch.Tensor] = None,
             want_mask: bool = True, want_pruned: bool = True, want_compressed: bool = True,
             stream: Optional[torch.cuda.Stream] = None):
    """score_nm and compress_nm of the same selection in one pass over W.
    Returns (mask_bits or None, W_pruned or None, values or None, meta or None)."""
    rows, cols, ld = _matrix(W, "W")
    if norm.dtype != torch.float32 or not norm.is_cuda or not norm.is_contiguous():
        raise ValueError("norm must be a contiguous CUDA float32 tensor")
    if norm.numel() != (rows if norm_axis == AXIS_ROWS else cols):
        raise ValueError("norm has the wrong length for norm_axis")
    if mask_bits is None and want_mask:
        mask_bits = _new(W, stream)((rows, mask_words_per_row(cols)), dtype=torch.int32)
    if W_pruned is None and want_pruned:
        W_pruned = _made(stream, W.device, lambda: W.new_empty_strided((rows, cols), (ld, 1)))
    if W_pruned is not None:
        prow, pcol, pld = _matrix(W_pruned, "W_pruned")
        if (prow, pcol, pld) != (rows, cols, ld) or W_pruned.dtype != W.dtype:
            raise ValueError("W_pruned must have W's shape, dtype and row pitch")
    if mask_bits is not None and (mask_bits.dtype != torch.int32 or not mask_bits.is_contiguous() or
                                  tuple(mask_bits.shape) != (rows, mask_words_per_row(cols))):
        raise ValueError("mask_bits must be a contiguous int32 [rows x ceil(cols/32)] tensor")
    if want_compressed or values is not None or meta is not None:
        vshape, mshape = compress_shapes(rows, cols, n_keep, m, group_axis)
        if values is None:
            values = _new(W, stream)(vshape)
        if meta is None:
            meta = _new(W, stream)(mshape, dtype=torch.int32)
        if tuple(values.shape) != vshape or not values.is_contiguous() or values.dtype != W.dtype:
            raise ValueError(f"values must be a contiguous {vshape} tensor of W's dtype")
        if tuple(meta.shape) != mshape or not meta.is_contiguous() or meta.dtype != torch.int32:
            raise ValueError(f"meta must be a contiguous int32 {mshape} tensor")
    code = load().dass_prune_nm(W.data_ptr(), rows, cols, ld, _dtype_code(W), norm.data_ptr(), int(norm_axis),
                                float(alpha), int(n_keep), int(m), int(group_axis),
                                _ptr(mask_bits), _ptr(W_pruned), _ptr(values), _ptr(meta), _stream(stream))
    _check(code, "dass_prune_nm")
    return mask_bits, W_pruned, values, meta


def prune_status(stream: Optional[torch.cuda.Stream] = None) -> None:
    """Waits for the stream and raises if, since the last query, a bounded wait inside a prune_nm or
    select_unstructured kernel ran out or the passes of a select_unstructured call disagreed."""
    _check(load().dass_prune_status(_stream(stream)), "dass_prune_status")


def bounds_report(stream: Optional[torch.cuda.Stream] = None) -> dict:
    """Checked-access build only: accesses outside the registered buffers since the last report (and clears it)."""
    n, addr, nbytes, line = ctypes.c_int(0), ctypes.c_ulonglong(0), ctypes.c_int(0), ctypes.c_int(0)
    _check(load().dass_bounds_report(ctypes.byref(n), ctypes.byref(addr), ctypes.byref(nbytes), ctypes.byref(line),
                                     _stream(stream)), "dass_bounds_report")
    return {"violations": n.value, "first_address": addr.value, "first_bytes": nbytes.value, "first_line": line.value}


def bounds_shrink_next(nbytes: int) -> None:
    """Checked-access build only (test hook): the next call registers every buffer `nbytes` shorter."""
    _check(load().dass_bounds_shrink_next(int(nbytes)), "dass_bounds_shrink_next")


def select_workspace(rows: int, cols: int, norm_axis: int, device="cuda") -> torch.Tensor:
    """A 16-byte aligned uint8 CUDA tensor of the size dass_select_unstructured needs."""
    need = ctypes.c_size_t(0)
    _check(load().dass_select_workspace_bytes(int(rows), int(cols), int(norm_axis), ctypes.byref(need)),
           "dass_select_workspace_bytes")
    buf = torch.empty(need.value + 16, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 16
    return buf[off:off + need.value]


def select_unstructured(W: torch.Tensor, norm: torch.Tensor, norm_axis: int, alpha: float, sparsity: float,
                        compare_axis: int, mask_bits: Optional[torch.Tensor] = None,
                        W_pruned: Optional[torch.Tensor] = None, want_mask: bool = True, want_pruned: bool = True,
                        workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Unstructured selection at `sparsity` inside every column (compare_axis = ROWS) or row (COLS).
    Returns (mask_bits or None, W_pruned or None)."""
    rows, cols, ld = _matrix(W, "W")
    if norm.dtype != torch.float32 or not norm.is_cuda or not norm.is_contiguous():
        raise ValueError("norm must be a contiguous CUDA float32 tensor")
    if norm.numel() != (rows if norm_axis == AXIS_ROWS else cols):
        raise ValueError("norm has the wrong length for norm_axis")
    if mask_bits is None and want_mask:
        mask_bits = _new(W, stream)((rows, mask_words_per_row(cols)), dtype=torch.int32)
    if W_pruned is None and want_pruned:
        W_pruned = _made(stream, W.device, lambda: W.new_empty_strided((rows, cols), (ld, 1)))
    if workspace is None:
        workspace = _made(stream, W.device, lambda: select_workspace(rows, cols, norm_axis, W.device))
    else:
        _workspace(workspace, W.device)
    code = load().dass_select_unstructured(W.data_ptr(), rows, cols, ld, _dtype_code(W), norm.data_ptr(), int(norm_axis),
                                           float(alpha), float(sparsity), int(compare_axis), _ptr(mask_bits),
                                           _ptr(W_pruned), workspace.data_ptr(), workspace.numel(), _stream(stream))
    _check(code, "dass_select_unstructured")
    return mask_bits, W_pruned


def selftest_wait_timeout(status_word: torch.Tensor, limit_us: int, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Launches the bounded-wait self-test; read the outcome with calib_status(status_word)."""
    if not status_word.is_cuda or status_word.dtype != torch.int32 or status_word.numel() < 1:
        raise ValueError("status_word must be a CUDA int32 tensor")
    _check(load().dass_selftest_wait_timeout(status_word.data_ptr(), int(limit_us), _stream(stream)),
           "dass_selftest_wait_timeout")


def feature_sumsq(X: torch.Tensor, sumsq: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """sumsq[j] += sum_t X[t,j]^2 (Eq. 1's squared input-feature norms). Returns sumsq (float64 [d])."""
    T, d, ldx = _matrix(X, "X")
    if sumsq is None:
        sumsq = _made(stream, X.device, lambda: X.new_zeros(d, dtype=torch.float64))
    if sumsq.dtype != torch.float64 or not sumsq.is_cuda or sumsq.numel() != d or not sumsq.is_contiguous():
        raise ValueError("sumsq must be a contiguous CUDA float64 tensor of d elements")
    need = ctypes.c_size_t(0)
    _check(load().dass_feature_workspace_bytes(T, d, ctypes.byref(need)), "dass_feature_workspace_bytes")
    if workspace is None:
        workspace = _new(X, stream)(need.value + 16, dtype=torch.uint8)
        off = (-workspace.data_ptr()) % 16
        workspace = workspace[off:off + need.value]
    else:
        _workspace(workspace, X.device)
    code = load().dass_feature_sumsq(X.data_ptr(), T, d, ldx, _dtype_code(X), sumsq.data_ptr(), workspace.data_ptr(),
                                     workspace.numel(), _stream(stream))
    _check(code, "dass_feature_sumsq")
    return sumsq


# ----------------------------------------------------------------------------- forward pass (Eq. 2, Eq. 3)

def mlp_forward_workspace_bytes(T: int, d: int, I: int, dtype: torch.dtype) -> Tuple[int, int]:
    """(smallest accepted, one-pass) workspace sizes of mlp_forward."""
    lo, full = ctypes.c_size_t(0), ctypes.c_size_t(0)
    code = load().dass_mlp_forward_workspace_bytes(int(T), int(d), int(I), BF16 if dtype == torch.bfloat16 else F32,
                                                   ctypes.byref(lo), ctypes.byref(full))
    _check(code, "dass_mlp_forward_workspace_bytes")
    return int(lo.value), int(full.value)


def mlp_forward_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """A 256-byte aligned uint8 CUDA tensor of nbytes."""
    buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf[off:off + nbytes]


def mlp_forward(X: torch.Tensor, Wg: torch.Tensor, Wu: torch.Tensor, Wd: torch.Tensor, act: int,
                Z: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Z = (act(X Wg^T) * (X Wu^T)) Wd^T in X's dtype, with the weights as given (pruned = zeros in place).

    Without ``workspace`` a one-pass workspace is allocated; a smaller one makes the call process the
    tokens in chunks.  The workspace's status word is read by calib_status(workspace)."""
    T, d, ldx = _matrix(X, "X")
    I, d2, ldw = _matrix(Wg, "Wg")
    I3, d3, ldw3 = _matrix(Wu, "Wu")
    d4, I4, ldd = _matrix(Wd, "Wd")
    if (d2, I3, d3, ldw3) != (d, I, d, ldw) or (d4, I4) != (d, I):
        raise ValueError("X [T x d], Wg / Wu [I x d] (same pitch) and Wd [d x I] must agree in d and I")
    if not (Wg.dtype == Wu.dtype == Wd.dtype == X.dtype):
        raise ValueError("X, Wg, Wu, Wd must have one dtype")
    if Z is None:
        Z = _new(X, stream)((T, d))
    Tz, dz, ldz = _matrix(Z, "Z")
    if (Tz, dz) != (T, d) or Z.dtype != X.dtype:
        raise ValueError("Z must be [T x d] in X's dtype")
    if workspace is None:
        nbytes = mlp_forward_workspace_bytes(T, d, I, X.dtype)[1]
        workspace = _made(stream, X.device, lambda: mlp_forward_workspace(nbytes, X.device))
    if not workspace.is_cuda or workspace.dtype != torch.uint8:
        raise ValueError("workspace must be a CUDA uint8 tensor (see mlp_forward_workspace)")
    code = load().dass_mlp_forward(X.data_ptr(), T, ldx, Wg.data_ptr(), Wu.data_ptr(), I, d, ldw,
                                   Wd.data_ptr(), ldd, _dtype_code(X), int(act), Z.data_ptr(), ldz,
                                   workspace.data_ptr(), workspace.numel(), _stream(stream))
    _check(code, "dass_mlp_forward")
    return Z


# ----------------------------------------------------------------------------- mixture of experts
#
# These calls are made once per layer and decode step, so what they do on the host is kept short: one pass over each
# tensor's shape and strides, outputs from new_empty, the stream by its handle.

_CODES = {torch.bfloat16: BF16, torch.float32: F32}


def _code(t: torch.Tensor) -> int:
    code = _CODES.get(t.dtype)
    return _dtype_code(t) if code is None else code


def _rows(t: torch.Tensor, name: str) -> Tuple[int, int, int]:
    """(rows, columns, pitch) of a row-major CUDA matrix of any pitch; a single row, or none, has the pitch of its length."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D row-major tensor (unit stride along columns)")
    rows, cols = t.shape
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{name} must be a 2-D row-major tensor (unit stride along columns)")
    return rows, cols, ld if rows > 1 or ld > cols else cols


def _same(t: torch.Tensor, name: str, shape: Tuple[int, ...], dtype: torch.dtype, device: torch.device) -> int:
    """Checks a dense tensor and returns its address."""
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")
    return t.data_ptr()


def _like(t: torch.Tensor, name: str, rows: int, cols: int, X: torch.Tensor) -> int:
    """Checks a row-major matrix of X's dtype and device and returns its pitch."""
    r, c, ld = _rows(t, name)
    if r != rows or c != cols or t.dtype != X.dtype or t.device != X.device:
        raise ValueError(f"{name} must be a {X.dtype} matrix of shape {(rows, cols)} on {X.device}")
    return ld


def route_topk(logits: torch.Tensor, k: int, renormalise: bool = True, expert: Optional[torch.Tensor] = None,
               weight: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """The k experts with the highest logits of every row and their softmax weights: over the k chosen
    (``renormalise``) or over all experts.  logits [T x E]; returns (expert int32 [T x k], weight float32 [T x k])."""
    T, E, ld = _rows(logits, "logits")
    k, dt = int(k), _code(logits)
    new = _new(logits, stream)
    if expert is None:
        expert = new((T, max(k, 0)), dtype=torch.int32)
    else:
        _same(expert, "expert", (T, k), torch.int32, logits.device)
    if weight is None:
        weight = new((T, max(k, 0)), dtype=torch.float32)
    else:
        _same(weight, "weight", (T, k), torch.float32, logits.device)
    if T:
        _check(load().dass_route_topk(logits.data_ptr(), T, E, ld, dt, k, ROUTE_CHOSEN if renormalise else ROUTE_ALL,
                                      expert.data_ptr(), weight.data_ptr(), _stream_of(logits, stream)), "dass_route_topk")
    return expert, weight


def route_topk_backward(logits: torch.Tensor, expert: torch.Tensor, dweight: torch.Tensor, renormalise: bool = True,
                        dlogits: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The logits' gradient [T x E] from that of route_topk's weights (``expert`` as it returned them)."""
    T, E, ld = _rows(logits, "logits")
    dt = _code(logits)
    k = expert.shape[1] if expert.dim() == 2 else -1
    ids = _same(expert, "expert", (T, k), torch.int32, logits.device)
    dw = _same(dweight, "dweight", (T, k), torch.float32, logits.device)
    if dlogits is None:
        dlogits, ldd = _new(logits, stream)((T, E)), E
    else:
        ldd = _like(dlogits, "dlogits", T, E, logits)
    if T:
        _check(load().dass_route_topk_backward(logits.data_ptr(), T, E, ld, dt, k, ROUTE_CHOSEN if renormalise else ROUTE_ALL,
                                               ids, dw, dlogits.data_ptr(), ldd, _stream_of(logits, stream)), "dass_route_topk_backward")
    return dlogits


def expert_sort_workspace_bytes(T: int, k: int, E: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().dass_expert_sort_workspace_bytes(int(T), int(k), int(E), ctypes.byref(out)), "dass_expert_sort_workspace_bytes")
    return int(out.value)


def expert_sort(expert: torch.Tensor, E: int, offsets: Optional[torch.Tensor] = None, slot: Optional[torch.Tensor] = None,
                source: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None):
    """The stable order by expert of the choices ``expert`` [T x k] int32 (ids outside [0, E) are dropped).
    Returns (offsets [E + 1], slot [T x k], source [T * k]), all int32: see dass_expert_sort."""
    if expert.dim() != 2 or not expert.is_cuda:
        raise ValueError("expert must be a 2-D CUDA tensor [T x k]")
    (T, k), E, dev = expert.shape, int(E), expert.device
    ids = _same(expert, "expert", (T, k), torch.int32, dev)
    edges = E + 1 if E > 0 else 1
    new = _new(expert, stream)
    if offsets is None:
        offsets = new(edges)
    else:
        _same(offsets, "offsets", (edges,), torch.int32, dev)
    if slot is None:
        slot = new((T, k))
    else:
        _same(slot, "slot", (T, k), torch.int32, dev)
    if source is None:
        source = new(T * k)
    else:
        _same(source, "source", (T * k,), torch.int32, dev)
    if workspace is None:
        need = expert_sort_workspace_bytes(T, k, E)
        workspace = new(need, dtype=torch.uint8) if need else None
    else:
        _workspace(workspace, dev)
    _check(load().dass_expert_sort(ids, T, k, E, offsets.data_ptr(), slot.data_ptr(), source.data_ptr(),
                                   _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream_of(expert, stream)),
           "dass_expert_sort")
    return offsets, slot, source


def _slots(slot: torch.Tensor, weight: Optional[torch.Tensor], device: torch.device) -> Tuple[int, int]:
    if slot.dim() != 2:
        raise ValueError("slot must be the [T x k] tensor expert_sort returned")
    shape = slot.shape
    _same(slot, "slot", shape, torch.int32, device)
    if weight is not None:
        _same(weight, "weight", shape, torch.float32, device)
    return shape


def _rows_used(offsets: Optional[torch.Tensor], device: torch.device) -> Optional[int]:
    if offsets is None:
        return None
    n = offsets.numel()
    if n == 0:
        raise ValueError("offsets must be the [E + 1] tensor expert_sort returned")
    return _same(offsets, "offsets", (n,), torch.int32, device) + 4 * (n - 1)


def expert_gather(X: torch.Tensor, slot: torch.Tensor, offsets: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                  Xs: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Xs[slot[t,j]] = (weight[t,j] *) X[t], [T * k x d] unless ``Xs`` is given.  With ``offsets`` the rows past the
    last expert's are zeroed; without them rows that no slot names keep what they held."""
    Tx, d, ldx = _rows(X, "X")
    T, k = _slots(slot, weight, X.device)
    if Tx != T:
        raise ValueError("X and slot must have the same number of tokens")
    if Xs is None:
        rows, ldxs = T * k, d
        Xs = _new(X, stream)((rows, d))
    else:
        rows = Xs.shape[0]
        ldxs = _like(Xs, "Xs", rows, d, X)
    _check(load().dass_expert_gather(X.data_ptr(), T, d, ldx, _code(X), slot.data_ptr(), k, _ptr(weight),
                                     _rows_used(offsets, X.device), Xs.data_ptr(), rows, ldxs, _stream_of(X, stream)), "dass_expert_gather")
    return Xs


def expert_combine(Ys: torch.Tensor, slot: torch.Tensor, weight: Optional[torch.Tensor] = None,
                   residual: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Y[t] = residual[t] + sum_j weight[t,j] * Ys[slot[t,j]]  (``Y`` may be the residual itself)."""
    rows, d, ldys = _rows(Ys, "Ys")
    T, k = _slots(slot, weight, Ys.device)
    ldr = _like(residual, "residual", T, d, Ys) if residual is not None else 0
    if Y is None:
        Y, ldy = _new(Ys, stream)((T, d)), d
    else:
        ldy = _like(Y, "Y", T, d, Ys)
    _check(load().dass_expert_combine(Ys.data_ptr(), rows, d, ldys, _code(Ys), slot.data_ptr(), T, k, _ptr(weight),
                                      _ptr(residual), ldr, Y.data_ptr(), ldy, _stream_of(Ys, stream)), "dass_expert_combine")
    return Y


def expert_gather_backward(dXs: torch.Tensor, slot: torch.Tensor, dX: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Gradient of the (unweighted) gather: dX[t] = sum_j dXs[slot[t,j]]."""
    return expert_combine(dXs, slot, Y=dX, stream=stream)


def expert_combine_backward(dY: torch.Tensor, Ys: torch.Tensor, slot: torch.Tensor, weight: Optional[torch.Tensor] = None,
                            offsets: Optional[torch.Tensor] = None, dYs: Optional[torch.Tensor] = None,
                            dweight: Optional[torch.Tensor] = None, want_rows: bool = True, want_weight: bool = True,
                            stream: Optional[torch.cuda.Stream] = None):
    """Gradients of expert_combine: (dYs [rows x d] or None, dweight float32 [T x k] or None).  With ``offsets`` the
    rows of dYs past the last expert's are zeroed."""
    Ty, d, lddy = _rows(dY, "dY")
    T, k = _slots(slot, weight, dY.device)
    rows = Ys.shape[0]
    ldys = _like(Ys, "Ys", rows, d, dY)
    if Ty != T:
        raise ValueError("dY and slot must have the same number of tokens")
    lddys = d
    new = _new(dY, stream)
    if dYs is not None:
        lddys = _like(dYs, "dYs", rows, d, dY)
    elif want_rows:
        dYs = new((rows, d))
    if dweight is not None:
        _same(dweight, "dweight", (T, k), torch.float32, dY.device)
    elif want_weight:
        dweight = new((T, k), dtype=torch.float32)
    dt = _code(dY)
    if T or (dYs is not None and offsets is not None):
        _check(load().dass_expert_combine_backward(dY.data_ptr(), T, d, lddy, Ys.data_ptr(), rows, ldys, dt, slot.data_ptr(), k,
                                                   _ptr(weight), _rows_used(offsets, dY.device), _ptr(dYs), lddys, _ptr(dweight),
                                                   _stream_of(dY, stream)), "dass_expert_combine_backward")
    return dYs, dweight


def linear(X: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor] = None, act: int = ACT_NONE,
           W_up: Optional[torch.Tensor] = None, bias_up: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
           offsets: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Y = act(X W^T + bias) [* (X W_up^T + bias_up)] + residual, rounded once to X's dtype.

    Dense: X [T x K], W (and W_up) [N x K], bias [N].  Per expert, with ``offsets`` (expert_sort's, on the device): W
    (and W_up) [G x N x K], bias [G x N]; rows offsets[g] .. offsets[g+1]-1 use matrix g, rows of no expert give zeros.
    ``Y`` may be the residual itself."""
    T, K, ldx = _rows(X, "X")
    dtype, device = X.dtype, X.device
    shape, strides = W.shape, W.stride()
    if len(shape) != (2 if offsets is None else 3) or shape[-1] != K or W.dtype != dtype or W.device != device or (strides[-1] != 1 and K > 1):
        raise ValueError(f"W must be a row-major {'[N x K]' if offsets is None else '[G x N x K]'} tensor of X's dtype and device")
    N = shape[-2]
    ldw = strides[-2] if N > 1 or strides[-2] > K else K
    if W_up is not None and (W_up.shape != shape or W_up.stride() != strides or W_up.dtype != dtype or W_up.device != device):
        raise ValueError("W_up must have W's shape, strides, dtype and device")
    if offsets is None:
        groups, group_stride, edges, per = 1, 0, None, (N,)
    else:
        groups, group_stride = shape[0], strides[0]
        edges, per = _same(offsets, "offsets", (groups + 1,), torch.int32, device), (groups, N)
    b = _same(bias, "bias", per, dtype, device) if bias is not None else None
    if bias_up is not None and W_up is None:
        raise ValueError("bias_up goes with W_up")
    bu = _same(bias_up, "bias_up", per, dtype, device) if bias_up is not None else None
    ldr = _like(residual, "residual", T, N, X) if residual is not None else 0
    dt = _code(X)
    if Y is None:
        Y, ldy = _new(X, stream)((T, N)), N
    else:
        ldy = _like(Y, "Y", T, N, X)
    if T:
        _check(load().dass_linear(X.data_ptr(), T, K, ldx, W.data_ptr(), _ptr(W_up), N, ldw, group_stride, b, bu, act, _ptr(residual), ldr,
                                  Y.data_ptr(), ldy, dt, edges, groups, _stream_of(X, stream)), "dass_linear")
    return Y


def linear_status(stream: Optional[torch.cuda.Stream] = None) -> None:
    """Waits for the stream and raises if a bounded wait inside a linear kernel ran out on the current device since the last
    query."""
    _check(load().dass_linear_status(_stream(stream)), "dass_linear_status")
