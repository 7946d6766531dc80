"""Thin binding of librobe.so: argument marshalling only.

Every function has the name of the C entry point it calls (see include/robe.h) and does
no arithmetic of the method itself.  torch is used for device memory and streams.  There
is no fallback: if a shared library is missing or does not load, importing this module
raises.

The calls of a training or serving loop go through `_robe_py` (csrc/robe_py.cpp), which reads the
tensors in native code: through ctypes alone a call costs about 8 us of Python, more than the
smallest lookups take on the GPU.  It declines, without calling anything, what is not plainly the
right kind of argument; the ctypes path below then makes the call or says what is wrong.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# ROBE_LIBRARY names another build of the same library to load instead (the index-check build
# librobe_debug.so); it is not a fallback: a name that does not exist fails below like the default.
LIB_PATH = os.environ.get("ROBE_LIBRARY") or os.path.join(_HERE, "librobe.so")

ROBE_OK = 0
ROBE_ERR_INVALID_ARG = -1
ROBE_ERR_NO_ARRAY = -2
ROBE_ERR_WORKSPACE = -3
ROBE_ERR_CUDA = -4
ROBE_ERR_UNSUPPORTED = -5

ROBE_F32 = 0
ROBE_BF16 = 1

ROBE_OPT_SIGN = 1
ROBE_OPT_BWD_MODE = 2
ROBE_OPT_VALIDATE = 3
ROBE_OPT_FWD_KERNEL = 4
ROBE_OPT_BWD_KERNEL = 5
ROBE_OPT_INDEX_TYPE = 6
ROBE_OPT_ARRAY_L2_KEEP = 8

ROBE_I64 = 0
ROBE_I32 = 1
ROBE_OPT_BAG_LAYOUT = 7
ROBE_BAGS_SAMPLE_MAJOR = 0
ROBE_BAGS_TABLE_MAJOR = 1

ROBE_BWD_ATOMIC = 0
ROBE_BWD_DETERMINISTIC = 1
ROBE_BWD_BINNED = 2

ROBE_STATIC_SCRATCH_BYTES = 32 << 20

ROBE_NORM_RMS = 0
ROBE_NORM_LAYER = 1
ROBE_GATE_NONE = 0
ROBE_GATE_ROW = 1
ROBE_GATE_VECTOR = 2

ROBE_DBG_SELFTEST = 99

EXPORTS = [
    "robe_create", "robe_destroy", "robe_set_option", "robe_attach_array",
    "robe_get_hash_constants", "robe_forward", "robe_backward_workspace_bytes", "robe_backward",
    "robe_set_status_word", "robe_last_device_status", "robe_status_string",
    "robe_backward_deterministic_static", "robe_backward_adam",
    "robe_forward_keep", "robe_backward_kept", "robe_apply_sgd",
    "robe_debug_status", "robe_debug_selftest", "robe_backward_adagrad",
    "robe_dropout", "robe_bias_create", "robe_bias_destroy", "robe_bias_num_buckets", "robe_bias_get_edges",
    "robe_bias_forward", "robe_bias_backward_workspace_bytes", "robe_bias_backward",
    "robe_residual_forward", "robe_residual_backward_workspace_bytes", "robe_residual_backward",
]

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2108_02191_b200.build` "
        "(there is no CPU or PyTorch fallback)")

_lib = C.CDLL(LIB_PATH)
from . import _robe_py as _native  # noqa: E402  (built beside the library; missing: ImportError)

_vp, _i64, _u64, _u32 = C.c_void_p, C.c_int64, C.c_uint64, C.c_uint32
_lib.robe_create.argtypes = [C.POINTER(_vp), _u64, _u32, _u32, _u32, _u64]
_lib.robe_destroy.argtypes = [_vp]
_lib.robe_set_option.argtypes = [_vp, C.c_int, _i64]
_lib.robe_attach_array.argtypes = [_vp, _vp, C.c_int]
_lib.robe_get_hash_constants.argtypes = [_vp, C.POINTER(_u64)]
_lib.robe_forward.argtypes = [_vp, _vp, _vp, _i64, _i64, _vp, _vp]
_lib.robe_forward_keep.argtypes = [_vp, _vp, _vp, _i64, _i64, _vp, _vp, C.c_size_t, _vp]
_lib.robe_backward_workspace_bytes.argtypes = [_vp, _i64, _i64]
_lib.robe_backward_workspace_bytes.restype = C.c_size_t
_lib.robe_backward.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp, C.c_float, _vp, C.c_size_t, _vp]
_lib.robe_backward_kept.argtypes = list(_lib.robe_backward.argtypes)
_lib.robe_backward_deterministic_static.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp, C.c_float, _vp]
_lib.robe_backward_adam.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp, _vp, C.c_float, C.c_float,
                                    C.c_float, C.c_float, _i64, _vp, C.c_size_t, _vp]
_lib.robe_apply_sgd.argtypes = [_vp, _vp, C.c_float, C.c_int, _vp]
_lib.robe_backward_adagrad.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp, C.c_float, C.c_float, _vp,
                                       C.c_size_t, _vp]
_lib.robe_debug_status.argtypes = [_vp]
_lib.robe_debug_selftest.argtypes = [_vp]
_lib.robe_set_status_word.argtypes = [_vp, _vp]
_lib.robe_last_device_status.argtypes = [_vp, _vp]


class _BiasCtx(C.Structure):
    """What a position-bias handle points to (opaque)."""


_BiasHandle = C.POINTER(_BiasCtx)


class _Residual(C.Structure):
    """robe_residual_t"""
    _fields_ = [("rows", _i64), ("d", _i64), ("dtype", C.c_int), ("norm", C.c_int), ("eps", C.c_float),
                ("scale", C.c_float), ("gate", C.c_int), ("gate_rows", _i64), ("p", C.c_float), ("seed", _u64),
                ("offset", _u64), ("step", _vp)]


_rows = [_vp, _i64]  # a matrix: pointer and leading dimension
_lib.robe_dropout.argtypes = _rows * 2 + [_i64, _i64, C.c_int, C.c_float, _u64, _u64, _vp, _vp]
_lib.robe_bias_create.argtypes = [C.POINTER(_BiasHandle), _u32, _u32, C.c_int]
_lib.robe_bias_destroy.argtypes = [_BiasHandle]
_lib.robe_bias_num_buckets.argtypes = [_BiasHandle]
_lib.robe_bias_get_edges.argtypes = [_BiasHandle, C.POINTER(_i64)]
_lib.robe_bias_forward.argtypes = [_BiasHandle] + _rows + [_u32] + [_i64] * 4 + [_vp, C.c_int] + _rows + [C.c_int, _vp]
_lib.robe_bias_backward_workspace_bytes.argtypes = [_BiasHandle, _u32, _i64, _i64, _i64]
_lib.robe_bias_backward_workspace_bytes.restype = C.c_size_t
_lib.robe_bias_backward.argtypes = ([_BiasHandle] + _rows + [_u32] + [_i64] * 4 + [_vp, C.c_int, C.c_int] + _rows
                                    + [_vp, C.c_size_t, _vp])
_lib.robe_residual_forward.argtypes = [C.POINTER(_Residual)] + _rows * 3 + [_vp, _vp] + _rows * 2 + [_vp]
_lib.robe_residual_backward_workspace_bytes.argtypes = [_i64, _i64, _i64]
_lib.robe_residual_backward_workspace_bytes.restype = C.c_size_t
_lib.robe_residual_backward.argtypes = ([C.POINTER(_Residual)] + _rows * 5 + [_vp, _vp] + _rows * 3
                                        + [_vp, _vp, _vp, C.c_size_t, _vp])
_lib.robe_status_string.argtypes = [C.c_int]
_lib.robe_status_string.restype = C.c_char_p
for _name in EXPORTS:
    if not _name.endswith("workspace_bytes") and _name != "robe_status_string":
        getattr(_lib, _name).restype = C.c_int

_native.set_calls(_vp, *(C.cast(getattr(_lib, _name), _vp).value for _name in (
    "robe_set_option", "robe_forward", "robe_forward_keep", "robe_backward", "robe_backward_kept",
    "robe_backward_adam", "robe_backward_adagrad", "robe_apply_sgd")))
_native.set_row_calls(_BiasHandle, *(C.cast(getattr(_lib, _name), _vp).value for _name in (
    "robe_dropout", "robe_bias_num_buckets", "robe_bias_forward", "robe_bias_backward", "robe_residual_forward",
    "robe_residual_backward")))
_NOT_TAKEN = 1  # from _native: nothing was called


class RobeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {robe_status_string(status)} ({status})")


def _check(status: int, where: str) -> None:
    if status != ROBE_OK:
        raise RobeError(status, where)


def _dev_ptr(t, dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


def _stream_ptr(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ids_ptr(t):
    """Device pointer of an id tensor: int64, or int32 for a handle set to ROBE_I32 (the handle's
    option says which the library reads; nothing is converted here)."""
    if t.dtype not in (torch.int64, torch.int32):
        raise TypeError(f"indices must be int64 or int32, got {t.dtype}")
    return _dev_ptr(t)


def _state_index_type(h, indices) -> None:
    """Tells the handle which element type the id tensor of the coming call has (the C ABI
    states it through ROBE_OPT_INDEX_TYPE, a tensor carries it in its dtype)."""
    _check(_lib.robe_set_option(h, ROBE_OPT_INDEX_TYPE,
                                ROBE_I32 if indices.dtype == torch.int32 else ROBE_I64), "robe_set_option")


def robe_status_string(status: int) -> str:
    return _lib.robe_status_string(status).decode()


def robe_create(M: int, Z: int, d: int, num_tables: int, hash_seed: int):
    h = _vp()
    if not (0 <= M < 2**64 and 0 <= Z < 2**32 and 0 <= d < 2**32 and 0 <= num_tables < 2**32):
        raise RobeError(ROBE_ERR_INVALID_ARG, "robe_create")
    _check(_lib.robe_create(C.byref(h), M, Z, d, num_tables, hash_seed & (2**64 - 1)), "robe_create")
    return h


def robe_destroy(h) -> None:
    _check(_lib.robe_destroy(h), "robe_destroy")


def robe_set_option(h, key: int, value: int) -> None:
    _check(_lib.robe_set_option(h, key, value), "robe_set_option")


def robe_attach_array(h, array: torch.Tensor) -> None:
    if array.dtype == torch.float32:
        dt = ROBE_F32
    elif array.dtype == torch.bfloat16:
        dt = ROBE_BF16
    else:
        raise TypeError("array must be float32 or bfloat16")
    _check(_lib.robe_attach_array(h, _dev_ptr(array), dt), "robe_attach_array")


def robe_get_hash_constants(h):
    out = (_u64 * 9)()
    _check(_lib.robe_get_hash_constants(h, out), "robe_get_hash_constants")
    return [int(v) for v in out]


def robe_forward(h, indices, offsets, batch: int, out, stream=None) -> None:
    rc = _native.forward(h, indices, offsets, batch, out, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_forward")
    _state_index_type(h, indices)
    _check(_lib.robe_forward(h, _ids_ptr(indices), _dev_ptr(offsets, torch.int64),
                             batch, indices.numel(), _dev_ptr(out, torch.float32),
                             _stream_ptr(stream)), "robe_forward")


def robe_forward_keep(h, indices, offsets, batch: int, out, workspace, stream=None) -> None:
    """robe_forward that also leaves the block starts in `workspace` for robe_backward_kept."""
    rc = _native.forward_keep(h, indices, offsets, batch, out, workspace, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_forward_keep")
    _state_index_type(h, indices)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.robe_forward_keep(h, _ids_ptr(indices), _dev_ptr(offsets, torch.int64),
                                  batch, indices.numel(), _dev_ptr(out, torch.float32),
                                  _dev_ptr(workspace), ws_bytes, _stream_ptr(stream)), "robe_forward_keep")


def robe_backward_workspace_bytes(h, batch: int, nnz: int) -> int:
    return int(_lib.robe_backward_workspace_bytes(h, batch, nnz))


def robe_backward(h, grad_out, indices, offsets, batch: int, grad_array=None, lr: float = 0.0,
                  workspace=None, stream=None) -> None:
    rc = _native.backward(h, grad_out, indices, offsets, batch, grad_array, lr, workspace, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_backward")
    _state_index_type(h, indices)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.robe_backward(h, _dev_ptr(grad_out, torch.float32), _ids_ptr(indices),
                              _dev_ptr(offsets, torch.int64), batch, indices.numel(),
                              _dev_ptr(grad_array, torch.float32), lr, _dev_ptr(workspace),
                              ws_bytes, _stream_ptr(stream)), "robe_backward")


def robe_backward_kept(h, grad_out, indices, offsets, batch: int, grad_array=None, lr: float = 0.0,
                       workspace=None, stream=None) -> None:
    """robe_backward on the block starts that robe_forward_keep left in `workspace`."""
    rc = _native.backward_kept(h, grad_out, indices, offsets, batch, grad_array, lr, workspace, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_backward_kept")
    _state_index_type(h, indices)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.robe_backward_kept(h, _dev_ptr(grad_out, torch.float32), _ids_ptr(indices),
                                   _dev_ptr(offsets, torch.int64), batch, indices.numel(),
                                   _dev_ptr(grad_array, torch.float32), lr, _dev_ptr(workspace),
                                   ws_bytes, _stream_ptr(stream)), "robe_backward_kept")


def robe_backward_deterministic_static(h, grad_out, indices, offsets, batch: int, grad_array=None,
                                       lr: float = 0.0, stream=None) -> None:
    """Deterministic backward on the library's built-in scratch array, for callers that cannot
    allocate a workspace (include/robe.h has the limit and the sharing rules).  No tensor is
    created here: the arguments are passed through as they are."""
    _state_index_type(h, indices)
    _check(_lib.robe_backward_deterministic_static(
        h, _dev_ptr(grad_out, torch.float32), _ids_ptr(indices),
        _dev_ptr(offsets, torch.int64), batch, indices.numel(), _dev_ptr(grad_array, torch.float32),
        lr, _stream_ptr(stream)), "robe_backward_deterministic_static")


def robe_backward_adam(h, grad_out, indices, offsets, batch: int, m1, m2, lr: float, beta1: float,
                       beta2: float, eps: float, step: int, workspace, stream=None) -> None:
    rc = _native.backward_adam(h, grad_out, indices, offsets, batch, m1, m2, lr, beta1, beta2, eps, step,
                               workspace, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_backward_adam")
    _state_index_type(h, indices)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.robe_backward_adam(
        h, _dev_ptr(grad_out, torch.float32), _ids_ptr(indices), _dev_ptr(offsets, torch.int64), batch,
        indices.numel(), _dev_ptr(m1, torch.float32), _dev_ptr(m2, torch.float32), lr, beta1, beta2, eps,
        step, _dev_ptr(workspace), ws_bytes, _stream_ptr(stream)), "robe_backward_adam")


def robe_backward_adagrad(h, grad_out, indices, offsets, batch: int, sum_sq, lr: float, eps: float,
                          workspace, stream=None) -> None:
    rc = _native.backward_adagrad(h, grad_out, indices, offsets, batch, sum_sq, lr, eps, workspace, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_backward_adagrad")
    _state_index_type(h, indices)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.robe_backward_adagrad(
        h, _dev_ptr(grad_out, torch.float32), _ids_ptr(indices), _dev_ptr(offsets, torch.int64), batch,
        indices.numel(), _dev_ptr(sum_sq, torch.float32), lr, eps, _dev_ptr(workspace), ws_bytes,
        _stream_ptr(stream)), "robe_backward_adagrad")


def robe_apply_sgd(h, grad_array, lr: float, zero_grad: bool = True, stream=None) -> None:
    """Dense SGD apply of the data-parallel step: array <- fma(-lr, grad_array, array)."""
    rc = _native.apply_sgd(h, grad_array, lr, zero_grad, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_apply_sgd")
    _check(_lib.robe_apply_sgd(h, _dev_ptr(grad_array, torch.float32), lr, 1 if zero_grad else 0,
                               _stream_ptr(stream)), "robe_apply_sgd")


# ---- row operators: what a model does next with the rows.  Tensors are on the current device; a matrix is a tensor whose
# last dimension is contiguous and whose others collapse to one (a column slice of a wider one, for instance).

_TYPES = {torch.float32: ROBE_F32, torch.bfloat16: ROBE_BF16}


def _here(t, what, dtype=None):
    """A CUDA tensor of the current device (and element type)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what}: expected a CUDA tensor")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{what}: on {t.device}, but the current device is cuda:{torch.cuda.current_device()}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what}: expected {dtype}, got {t.dtype}")
    return t


def _matrix(t, what, dtype=None):
    """(pointer, leading dimension, rows, columns)"""
    _here(t, what, dtype)
    if t.dtype not in _TYPES:
        raise TypeError(f"{what}: expected float32 or bfloat16, got {t.dtype}")
    if t.dim() == 0:
        raise ValueError(f"{what}: expected a tensor of rows")
    cols = t.shape[-1]
    rows = t.numel() // cols if cols else 0
    if t.numel() == 0:
        return 0, cols, rows, cols
    if cols > 1 and t.stride(-1) != 1:
        raise ValueError(f"{what}: the last dimension is not contiguous")
    ld, span = cols, None
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if span is None:
            ld = stride
            if ld < cols:
                raise ValueError(f"{what}: rows overlap")
        elif stride != span:
            raise ValueError(f"{what}: the rows are not equally far apart")
        span = stride * size
    return t.data_ptr(), ld, rows, cols


def _matrix_like(t, what, dtype, rows, cols):
    """Pointer and leading dimension of a matrix of that type and size; of None: (None, 0)."""
    if t is None:
        return None, 0
    p, ld, r, c = _matrix(t, what, dtype)
    if (r, c) != (rows, cols):
        raise ValueError(f"{what}: {r} rows of {c}, expected {rows} of {cols}")
    return p, ld


def _vector(t, what, n, dtype=torch.float32):
    """Pointer of a contiguous vector of n elements; of None: None."""
    if t is None:
        return None
    _here(t, what, dtype)
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what}: expected {n} contiguous elements")
    return t.data_ptr()


def _workspace(t):
    """(pointer, bytes)"""
    if t is None:
        return None, 0
    if not _here(t, "workspace").is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor")
    return t.data_ptr(), t.numel() * t.element_size()


def _step_ptr(step):
    if step is None:
        return None
    if _here(step, "step").dtype not in (torch.int64, torch.uint64) or step.numel() != 1:
        raise TypeError("step: expected one int64 or uint64 element")
    return step.data_ptr()


def robe_dropout(x, out, p: float, seed: int, offset: int = 0, step=None, stream=None) -> None:
    """out = dropout of the rows x.  The gradient of the call is the same call on the gradient of `out`."""
    rc = _native.dropout(x, out, p, seed, offset, step, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_dropout")
    ptr, ld, rows, cols = _matrix(x, "x")
    out_ptr, out_ld = _matrix_like(out, "out", x.dtype, rows, cols)
    _check(_lib.robe_dropout(ptr, ld, out_ptr, out_ld, rows, cols, _TYPES[x.dtype], p, seed & (2**64 - 1),
                             offset & (2**64 - 1), _step_ptr(step), _stream_ptr(stream)), "robe_dropout")


def robe_bias_create(num_buckets: int, max_distance: int, two_sided: bool):
    b = _BiasHandle()
    if not (0 <= num_buckets < 2**32 and 0 <= max_distance < 2**32):
        raise RobeError(ROBE_ERR_INVALID_ARG, "robe_bias_create")
    _check(_lib.robe_bias_create(C.byref(b), num_buckets, max_distance, 1 if two_sided else 0), "robe_bias_create")
    return b


def robe_bias_destroy(b) -> None:
    _check(_lib.robe_bias_destroy(b), "robe_bias_destroy")


def robe_bias_num_buckets(b) -> int:
    n = int(_lib.robe_bias_num_buckets(b))
    _check(min(n, 0), "robe_bias_num_buckets")
    return n


def robe_bias_get_edges(b):
    """Smallest distance of each bucket."""
    out = (_i64 * robe_bias_num_buckets(b))()
    _check(_lib.robe_bias_get_edges(b, out), "robe_bias_get_edges")
    return [int(v) for v in out]


def _bias_matrix(t, what):
    """(pointer, leading dimension, batch, heads, queries, keys) of [batch, heads, queries, keys] or [heads, ..]."""
    if isinstance(t, torch.Tensor) and t.dim() not in (3, 4):
        raise ValueError(f"{what}: expected [batch, heads, queries, keys] or [heads, queries, keys]")
    p, ld, _, _ = _matrix(t, what)
    n, h, q, k = (1, *t.shape) if t.dim() == 3 else t.shape
    return p, ld, n, h, q, k


def _starts(q_start, batch):
    """(start of all, pointer to starts)"""
    if isinstance(q_start, torch.Tensor):
        return 0, _vector(q_start, "q_start", batch, torch.int64)
    if not -2**63 <= q_start < 2**63:  # (ctypes would take it modulo 2^64)
        raise ValueError(f"q_start: {q_start} is beyond 64 bits")
    return q_start, None


def robe_bias_forward(b, rows, out, q_start=0, causal: bool = False, stream=None) -> None:
    """out[n,h,i,j] = rows[bucket(j - (start_n + i)), h]; q_start an int or an int64 tensor of one start per sequence."""
    rc = _native.bias_forward(b, rows, out, q_start, causal, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_bias_forward")
    p, ld, n, h, q, k = _bias_matrix(out, "out")
    table, table_ld = _matrix_like(rows, "rows", torch.float32, robe_bias_num_buckets(b), h)
    start, starts = _starts(q_start, n)
    _check(_lib.robe_bias_forward(b, table, table_ld, h, n, q, k, start, starts, 1 if causal else 0, p, ld,
                                  _TYPES[out.dtype], _stream_ptr(stream)), "robe_bias_forward")


def robe_bias_backward_workspace_bytes(b, heads: int, batch: int, q_len: int, k_len: int) -> int:
    if not (0 <= heads < 2**32 and all(-2**63 <= n < 2**63 for n in (batch, q_len, k_len))):
        return 0
    return int(_lib.robe_bias_backward_workspace_bytes(b, heads, batch, q_len, k_len))


def robe_bias_backward(b, grad, grad_rows, workspace, q_start=0, causal: bool = False, stream=None) -> None:
    """grad_rows[b,h] = sum of grad[n,h,i,j] over bucket b."""
    rc = _native.bias_backward(b, grad, grad_rows, workspace, q_start, causal, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_bias_backward")
    p, ld, n, h, q, k = _bias_matrix(grad, "grad")
    table, table_ld = _matrix_like(grad_rows, "grad_rows", torch.float32, robe_bias_num_buckets(b), h)
    start, starts = _starts(q_start, n)
    _check(_lib.robe_bias_backward(b, p, ld, h, n, q, k, start, starts, 1 if causal else 0, _TYPES[grad.dtype], table,
                                   table_ld, *_workspace(workspace), _stream_ptr(stream)), "robe_bias_backward")


def _residual(x, gate, scale, norm, eps, p, seed, offset, step):
    """robe_residual_t of a call, x's matrix, the gate's (pointer, leading dimension) and (rows, columns)."""
    ptr, ld, rows, d = _matrix(x, "x")
    kind, gate_rows, gate_at, gate_size = ROBE_GATE_NONE, 0, (None, 0), (0, 0)
    if gate is not None:
        g_ptr, g_ld, g_rows, g_cols = _matrix(gate, "gate", x.dtype)
        if g_cols == d and g_rows and rows % g_rows == 0:
            kind, gate_rows = ROBE_GATE_VECTOR, max(1, rows // g_rows)
        elif g_cols == 1 and g_rows == rows:
            kind = ROBE_GATE_ROW
        elif rows == 0 and g_rows == 0:
            kind, gate_rows = ROBE_GATE_VECTOR, 1
        else:
            raise ValueError(f"gate: {g_rows} rows of {g_cols} for {rows} rows of {d}")
        gate_at, gate_size = (g_ptr, g_ld), (g_rows, g_cols)
    if norm not in (ROBE_NORM_RMS, ROBE_NORM_LAYER):
        raise RobeError(ROBE_ERR_INVALID_ARG, "norm")
    c = _Residual(rows, d, _TYPES[x.dtype], norm, eps, scale, kind, gate_rows, p, seed & (2**64 - 1),
                  offset & (2**64 - 1), _step_ptr(step))
    return c, (ptr, ld), gate_at, gate_size


def robe_residual_forward(x, residual, out, normed=None, w_post=None, w_pre=None, gate=None, scale: float = 1.0,
                          norm: int = ROBE_NORM_RMS, eps: float = 1e-6, p: float = 0.0, seed: int = 0, offset: int = 0,
                          step=None, stream=None) -> None:
    """out = residual + scale * gate * dropout(norm(x) w_post), normed = norm(out) w_pre.  gate: [rows, 1], [rows, d] or
    [rows / k, d] (k rows in turn share a vector)."""
    rc = _native.residual_forward(x, residual, out, normed, w_post, w_pre, gate, scale, norm, eps, p, seed, offset, step,
                                  stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_residual_forward")
    c, x_at, gate_at, _ = _residual(x, gate, scale, norm, eps, p, seed, offset, step)
    like = lambda t, what: _matrix_like(t, what, x.dtype, c.rows, c.d)
    _check(_lib.robe_residual_forward(C.byref(c), *x_at, *like(residual, "residual"), *gate_at,
                                      _vector(w_post, "w_post", c.d), _vector(w_pre, "w_pre", c.d), *like(out, "out"),
                                      *like(normed, "normed"), _stream_ptr(stream)), "robe_residual_forward")


def robe_residual_backward_workspace_bytes(rows: int, d: int, gates: int = 0) -> int:
    """gates: rows of a gate of [rows / k, d]; 0 for no gate or one of [rows, 1]."""
    if not all(-2**63 <= n < 2**63 for n in (rows, d, gates)):
        return 0
    return int(_lib.robe_residual_backward_workspace_bytes(rows, d, gates))


def robe_residual_backward(grad_out, grad_normed, x, out, grad_x, grad_residual=None, w_post=None, w_pre=None, gate=None,
                           grad_w_post=None, grad_w_pre=None, grad_gate=None, workspace=None, scale: float = 1.0,
                           norm: int = ROBE_NORM_RMS, eps: float = 1e-6, p: float = 0.0, seed: int = 0, offset: int = 0,
                           step=None, stream=None) -> None:
    """Gradients of robe_residual_forward from x, out and gate as that call had and left them."""
    rc = _native.residual_backward(grad_out, grad_normed, x, out, grad_x, grad_residual, w_post, w_pre, gate, grad_w_post,
                                   grad_w_pre, grad_gate, workspace, scale, norm, eps, p, seed, offset, step, stream)
    if rc != _NOT_TAKEN:
        return _check(rc, "robe_residual_backward")
    c, x_at, gate_at, gate_size = _residual(x, gate, scale, norm, eps, p, seed, offset, step)
    like = lambda t, what: _matrix_like(t, what, x.dtype, c.rows, c.d)
    if grad_gate is not None and gate is None:
        raise ValueError("grad_gate: there is no gate")
    _check(_lib.robe_residual_backward(
        C.byref(c), *like(grad_out, "grad_out"), *like(grad_normed, "grad_normed"), *x_at, *like(out, "out"), *gate_at,
        _vector(w_post, "w_post", c.d), _vector(w_pre, "w_pre", c.d), *like(grad_x, "grad_x"),
        *like(grad_residual, "grad_residual"), *_matrix_like(grad_gate, "grad_gate", x.dtype, *gate_size),
        _vector(grad_w_post, "grad_w_post", c.d), _vector(grad_w_pre, "grad_w_pre", c.d), *_workspace(workspace),
        _stream_ptr(stream)), "robe_residual_backward")
    if c.rows == 0 and grad_gate is not None and grad_gate.numel() > 0:
        # gate vectors of no rows each, which the C ABI (rows / gate_rows of them) does not know of: everything dropped is zeros
        p_gate, ld, rows, cols = _matrix(grad_gate, "grad_gate")
        _check(_lib.robe_dropout(p_gate, ld, p_gate, ld, rows, cols, c.dtype, 1.0, 0, 0, None, _stream_ptr(stream)),
               "robe_residual_backward")


def robe_debug_status(stream=None) -> int:
    """Index-check build only: the first recorded ROBE_DBG_* code (0 = none), cleared by the call;
    ROBE_ERR_UNSUPPORTED (-5) from the release library."""
    return int(_lib.robe_debug_status(_stream_ptr(stream)))


def robe_debug_selftest(stream=None) -> int:
    return int(_lib.robe_debug_selftest(_stream_ptr(stream)))


def robe_set_status_word(h, word) -> None:
    _check(_lib.robe_set_status_word(h, _dev_ptr(word, torch.int32)), "robe_set_status_word")


def robe_last_device_status(h, stream=None) -> int:
    return int(_lib.robe_last_device_status(h, _stream_ptr(stream)))


def raw():
    """The ctypes library object itself, for callers that drive the C ABI with raw addresses
    (the host-side argument tests do)."""
    return _lib
