"""Thin ctypes binding of libmfet.so: same names as include/mfet.h, argument
marshalling only. Every step of the lookup path runs in the library's CUDA
kernels; if the library is missing this module raises at import instead of
falling back to anything else.

Pointers may be given as torch tensors (their data_ptr is taken), numpy arrays
(host arguments), or plain integers.
"""
from __future__ import annotations

import ctypes as C
import os
from operator import index
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# MFET_LIBRARY selects another build of the same library (the bounds-checked one, libmfet_checked.so)
LIB_PATH = os.environ.get("MFET_LIBRARY") or os.path.join(_HERE, "libmfet.so")

F32, F16, BF16, INT4, MXFP4 = 0, 1, 2, 3, 4
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU, ACT_SIGMOID = 0, 1, 2, 3, 4
POOL_SUM, POOL_MEAN, POOL_WSUM = 0, 1, 2
LOC_DEVICE, LOC_HOST = 0, 1
VAL_NORMAL, VAL_GRID = 0, 1
OPT_GROUP_POLICY = 1
OPT_TILE = 2
OPT_PROFILE = 3
OPT_STAGE_IDS = 4
OPT_OVERLAP_LAUNCHES = 5
OK = 0
ERR_INVALID_ARG, ERR_NOT_REGISTERED, ERR_ALIGNMENT, ERR_UNSUPPORTED_DIM = -1, -2, -3, -4
ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = -5, -6, -7
DEV_ROW_RANGE, DEV_OFFSETS, DEV_CAPACITY, DEV_BOUNDS, DEV_STALLED = 1, 2, 4, 8, 16

EXPORTS = [
    "mfet_row_bytes", "mfet_tables_create", "mfet_tables_destroy", "mfet_host_tables_register",
    "mfet_hash_ids", "mfet_embedding_bag_forward", "mfet_dedup_rows", "mfet_cache_bytes",
    "mfet_cache_build", "mfet_workspace_bytes", "mfet_set_workspace", "mfet_host_io_bytes",
    "mfet_embedding_bag_forward_host", "mfet_table_fill", "mfet_query_status", "mfet_set_option",
    "mfet_launch_count", "mfet_status_string", "mfet_dedup_rows_static", "mfet_profile_read", "mfet_host_path_counts", "mfet_tables_set_version", "mfet_tables_version",
    "mfet_host_prefetch", "mfet_embedding_bag_backward", "mfet_embedding_bag_forward_host_async",
    "mfet_host_path_result", "mfet_host_fetch_rows",
    "mfet_grad_clip_bytes", "mfet_grad_clip", "mfet_rows_write", "mfet_rows_read", "mfet_mx4_code_bytes",
    "mfet_mx4_scale_bytes", "mfet_mx4_quantize", "mfet_mx4_matmul", "mfet_mx4_linear_bytes", "mfet_mx4_linear",
    "mfet_layer_norm", "mfet_layer_norm_backward_bytes", "mfet_layer_norm_backward", "mfet_gated_linear_bytes", "mfet_gated_linear",
    "mfet_gated_linear_backward_bytes", "mfet_gated_linear_backward", "mfet_orthogonalize_bytes", "mfet_orthogonalize",
]
BATCH_IDS_ARE_ROWS, BATCH_PREFETCHED = 1, 2
STATIC_DEDUP_MAX_IDS = 262144


class TableDesc(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_uint64), ("dim", C.c_uint32), ("dtype", C.c_uint32),
                ("location", C.c_uint32), ("flags", C.c_uint32), ("hash_seed", C.c_uint64),
                ("row_stride_bytes", C.c_uint64)]


class BatchShape(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_features", C.c_int32), ("n_slots", C.c_int32),
                ("flags", C.c_int32), ("slot_feature", C.POINTER(C.c_int32)), ("out_ld", C.c_int64)]


class Grad(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64),
                ("n_rows", C.c_void_p), ("dtype", C.c_uint32), ("flags", C.c_uint32)]


if not os.path.exists(LIB_PATH):
    raise ImportError("libmfet.so is missing: build it with `python -m paper_2508_05700_b200.build` "
                      "(there is no fallback path)")
_lib = C.CDLL(LIB_PATH)
try:
    from . import _fastcall  # noqa: E402  (built with the library, for the Python that built it)
except ImportError:
    _fastcall = None

_P = C.c_void_p
_lib.mfet_row_bytes.restype = C.c_uint64
_lib.mfet_row_bytes.argtypes = [C.c_uint32, C.c_uint32]
_lib.mfet_status_string.restype = C.c_char_p
_lib.mfet_status_string.argtypes = [C.c_int]
_lib.mfet_tables_create.argtypes = [C.POINTER(TableDesc), C.c_int32, C.c_int32, C.POINTER(_P)]
_lib.mfet_tables_destroy.argtypes = [_P]
_lib.mfet_host_tables_register.argtypes = [_P, C.c_int32, _P, C.c_uint64, C.c_uint32]
_lib.mfet_hash_ids.argtypes = [_P, C.c_int32, _P, C.c_int64, _P, _P]
_lib.mfet_embedding_bag_forward.argtypes = [_P, C.POINTER(BatchShape), _P, _P, _P, _P, _P, _P, _P]
_lib.mfet_dedup_rows.argtypes = [_P, _P, C.c_int64, _P, _P, _P, C.c_int64, _P]
_lib.mfet_dedup_rows_static.argtypes = [C.c_int32, _P, C.c_int64, _P, _P, _P, C.c_int64, _P]
_lib.mfet_cache_bytes.argtypes = [_P, C.c_int32, C.c_int64, C.POINTER(C.c_uint64)]
_lib.mfet_cache_build.argtypes = [_P, C.c_int32, _P, C.c_int64, _P, C.c_uint64, _P]
_lib.mfet_workspace_bytes.argtypes = [_P, C.c_int64, C.POINTER(C.c_uint64)]
_lib.mfet_set_workspace.argtypes = [_P, _P, C.c_uint64, C.c_int64]
_lib.mfet_host_io_bytes.argtypes = [_P, C.POINTER(BatchShape), _P, C.c_int64, C.POINTER(C.c_uint64)]
_lib.mfet_embedding_bag_forward_host.argtypes = [_P, C.POINTER(BatchShape), _P, _P, _P, C.c_int64, _P, _P, _P,
                                                 _P, C.c_uint64, _P]
_lib.mfet_embedding_bag_forward_host_async.argtypes = _lib.mfet_embedding_bag_forward_host.argtypes
_lib.mfet_table_fill.argtypes = [_P, C.c_uint64, C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint64, C.c_uint64,
                                 C.c_uint32, _P]
_lib.mfet_query_status.argtypes = [_P, C.POINTER(C.c_uint32), C.c_int32]
_lib.mfet_set_option.argtypes = [_P, C.c_int32, C.c_int64]
_lib.mfet_profile_read.argtypes = [_P, C.POINTER(C.c_float)]
_lib.mfet_host_path_counts.argtypes = [_P, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
_lib.mfet_host_path_result.argtypes = [_P, _P, _P, _P, C.c_int64]
_lib.mfet_host_fetch_rows.argtypes = [_P, C.c_int32, _P, C.c_int64, _P, _P]
_lib.mfet_tables_set_version.argtypes = [_P, C.c_uint64]
_lib.mfet_tables_version.argtypes = [_P, C.POINTER(C.c_uint64)]
_lib.mfet_host_prefetch.argtypes = [_P, C.POINTER(BatchShape), _P, _P, _P, _P]
_lib.mfet_embedding_bag_backward.argtypes = [_P, C.POINTER(BatchShape), _P, _P, _P, _P, _P, _P, C.c_int32, _P, _P, _P, _P]
_lib.mfet_launch_count.argtypes = [_P, C.POINTER(C.c_uint64)]
_BYTES = ("mfet_grad_clip_bytes", "mfet_mx4_code_bytes", "mfet_mx4_scale_bytes", "mfet_mx4_linear_bytes", "mfet_layer_norm_backward_bytes",
          "mfet_gated_linear_bytes", "mfet_gated_linear_backward_bytes", "mfet_orthogonalize_bytes")
for _n in _BYTES:
    getattr(_lib, _n).restype = C.c_uint64
    getattr(_lib, _n).argtypes = [C.c_int32] if _n == "mfet_grad_clip_bytes" else [C.c_int64] * (3 if "gated" in _n else 2)
for _n in EXPORTS:
    if _n not in ("mfet_row_bytes", "mfet_status_string") + _BYTES:
        getattr(_lib, _n).restype = C.c_int


class MfetError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (%d)" % (where, status_string(status), status))


def _ptr(x) -> Optional[int]:
    """Address of a torch tensor, numpy array, ctypes pointer or int; None stays NULL."""
    if x is None or type(x) is int:
        return x
    try:
        return x.data_ptr()  # what most arguments are: no look-up ahead of the call
    except AttributeError:
        pass
    if isinstance(x, int):
        return int(x)
    if isinstance(x, np.ndarray):
        return int(x.ctypes.data)
    return C.cast(x, C.c_void_p).value


def _check(status: int, where: str) -> None:
    if status != OK:
        raise MfetError(status, where)


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a), dtype=np.int32)


def status_string(status: int) -> str:
    return _lib.mfet_status_string(status).decode()


def row_bytes(dim: int, dtype: int) -> int:
    return int(_lib.mfet_row_bytes(dim, dtype))


def make_shape(batch: int, n_features: int, slot_feature, out_ld: int = 0, ids_are_rows: bool = False):
    """(BatchShape, keep-alive) for the forward calls."""
    sf = _i32(slot_feature)
    sh = BatchShape(batch, n_features, int(sf.size), 1 if ids_are_rows else 0,
                    sf.ctypes.data_as(C.POINTER(C.c_int32)), out_ld)
    return sh, sf


def mfet_tables_create(descs: Sequence[TableDesc], device: int = 0) -> int:
    arr = (TableDesc * len(descs))(*descs)
    h = _P()
    _check(_lib.mfet_tables_create(arr, len(descs), device, C.byref(h)), "mfet_tables_create")
    return h.value


def mfet_tables_destroy(h) -> None:
    _check(_lib.mfet_tables_destroy(h), "mfet_tables_destroy")


def mfet_host_tables_register(h, table_id: int, host_ptr, nbytes: int, flags: int = 0) -> None:
    _check(_lib.mfet_host_tables_register(h, table_id, _ptr(host_ptr), nbytes, flags), "mfet_host_tables_register")


def mfet_hash_ids(h, table_id: int, ids, n: int, rows_out, stream=None) -> None:
    _check(_lib.mfet_hash_ids(h, table_id, _ptr(ids), n, _ptr(rows_out), _ptr(stream)), "mfet_hash_ids")


def mfet_embedding_bag_forward(h, shape: BatchShape, ids, offsets, weights, table_ids, pooling, out,
                               stream=None) -> None:
    ti, po = _i32(table_ids), _i32(pooling)
    _check(_lib.mfet_embedding_bag_forward(h, C.byref(shape), _ptr(ids), _ptr(offsets), _ptr(weights),
                                           ti.ctypes.data, po.ctypes.data, _ptr(out), _ptr(stream)),
           "mfet_embedding_bag_forward")


def mfet_dedup_rows(h, rows, n: int, uniq, inverse, n_unique, max_row: int = 0, stream=None) -> None:
    _check(_lib.mfet_dedup_rows(h, _ptr(rows), n, _ptr(uniq), _ptr(inverse), _ptr(n_unique), max_row,
                                _ptr(stream)), "mfet_dedup_rows")


def mfet_dedup_rows_static(device: int, rows, n: int, uniq, inverse, n_unique, max_row: int = 0, stream=None) -> None:
    """Dedup on the library's built-in scratch array: no workspace, no allocation anywhere
    (n <= STATIC_DEDUP_MAX_IDS). Calls on one GPU share that array and must not overlap."""
    _check(_lib.mfet_dedup_rows_static(device, _ptr(rows), n, _ptr(uniq), _ptr(inverse), _ptr(n_unique), max_row,
                                       _ptr(stream)), "mfet_dedup_rows_static")


def mfet_cache_bytes(h, table_id: int, n: int) -> int:
    b = C.c_uint64()
    _check(_lib.mfet_cache_bytes(h, table_id, n, C.byref(b)), "mfet_cache_bytes")
    return int(b.value)


def mfet_cache_build(h, table_id: int, rows_sorted: np.ndarray, cache_mem, cache_bytes: int, stream=None) -> None:
    rs = np.ascontiguousarray(rows_sorted, dtype=np.int64)
    _check(_lib.mfet_cache_build(h, table_id, rs.ctypes.data, rs.size, _ptr(cache_mem), cache_bytes, _ptr(stream)),
           "mfet_cache_build")


def mfet_workspace_bytes(h, max_ids: int) -> int:
    b = C.c_uint64()
    _check(_lib.mfet_workspace_bytes(h, max_ids, C.byref(b)), "mfet_workspace_bytes")
    return int(b.value)


def mfet_set_workspace(h, dev_ptr, nbytes: int, max_ids: int) -> None:
    _check(_lib.mfet_set_workspace(h, _ptr(dev_ptr), nbytes, max_ids), "mfet_set_workspace")


def mfet_host_io_bytes(h, shape: BatchShape, table_ids, nnz: int) -> int:
    ti = _i32(table_ids)
    b = C.c_uint64()
    _check(_lib.mfet_host_io_bytes(h, C.byref(shape), ti.ctypes.data, nnz, C.byref(b)), "mfet_host_io_bytes")
    return int(b.value)


def mfet_embedding_bag_forward_host(h, shape: BatchShape, ids_host, offsets_host, weights_host, nnz: int,
                                    table_ids, pooling, out_host, dev_io, dev_io_bytes: int, stream=None) -> None:
    ti, po = _i32(table_ids), _i32(pooling)
    _check(_lib.mfet_embedding_bag_forward_host(h, C.byref(shape), _ptr(ids_host), _ptr(offsets_host),
                                                _ptr(weights_host), nnz, ti.ctypes.data, po.ctypes.data,
                                                _ptr(out_host), _ptr(dev_io), dev_io_bytes, _ptr(stream)),
           "mfet_embedding_bag_forward_host")


def mfet_embedding_bag_forward_host_async(h, shape: BatchShape, ids_host, offsets_host, weights_host, nnz: int,
                                          table_ids, pooling, out_host, dev_io, dev_io_bytes: int, stream=None) -> None:
    ti, po = _i32(table_ids), _i32(pooling)
    _check(_lib.mfet_embedding_bag_forward_host_async(h, C.byref(shape), _ptr(ids_host), _ptr(offsets_host),
                                                      _ptr(weights_host), nnz, ti.ctypes.data, po.ctypes.data,
                                                      _ptr(out_host), _ptr(dev_io), dev_io_bytes, _ptr(stream)),
           "mfet_embedding_bag_forward_host_async")


def mfet_table_fill(data, row0: int, n_rows: int, dim: int, dtype: int, row_stride_bytes: int, value_key: int,
                    value_mode: int = VAL_NORMAL, stream=None) -> None:
    _check(_lib.mfet_table_fill(_ptr(data), row0, n_rows, dim, dtype, row_stride_bytes,
                                value_key & (2**64 - 1), value_mode, _ptr(stream)), "mfet_table_fill")


def mfet_query_status(h, clear: bool = False) -> int:
    bits = C.c_uint32()
    _check(_lib.mfet_query_status(h, C.byref(bits), 1 if clear else 0), "mfet_query_status")
    return int(bits.value)


def mfet_set_option(h, option: int, value: int) -> None:
    _check(_lib.mfet_set_option(h, option, value), "mfet_set_option")


def mfet_profile_read(h):
    """(dedup_ms, fetch_ms, pool_ms) of the last forward call's host-table path."""
    ms = (C.c_float * 3)()
    _check(_lib.mfet_profile_read(h, ms), "mfet_profile_read")
    return tuple(float(x) for x in ms)


def mfet_host_path_counts(h):
    """(distinct rows, distinct rows missing from the cache) of the last host-table slot."""
    a, b = C.c_int64(), C.c_int64()
    _check(_lib.mfet_host_path_counts(h, C.byref(a), C.byref(b)), "mfet_host_path_counts")
    return int(a.value), int(b.value)


def mfet_host_path_result(h, uniq, src, miss_rows, capacity: int) -> None:
    _check(_lib.mfet_host_path_result(h, _ptr(uniq), _ptr(src), _ptr(miss_rows), capacity), "mfet_host_path_result")


def mfet_host_fetch_rows(h, table_id: int, rows, n: int, dst, stream=None) -> None:
    _check(_lib.mfet_host_fetch_rows(h, table_id, _ptr(rows), n, _ptr(dst), _ptr(stream)), "mfet_host_fetch_rows")


def mfet_tables_set_version(h, version: int) -> None:
    _check(_lib.mfet_tables_set_version(h, version & (2**64 - 1)), "mfet_tables_set_version")


def mfet_tables_version(h) -> int:
    v = C.c_uint64()
    _check(_lib.mfet_tables_version(h, C.byref(v)), "mfet_tables_version")
    return int(v.value)


def mfet_host_prefetch(h, shape: BatchShape, ids, offsets, table_ids, stream=None) -> None:
    ti = _i32(table_ids)
    _check(_lib.mfet_host_prefetch(h, C.byref(shape), _ptr(ids), _ptr(offsets), ti.ctypes.data, _ptr(stream)),
           "mfet_host_prefetch")


def mfet_embedding_bag_backward(h, shape: BatchShape, ids, offsets, weights, table_ids, pooling, grad_out, slot: int,
                                grad_rows, grad_vals, n_rows, stream=None) -> None:
    ti, po = _i32(table_ids), _i32(pooling)
    _check(_lib.mfet_embedding_bag_backward(h, C.byref(shape), _ptr(ids), _ptr(offsets), _ptr(weights), ti.ctypes.data,
                                            po.ctypes.data, _ptr(grad_out), slot, _ptr(grad_rows), _ptr(grad_vals),
                                            _ptr(n_rows), _ptr(stream)), "mfet_embedding_bag_backward")


def mfet_launch_count(h) -> int:
    n = C.c_uint64()
    _check(_lib.mfet_launch_count(h, C.byref(n)), "mfet_launch_count")
    return int(n.value)


_DTYPES = {}  # torch dtype -> MFET_*, filled as dtypes are met


def dtype_of(t) -> int:
    """MFET_F32 / F16 / BF16 of a torch tensor."""
    d = _DTYPES.get(t.dtype)
    if d is None:
        d = {"torch.float32": F32, "torch.float16": F16, "torch.bfloat16": BF16}.get(str(t.dtype))
        if d is None:
            raise MfetError(ERR_INVALID_ARG, "dtype_of(%s)" % t.dtype)
        _DTYPES[t.dtype] = d
    return d


def make_grads(src, dst, counts=None):
    """The list of gradient tensors of mfet_grad_clip, to be kept and used for every step: `src` and `dst` (entries may be
    None, or the source itself) are torch tensors of one or two dimensions whose last one is dense and whose rows do not overlap
    (an expanded tensor is refused: make it contiguous first); counts: dense i64 tensor on their device with the number of
    live rows of every tensor, or None. The list keeps the tensors alive and goes on using their memory: a program whose
    gradients are new tensors in every step (zero_grad(set_to_none=True)) makes a new list in every step."""
    if len(src) != len(dst):
        raise MfetError(ERR_INVALID_ARG, "make_grads: %d tensors and %d destinations" % (len(src), len(dst)))
    if counts is not None:
        elsewhere = {t.device for t in src} - {counts.device}
        if str(counts.dtype) != "torch.int64" or not counts.is_contiguous() or counts.numel() < len(src) or elsewhere:
            raise MfetError(ERR_INVALID_ARG, "make_grads: counts is not a dense int64 tensor of %d entries beside the gradients" % len(src))
    arr = (Grad * max(len(src), 1))()
    for i, (a, b) in enumerate(zip(src, dst)):
        if b is not None and (b.dtype != a.dtype or b.shape != a.shape or b.stride() != a.stride() or b.device != a.device):
            raise MfetError(ERR_INVALID_ARG, "make_grads: tensor %d and its destination differ in type, shape, strides or device" % i)
        two = a if a.dim() == 2 else a.reshape(1, -1) if a.is_contiguous() else None
        if two is None or (two.shape[1] > 1 and two.stride(1) != 1):
            raise MfetError(ERR_INVALID_ARG, "make_grads: tensor %d is not rows of neighbouring elements" % i)
        rows, cols = two.shape
        if rows > 1 and two.stride(0) < cols:  # an expanded tensor: its stride of 0 would mean `cols` to the library
            raise MfetError(ERR_INVALID_ARG, "make_grads: rows of tensor %d share memory" % i)
        ld = two.stride(0) if rows > 1 else cols
        arr[i] = Grad(_ptr(a), _ptr(b), rows, cols, ld, None if counts is None else _ptr(counts) + 8 * i, dtype_of(a), 0)
    arr.tensors = (list(src), list(dst), counts)  # what the addresses point at lives as long as the list
    return arr, len(src)


def mfet_grad_clip_bytes(n_grads: int) -> int:
    return int(_lib.mfet_grad_clip_bytes(n_grads))


def mfet_mx4_code_bytes(rows: int, k: int) -> int:
    return int(_lib.mfet_mx4_code_bytes(rows, k))


def mfet_mx4_scale_bytes(rows: int, k: int) -> int:
    return int(_lib.mfet_mx4_scale_bytes(rows, k))


def mfet_mx4_linear_bytes(m: int, k: int) -> int:
    return int(_lib.mfet_mx4_linear_bytes(m, k))


def mfet_layer_norm_backward_bytes(rows: int, cols: int) -> int:
    return int(_lib.mfet_layer_norm_backward_bytes(rows, cols))


def mfet_gated_linear_bytes(m: int, n: int, k: int) -> int:
    return int(_lib.mfet_gated_linear_bytes(m, n, k))


def mfet_gated_linear_backward_bytes(m: int, n: int, k: int) -> int:
    return int(_lib.mfet_gated_linear_backward_bytes(m, n, k))


def mfet_orthogonalize_bytes(rows: int, cols: int) -> int:
    return int(_lib.mfet_orthogonalize_bytes(rows, cols))


def mfet_orthogonalize(g, dtype: int, ld: int, rows: int, cols: int, coefficients, steps: int, scale: float, out, out_dtype: int, out_ld: int,
                       scratch, scratch_bytes: int, status=None, stream=None) -> None:
    """coefficients: None, or a, b, c of every step (any host sequence or array of 3 * steps numbers)."""
    if coefficients is not None:
        coefficients = np.ascontiguousarray(coefficients, dtype=np.float32)
        if coefficients.size != 3 * steps:
            _fail(ERR_INVALID_ARG, "mfet_orthogonalize")
    _orthogonalize(g, dtype, ld, rows, cols, None if coefficients is None else coefficients.ctypes.data, steps, scale, out, out_dtype, out_ld,
                   scratch, scratch_bytes, status, stream)


# The calls that a step makes many times go through a small extension instead of ctypes (csrc/fastcall.c). It is built for one version of
# Python; another one makes the same calls, with the same names, arguments and errors, through ctypes. Per call: the kinds of its arguments
# (as in fastcall.c) and how many of them have to be given.
_FAST = {"mfet_grad_clip": ("ofppzp", 5), "mfet_rows_write": ("bpippuipp", 7), "mfet_rows_read": ("bpippuipp", 7),
         "mfet_mx4_quantize": ("puiiippp", 7), "mfet_mx4_matmul": ("ppippiipupuipp", 12), "mfet_mx4_linear": ("puiippiipupuipzpp", 15),
         "mfet_layer_norm": ("puiiippfpuip", 11), "mfet_layer_norm_backward": ("puiiipfpuipipppzp", 16),
         "mfet_gated_linear": ("puiipipiiiupipzpp", 15), "mfet_gated_linear_backward": ("puiipipiiiupipipipipzpp", 21),
         "mfet_orthogonalize": ("puiiipdfpuipzpp", 13)}
_KINDS = {"p": C.c_void_p, "b": C.c_void_p, "f": C.c_float, "i": C.c_int64, "u": C.c_uint32, "d": C.c_int32, "z": C.c_uint64}
_RANGES = {"i": (-2**63, 2**63), "u": (0, 2**32), "d": (-2**31, 2**31), "z": (0, 2**63)}


def _fail(status: int, where: str) -> None:
    raise MfetError(status, where)


def _through_ctypes(name: str):
    kinds, least = _FAST[name]
    in_c = kinds.replace("o", "bd")  # a list of gradients: its memory and its length
    size = C.sizeof(Grad if "o" in kinds else TableDesc)
    fn = getattr(_lib, name)
    fn.argtypes = [_KINDS[k] for k in in_c]

    def convert(kind, v):
        if kind == "p":
            return v if v is None or isinstance(v, int) else v.data_ptr()
        if kind == "f":
            return float(v)
        if kind == "b":
            return v if v is None else np.frombuffer(v, np.uint8).ctypes.data
        v, (lo, hi) = index(v), _RANGES[kind]
        if not lo <= v < hi:
            _fail(ERR_INVALID_ARG, name)
        return v

    def call(*args):
        if not least <= len(args) <= len(kinds):
            raise TypeError("%s takes %d to %d arguments (%d given)" % (name, least, len(kinds), len(args)))
        args += (None,) * (len(kinds) - len(args))
        if "o" in kinds:
            if not isinstance(args[0], tuple) or len(args[0]) != 2:
                raise TypeError("%s: what make_grads gave is wanted" % name)
            args = args[0] + args[1:]
        lent = args[0]
        if "b" in in_c and lent is not None and memoryview(lent).nbytes < size * (args[1] if "o" in kinds else 1):
            _fail(ERR_INVALID_ARG, name)
        _check(fn(*[convert(k, v) for k, v in zip(in_c, args)]), name)
    call.__name__ = name
    return call


if _fastcall is not None:
    _fastcall.bind(_fail, *(C.cast(getattr(_lib, _n), C.c_void_p).value for _n in _FAST))
(mfet_grad_clip, mfet_rows_write, mfet_rows_read, mfet_mx4_quantize, mfet_mx4_matmul, mfet_mx4_linear, mfet_layer_norm, mfet_layer_norm_backward,
 mfet_gated_linear, mfet_gated_linear_backward, _orthogonalize) = (
    _through_ctypes(_n) if _fastcall is None else getattr(_fastcall, _n) for _n in _FAST)
