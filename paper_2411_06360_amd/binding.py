"""ctypes binding of ``librsr.so`` (C ABI: ``include/rsr.h``).  Marshalling only.

Host arrays are numpy; device buffers are anything with ``data_ptr()`` (torch tensors on the
GPU) or a plain integer address; streams are an integer ``hipStream_t`` (``None``/0 = default,
``torch.cuda.current_stream().cuda_stream`` for torch's).
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "librsr.so"
_lib: Optional[ctypes.CDLL] = None

RSR_OK = 0


class RsrError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"rsr error {code}: {message}")
        self.code = code
        self.message = message


class RsrInfo(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
        ("k", ctypes.c_int32), ("parts", ctypes.c_int32),
        ("nblocks", ctypes.c_int64),
        ("last_block_width", ctypes.c_int32), ("lo_bits", ctypes.c_int32), ("hi_bits", ctypes.c_int32),
        ("stored_rows", ctypes.c_int64), ("segments", ctypes.c_int64), ("work_units", ctypes.c_int64),
        ("index_bytes", ctypes.c_int64), ("segment_bytes", ctypes.c_int64),
        ("schedule_bytes", ctypes.c_int64), ("table_bytes", ctypes.c_int64),
        ("device", ctypes.c_int32), ("compute_units", ctypes.c_int32),
        ("row_tiles", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]

    def as_dict(self) -> dict:
        return {name: getattr(self, name) for name, _ in self._fields_}


# numpy view of the 32-byte unit descriptors (csrc/rsr_format.h)
UNIT_DTYPE = np.dtype(
    [
        ("stream_off", "<u4"), ("block", "<u4"), ("window", "<u2"), ("part", "u1"), ("npos", "u1"),
        ("units_in_block", "<u2"), ("index_in_block", "<u2"), ("slot0", "<u2"), ("reserved0", "<u2"),
        ("nrows", "<u4"), ("nheads", "<u4"), ("nentries", "<u4"),
    ]
)
assert UNIT_DTYPE.itemsize == 32


def lib_path() -> str:
    """The built library, next to this file."""
    return os.path.join(HERE, _LIB_NAME)


def load(path: Optional[str] = None) -> ctypes.CDLL:
    """Load the built library (once per process; `path` names another build of the same sources and
    only counts on the first call).  Never builds and never falls back to anything else."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or lib_path()
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} is missing: the HIP library has not been built "
            "(run `python -m paper_2411_06360_amd.build`); there is no CPU fallback"
        )
    # One HIP runtime per process: PyTorch ships its own libamdhip64 and owns the device buffers
    # and streams handed to this library, so its copy has to be the one that is already loaded
    # when librsr.so resolves its dependency (same SONAME).  Loading in the other order leaves
    # two runtimes in the process and torch then finds no GPU.
    import torch  # noqa: F401

    L = ctypes.CDLL(path)
    vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    L.rsr_preprocess.argtypes = [vp, i64, i64, ci]
    L.rsr_preprocess.restype = vp
    L.rsr_preprocess_device.argtypes = [vp, i64, i64, ci]
    L.rsr_preprocess_device.restype = vp
    L.rsr_matvec.argtypes = [vp, vp, vp, ci, vp]
    L.rsr_matvec.restype = ci
    L.rsr_matvec_i8.argtypes = [vp, vp, vp, ci, vp]
    L.rsr_matvec_i8.restype = ci
    L.rsr_matvec_multi.argtypes = [vp, ci, ci, vp]
    L.rsr_matvec_multi.restype = ci
    L.rsr_matvec_multi_i8.argtypes = [vp, ci, ci, vp]
    L.rsr_matvec_multi_i8.restype = ci
    L.rsr_set_step2.argtypes = [vp, ci]
    L.rsr_set_step2.restype = ci
    L.rsr_model_k.argtypes = [i64, ci, ci]
    L.rsr_model_k.restype = ci
    L.rsr_autotune_k.argtypes = [vp, i64, i64, ci, ci, ci, ci, ci, ctypes.POINTER(ci), vp]
    L.rsr_autotune_k.restype = ci
    L.rsr_destroy.argtypes = [vp]
    L.rsr_destroy.restype = None
    L.rsr_last_error.argtypes = []
    L.rsr_last_error.restype = ctypes.c_char_p
    L.rsr_info.argtypes = [vp, ctypes.POINTER(RsrInfo)]
    L.rsr_info.restype = ci
    L.rsr_export_block.argtypes = [vp, ci, i64, vp, vp]
    L.rsr_export_block.restype = ci
    L.rsr_host_pack.argtypes = [vp, i64, i64, ci]
    L.rsr_host_pack.restype = vp
    L.rsr_host_free.argtypes = [vp]
    L.rsr_host_free.restype = None
    L.rsr_host_info.argtypes = [vp, ctypes.POINTER(RsrInfo)]
    L.rsr_host_info.restype = ci
    L.rsr_host_export_block.argtypes = [vp, ci, i64, vp, vp]
    L.rsr_host_export_block.restype = ci
    L.rsr_host_streams.argtypes = ([vp, ci] + [ctypes.POINTER(vp), ctypes.POINTER(i64)] * 2 + [ctypes.POINTER(vp)]
                                   + [ctypes.POINTER(i64)] * 2)
    L.rsr_host_streams.restype = ci
    L.rsr_matvec_acc.argtypes = [vp, vp, vp, ctypes.c_float, ci, vp]
    L.rsr_matvec_acc.restype = ci
    L.rsr_matvec_acc_i8.argtypes = [vp, vp, vp, ctypes.c_int32, ci, vp]
    L.rsr_matvec_acc_i8.restype = ci
    L.rsr_qbit_preprocess.argtypes = [vp, i64, i64, ci, ci]
    L.rsr_qbit_preprocess.restype = vp
    L.rsr_qbit_matvec.argtypes = [vp, vp, vp, ci, vp]
    L.rsr_qbit_matvec.restype = ci
    L.rsr_qbit_matvec_i8.argtypes = [vp, vp, vp, ci, vp]
    L.rsr_qbit_matvec_i8.restype = ci
    L.rsr_qbit_planes.argtypes = [vp]
    L.rsr_qbit_planes.restype = ci
    L.rsr_qbit_table_bytes.argtypes = [vp]
    L.rsr_qbit_table_bytes.restype = i64
    L.rsr_qbit_destroy.argtypes = [vp]
    L.rsr_qbit_destroy.restype = None
    L.rsr_dense_preprocess.argtypes = [vp, i64, i64]
    L.rsr_dense_preprocess.restype = vp
    L.rsr_dense_matvec.argtypes = [vp, vp, vp, ci, vp]
    L.rsr_dense_matvec.restype = ci
    L.rsr_dense_matvec_i8.argtypes = [vp, vp, vp, ci, vp]
    L.rsr_dense_matvec_i8.restype = ci
    L.rsr_dense_matvec_static.argtypes = [vp, vp, vp, ci, vp]
    L.rsr_dense_matvec_static.restype = ci
    L.rsr_dense_table_bytes.argtypes = [vp]
    L.rsr_dense_table_bytes.restype = i64
    L.rsr_dense_destroy.argtypes = [vp]
    L.rsr_dense_destroy.restype = None
    L.rsr_tree_attention_workspace.argtypes = [vp, vp, ci]
    L.rsr_tree_attention_workspace.restype = i64
    L.rsr_tree_attention.argtypes = [vp, vp, vp, i64, vp, vp, i64, vp, i64, ci, ci, ctypes.c_float, vp, i64, vp]
    L.rsr_tree_attention.restype = ci
    L.rsr_cache_slots.argtypes = [vp, vp, ci, vp, ci, ci, vp, vp, vp, vp, i64, vp, vp, vp]
    L.rsr_cache_slots.restype = ci
    L.rsr_cache_slots_bounded.argtypes = [vp, vp, ci, vp, ci, ci, vp, i64, vp, vp, vp, i64, vp, vp, vp]
    L.rsr_cache_slots_bounded.restype = ci
    L.rsr_cache_append.argtypes = [vp, vp, vp, i64, i64, ci, vp, vp, i64, vp]
    L.rsr_cache_append.restype = ci
    L.rsr_tree_masks.argtypes = [vp, vp, ci, ci, vp, vp, vp]
    L.rsr_tree_masks.restype = ci
    L.rsr_head_rotate.argtypes = [vp, vp, i64, ci, vp, i64, ci, ci, vp, i64, vp, i64, vp, i64, ci, vp]
    L.rsr_head_rotate.restype = ci
    L.rsr_sample_workspace.argtypes = [i64, i64]
    L.rsr_sample_workspace.restype = i64
    L.rsr_sample.argtypes = [vp, i64, i64, i64, ci, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
    L.rsr_sample.restype = ci
    L.rsr_tree_keep.argtypes = [vp, vp, vp, vp, ci, ci, vp, vp, vp, vp, vp]
    L.rsr_tree_keep.restype = ci
    _lib = L
    return L


def rsr_last_error() -> str:
    return (load().rsr_last_error() or b"").decode("utf-8", "replace")


def _check(code: int) -> None:
    if code != RSR_OK:
        raise RsrError(code, rsr_last_error())


def _host_matrix(A) -> np.ndarray:
    A = np.asarray(A)
    if A.dtype != np.int8:
        raise TypeError("A must be int8")
    if A.ndim != 2:
        raise ValueError("A must be 2-D (rows x cols)")
    return np.ascontiguousarray(A)


def _addr(x) -> int:
    if type(x) is int:
        return x
    if x is None:
        return 0
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr())
    return int(x)


def rsr_preprocess(A, k: int) -> int:
    """``A``: host int8 array ``rows x cols``.  Returns the handle (an integer address)."""
    A = _host_matrix(A)
    h = load().rsr_preprocess(A.ctypes.data, A.shape[0], A.shape[1], int(k))
    if not h:
        raise RsrError(-1, rsr_last_error())
    return int(h)


def rsr_preprocess_device(A_dev, rows: int, cols: int, k: int) -> int:
    """``A_dev``: device int8 buffer ``rows x cols`` (row-major).  Returns the handle."""
    h = load().rsr_preprocess_device(_addr(A_dev), int(rows), int(cols), int(k))
    if not h:
        raise RsrError(-1, rsr_last_error())
    return int(h)


def rsr_matvec(handle: int, v, out, batch: int, stream=None) -> None:
    """``v``: device float32 ``[batch][rows]``; ``out``: device float32 ``[batch][cols]``."""
    _check(load().rsr_matvec(handle, _addr(v), _addr(out), int(batch), _addr(stream)))


def rsr_matvec_i8(handle: int, v, out, batch: int, stream=None) -> None:
    """``v``: device int8 ``[batch][rows]``; ``out``: device int32 ``[batch][cols]``."""
    _check(load().rsr_matvec_i8(handle, _addr(v), _addr(out), int(batch), _addr(stream)))


def rsr_matvec_acc(handle: int, v, out, scale: float, batch: int, stream=None) -> None:
    """``out += scale * (v . A)`` on device float32 buffers."""
    _check(load().rsr_matvec_acc(handle, _addr(v), _addr(out), float(scale), int(batch), _addr(stream)))


def rsr_matvec_acc_i8(handle: int, v, out, scale: int, batch: int, stream=None) -> None:
    """``out += scale * (v . A)`` for device int8 activations and int32 results."""
    _check(load().rsr_matvec_acc_i8(handle, _addr(v), _addr(out), int(scale), int(batch), _addr(stream)))


# ---- q-bit matrices as weighted binary planes (include/rsr_qbit.h) ----
def rsr_qbit_preprocess(A, k: int, q: int) -> int:
    A = _host_matrix(A)
    h = load().rsr_qbit_preprocess(A.ctypes.data, A.shape[0], A.shape[1], int(k), int(q))
    if not h:
        raise RsrError(-1, rsr_last_error())
    return int(h)


def rsr_qbit_matvec(handle: int, v, out, batch: int, stream=None) -> None:
    _check(load().rsr_qbit_matvec(handle, _addr(v), _addr(out), int(batch), _addr(stream)))


def rsr_qbit_matvec_i8(handle: int, v, out, batch: int, stream=None) -> None:
    _check(load().rsr_qbit_matvec_i8(handle, _addr(v), _addr(out), int(batch), _addr(stream)))


def rsr_qbit_planes(handle: int) -> int:
    return int(load().rsr_qbit_planes(handle))


def rsr_qbit_table_bytes(handle: int) -> int:
    return int(load().rsr_qbit_table_bytes(handle))


def rsr_qbit_destroy(handle: Optional[int]) -> None:
    if handle:
        load().rsr_qbit_destroy(handle)


RSR_STEP2_FOLD, RSR_STEP2_PLAIN = 0, 1


def rsr_set_step2(handle: int, step2: int) -> None:
    """Step 2 as the RSR++ fold (RSR_STEP2_FOLD, default) or as the plain product (RSR_STEP2_PLAIN)."""
    _check(load().rsr_set_step2(handle, int(step2)))


def rsr_model_k(rows: int, k_min: int, k_max: int) -> int:
    k = load().rsr_model_k(int(rows), int(k_min), int(k_max))
    if k < 0:
        raise RsrError(k, rsr_last_error())
    return k


def rsr_autotune_k(A, batch: int, k_min: int, k_max: int, reps: int = 50, cold: bool = True):
    """Returns (best k, {k: microseconds per product})."""
    A = _host_matrix(A)
    best = ctypes.c_int(0)
    us = np.zeros(k_max - k_min + 1, dtype=np.float64)
    _check(load().rsr_autotune_k(A.ctypes.data, A.shape[0], A.shape[1], int(batch), int(k_min), int(k_max), int(reps),
                                 1 if cold else 0, ctypes.byref(best), us.ctypes.data))
    return int(best.value), {k_min + i: float(x) for i, x in enumerate(us)}


# ---- the bit-packed comparator (include/rsr_dense.h) ----
def rsr_dense_preprocess(A) -> int:
    A = _host_matrix(A)
    h = load().rsr_dense_preprocess(A.ctypes.data, A.shape[0], A.shape[1])
    if not h:
        raise RsrError(-1, rsr_last_error())
    return int(h)


def rsr_dense_matvec(handle: int, v, out, batch: int, stream=None) -> None:
    _check(load().rsr_dense_matvec(handle, _addr(v), _addr(out), int(batch), _addr(stream)))


def rsr_dense_matvec_i8(handle: int, v, out, batch: int, stream=None) -> None:
    _check(load().rsr_dense_matvec_i8(handle, _addr(v), _addr(out), int(batch), _addr(stream)))


def rsr_dense_matvec_static(handle: int, v, out, batch: int, stream=None) -> None:
    """As rsr_dense_matvec, with the partial sums in the library's static device buffer (allocates nothing)."""
    _check(load().rsr_dense_matvec_static(handle, _addr(v), _addr(out), int(batch), _addr(stream)))


def rsr_dense_table_bytes(handle: int) -> int:
    return int(load().rsr_dense_table_bytes(handle))


def rsr_dense_destroy(handle: Optional[int]) -> None:
    if handle:
        load().rsr_dense_destroy(handle)


# ---- the paged cache and the attention over it (include/rsr_cache.h) ----
RSR_F32, RSR_F16, RSR_BF16 = 0, 1, 2


class RsrCache(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
        ("dtype", ctypes.c_int32), ("pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]


class RsrStep(ctypes.Structure):
    _fields_ = [
        ("table", ctypes.c_void_p), ("held", ctypes.c_void_p), ("start", ctypes.c_void_p), ("mask", ctypes.c_void_p),
        ("requests", ctypes.c_int32), ("tokens", ctypes.c_int32), ("max_new", ctypes.c_int32), ("max_pages", ctypes.c_int32),
    ]


_dtypes: dict = {}  # torch's types to the header's (torch is imported by load(), not here)


def _dtype(x) -> int:
    code = _dtypes.get(x.dtype)
    if code is None:
        import torch

        _dtypes.update({torch.float32: RSR_F32, torch.float16: RSR_F16, torch.bfloat16: RSR_BF16})
        code = _dtypes.get(x.dtype)
        if code is None:
            raise TypeError(f"float32, float16 or bfloat16 wanted, not {x.dtype}")
    return code


def _rows(x, rows: int, width: int) -> int:
    """Stride of a 2-D tensor of `rows` rows of `width` elements that lie side by side (that of a single row means nothing)."""
    shape, stride = x.shape, x.stride()
    if len(shape) != 2 or shape[0] != rows or shape[1] != width or (stride[1] != 1 and width > 1):
        raise ValueError(f"a 2-D tensor with {rows} contiguous rows of {width} elements is wanted")
    return stride[0] if rows > 1 else width


_WHOLE: dict = {32: {"torch.int32"}, 64: {"torch.int64", "torch.uint64"}}  # names, and then the types themselves


def _whole(x, bits: int, count: int) -> int:
    """Address of a contiguous tensor of whole numbers of so many bits, with at least `count` elements."""
    dtype, known = x.dtype, _WHOLE[bits]
    if dtype not in known:
        if str(dtype) not in known:
            raise ValueError(f"a tensor of {bits}-bit integers is wanted, not {dtype}")
        known.add(dtype)
    if x.numel() < count or not x.is_contiguous():
        raise ValueError(f"a contiguous tensor of {count} integers is wanted")
    return x.data_ptr()


def make_cache(k, v) -> RsrCache:
    """rsr_cache_t of device tensors ``[pages][kv_heads][page_size][head_dim]`` (any strides between rows; keep the tensors alive)."""
    if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride() or k.stride(3) != 1:
        raise ValueError("two 4-D tensors of the same type, shape and strides, with contiguous rows, are wanted")
    pages, kv_heads, page_size, head_dim = k.shape
    return RsrCache(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2), _dtype(k), pages, page_size, kv_heads, head_dim, 0)


def make_step(table, held, start, tokens: int, max_new: int, mask=None) -> RsrStep:
    """rsr_step_t of device tensors: ``table [requests][max_pages]``, ``held [requests]``, ``start [requests+1]`` (int32) and
    ``mask [tokens]`` (64 bits) or None.  Keep the tensors alive; what they hold may change between calls."""
    requests = held.numel()
    if table.dim() != 2 or table.shape[0] != requests:
        raise ValueError("the table has a row for each request")
    return RsrStep(_whole(table, 32, 0), _whole(held, 32, 0), _whole(start, 32, requests + 1), None if mask is None else _whole(mask, 64, tokens),
                   requests, int(tokens), int(max_new), table.shape[1])


def rsr_tree_attention_workspace(cache: RsrCache, step: RsrStep, heads: int) -> int:
    """Bytes of workspace that rsr_tree_attention takes (zero it once)."""
    n = load().rsr_tree_attention_workspace(ctypes.addressof(cache), ctypes.addressof(step), int(heads))
    if n < 0:
        raise RsrError(n, rsr_last_error())
    return n


def rsr_tree_attention(cache: RsrCache, step: RsrStep, q, k, v, out, heads: int, scale: float, workspace, stream=None) -> None:
    """``q``, ``out``: device ``[tokens][heads * head_dim]``; ``k``, ``v``: ``[tokens][kv_heads * head_dim]`` (slices of wider rows
    will do), all float32 or of the cache's type; ``workspace``: device bytes that were zero at first."""
    dtype, tokens, width, kv_width = q.dtype, step.tokens, heads * cache.head_dim, cache.kv_heads * cache.head_dim
    kv_stride = _rows(k, tokens, kv_width)
    if out.dtype != dtype or k.dtype != dtype or v.dtype != dtype or _rows(v, tokens, kv_width) != kv_stride:
        raise ValueError("q, k, v and out must have one type, k and v one stride")
    code = (_lib or load()).rsr_tree_attention(
        ctypes.addressof(cache), ctypes.addressof(step), q.data_ptr(), _rows(q, tokens, width), k.data_ptr(), v.data_ptr(), kv_stride,
        out.data_ptr(), _rows(out, tokens, width), _dtypes.get(dtype) or _dtype(q), heads, scale, workspace.data_ptr(), workspace.nbytes, _addr(stream))
    if code:
        _check(code)


def rsr_cache_slots(held, add, table, page_size: int, free_pages, free_count, slots, start, now, free_left, stream=None) -> None:
    """Pages and slots for the next ``add[r]`` tokens of every request; all device int32, see the header.  A ``free_count`` above the
    length of ``free_pages`` is taken as that."""
    requests = held.numel()
    if table.dim() != 2 or table.shape[0] != requests:
        raise ValueError("the table has a row for each request")
    code = (_lib or load()).rsr_cache_slots_bounded(
        _whole(held, 32, 0), _whole(add, 32, requests), requests, _whole(table, 32, 0), table.shape[1], int(page_size), _whole(free_pages, 32, 0),
        free_pages.numel(), _whole(free_count, 32, 1), _whole(free_left, 32, 1), _whole(slots, 32, 0), slots.numel(), _whole(start, 32, requests + 1),
        _whole(now, 32, requests), _addr(stream))
    if code:
        _check(code)


def rsr_cache_append(cache: RsrCache, k, v, slots, rows=None, stream=None) -> None:
    """Row ``rows[i]`` (None: row ``i``) of ``k`` and ``v`` (``[nrows][kv_heads * head_dim]``) goes to ``slots[i]``."""
    count, nrows, width = slots.numel(), k.shape[0], cache.kv_heads * cache.head_dim
    stride = _rows(k, nrows, width)
    if k.dtype != v.dtype or _rows(v, nrows, width) != stride:
        raise ValueError("keys and values must have one type and stride")
    code = (_lib or load()).rsr_cache_append(
        ctypes.addressof(cache), k.data_ptr(), v.data_ptr(), stride, nrows, _dtypes.get(k.dtype) or _dtype(k),
        None if rows is None else _whole(rows, 32, count), _whole(slots, 32, 0), count, _addr(stream))
    if code:
        _check(code)


def rsr_tree_masks(parent, start, mask, depth, stream=None) -> None:
    """``mask`` (64 bits) and ``depth`` (int32) of the drafted tokens from their ``parent`` (int32, -1: hangs on the cache)."""
    tokens, requests = parent.numel(), start.numel() - 1
    code = (_lib or load()).rsr_tree_masks(_whole(parent, 32, 0), _whole(start, 32, 1), requests, tokens, _whole(mask, 64, tokens),
                                           _whole(depth, 32, tokens), _addr(stream))
    if code:
        _check(code)


# ---- both sides of the attention (include/rsr_decode.h) ----
class RsrRotary(ctypes.Structure):
    _fields_ = [
        ("frequency", ctypes.c_void_p), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
        ("norm", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("rotated", ctypes.c_int32), ("pairs", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]


_REAL: dict = {"torch.float32": set(), "torch.float64": set()}  # names, and the types themselves once they were seen


def _numbers(x, kind: str, count: int) -> Optional[int]:
    """Address of a contiguous tensor of floating-point numbers of that type, with at least `count` elements (None stays None)."""
    if x is None:
        return None
    dtype, known = x.dtype, _REAL[kind]
    if dtype not in known:
        if str(dtype) != kind:
            raise ValueError(f"a contiguous tensor of {count} numbers of {kind} is wanted, not {dtype}")
        known.add(dtype)
    if x.numel() < count or not x.is_contiguous():
        raise ValueError(f"a contiguous tensor of {count} numbers is wanted")
    return x.data_ptr()


def make_rotary(frequency, head_dim: int, eps=None, q_weight=None, k_weight=None, pairs: bool = False) -> RsrRotary:
    """rsr_rotary_t: ``frequency`` device float64, one for each pair of rotated dimensions (None: none are rotated); ``eps`` of the
    norm (None: heads are not normed); ``q_weight``, ``k_weight`` device float32 ``[head_dim]`` or None.  It keeps the tensors alive."""
    if eps is None and (q_weight is not None or k_weight is not None):
        raise ValueError("weights are the norm's: without eps there is none")
    rotated = 0 if frequency is None else 2 * frequency.numel()
    rotary = RsrRotary(_numbers(frequency, "torch.float64", 0), _numbers(q_weight, "torch.float32", head_dim), _numbers(k_weight, "torch.float32", head_dim),
                       0.0 if eps is None else eps, eps is not None, head_dim, rotated, bool(pairs), 0)
    rotary.tensors = frequency, q_weight, k_weight
    return rotary


def _heads(x, out, tokens: int, dim: int):
    """(stride, heads, stride of the results) of rows of heads; nothing of None."""
    if x is None or out is None:
        if x is not out:
            raise ValueError("rows and their results come together")
        return 0, 0, 0
    width = x.shape[-1]
    if width % dim:
        raise ValueError("a row is not a whole number of heads")
    return _rows(x, tokens, width), width // dim, _rows(out, tokens, width)


def rsr_head_rotate(rotary: RsrRotary, q, k, position, q_out, k_out, stream=None) -> None:
    """``q``, ``q_out``: device ``[tokens][heads * head_dim]``, ``k``, ``k_out``: ``[tokens][kv_heads * head_dim]`` (slices of wider rows
    will do; either pair may be None), inputs of one type and results of one type; ``position``: device int32 ``[tokens]``."""
    some, result = (q, q_out) if q is not None else (k, k_out)
    tokens, dim = position.numel(), rotary.head_dim
    q_stride, heads, q_out_stride = _heads(q, q_out, tokens, dim)
    k_stride, kv_heads, k_out_stride = _heads(k, k_out, tokens, dim)
    dtype, out_dtype = some.dtype, result.dtype
    if kv_heads and (k.dtype != dtype or k_out.dtype != out_dtype):
        raise ValueError("queries and keys must have one type, and their results")
    code = (_lib or load()).rsr_head_rotate(
        ctypes.addressof(rotary), _addr(q), q_stride, heads, _addr(k), k_stride, kv_heads, _dtypes.get(dtype) or _dtype(some), _whole(position, 32, 0), tokens,
        _addr(q_out), q_out_stride, _addr(k_out), k_out_stride, _dtypes.get(out_dtype) or _dtype(result), _addr(stream))
    if code:
        _check(code)


def rsr_sample_workspace(rows: int, columns: int) -> int:
    """Bytes of workspace that rsr_sample takes (zero it once)."""
    n = load().rsr_sample_workspace(int(rows), int(columns))
    if n < 0:
        raise RsrError(n, rsr_last_error())
    return n


def rsr_sample(logits, uniform, token, workspace, temperature=None, top_k=None, top_p=None, min_p=None, probability=None, kept=None, stream=None) -> None:
    """A ``token`` (device int32 ``[rows]``) for every row of ``logits`` (device ``[rows][columns]``, float32, float16 or bfloat16): the
    parameters are device tensors with one number a row (``top_k`` int32, the others float32) or None, ``uniform`` float32 in [0, 1);
    ``probability`` (float32) and ``kept`` (int32) are written unless they are None; ``workspace``: device bytes that were zero at first."""
    rows, columns = logits.shape
    real = "torch.float32"
    code = (_lib or load()).rsr_sample(
        logits.data_ptr(), rows, columns, _rows(logits, rows, columns), _dtypes.get(logits.dtype) or _dtype(logits), _numbers(temperature, real, rows),
        None if top_k is None else _whole(top_k, 32, rows), _numbers(top_p, real, rows), _numbers(min_p, real, rows), _numbers(uniform, real, rows),
        _whole(token, 32, rows), _numbers(probability, real, rows), None if kept is None else _whole(kept, 32, rows), workspace.data_ptr(), workspace.nbytes,
        _addr(stream))
    if code:
        _check(code)


def rsr_tree_keep(drafted, chosen, parent, start, rows, found, add, first, stream=None) -> None:
    """The paths of drafted trees that agree with what was chosen: ``rows`` and ``found`` (device int32, one a token), ``add`` (one a
    request) and ``first`` (one more), from ``drafted``, ``chosen`` and ``parent`` (None: chains) of the tokens; all int32."""
    tokens, requests = drafted.numel(), start.numel() - 1
    code = (_lib or load()).rsr_tree_keep(
        _whole(drafted, 32, 0), _whole(chosen, 32, tokens), None if parent is None else _whole(parent, 32, tokens), _whole(start, 32, 1), requests, tokens,
        _whole(rows, 32, tokens), _whole(found, 32, tokens), _whole(add, 32, requests), _whole(first, 32, requests + 1), _addr(stream))
    if code:
        _check(code)


class RsrJob(ctypes.Structure):
    _fields_ = [("h", ctypes.c_void_p), ("v", ctypes.c_void_p), ("out", ctypes.c_void_p)]


def make_jobs(jobs):
    """A C array of rsr_job from (handle, v, out) triples; keep it alive while it is in use."""
    arr = (RsrJob * len(jobs))()
    for i, (h, v, out) in enumerate(jobs):
        arr[i].h, arr[i].v, arr[i].out = int(h), _addr(v), _addr(out)
    return arr


def rsr_matvec_multi(jobs, batch: int, stream=None) -> None:
    """``jobs``: (handle, v, out) triples with float activations, or an array made by make_jobs."""
    arr = jobs if isinstance(jobs, ctypes.Array) else make_jobs(jobs)
    _check(load().rsr_matvec_multi(ctypes.cast(arr, ctypes.c_void_p), len(arr), int(batch), _addr(stream)))


def rsr_matvec_multi_i8(jobs, batch: int, stream=None) -> None:
    arr = jobs if isinstance(jobs, ctypes.Array) else make_jobs(jobs)
    _check(load().rsr_matvec_multi_i8(ctypes.cast(arr, ctypes.c_void_p), len(arr), int(batch), _addr(stream)))


def rsr_destroy(handle: Optional[int]) -> None:
    if handle:
        load().rsr_destroy(handle)


def rsr_info(handle: int) -> RsrInfo:
    info = RsrInfo()
    _check(load().rsr_info(handle, ctypes.byref(info)))
    return info


def _export(fn, handle: int, part: int, block: int, rows: int, width: int) -> Tuple[np.ndarray, np.ndarray]:
    sigma = np.empty(rows, dtype=np.int32)
    L = np.empty((1 << width) + 1, dtype=np.int32)
    _check(fn(handle, int(part), int(block), sigma.ctypes.data, L.ctypes.data))
    return sigma, L


def rsr_export_block(handle: int, part: int, block: int) -> Tuple[np.ndarray, np.ndarray]:
    """``(sigma, L)`` of one block, counted from 0; ``L`` has ``2^width + 1`` entries."""
    info = rsr_info(handle)
    width = info.last_block_width if block == info.nblocks - 1 else info.k
    return _export(load().rsr_export_block, handle, part, block, info.rows, width)


def rsr_host_pack(A, k: int) -> int:
    A = _host_matrix(A)
    x = load().rsr_host_pack(A.ctypes.data, A.shape[0], A.shape[1], int(k))
    if not x:
        raise RsrError(-1, rsr_last_error())
    return int(x)


def rsr_host_free(x: Optional[int]) -> None:
    if x:
        load().rsr_host_free(x)


def rsr_host_info(x: int) -> RsrInfo:
    info = RsrInfo()
    _check(load().rsr_host_info(x, ctypes.byref(info)))
    return info


def rsr_host_export_block(x: int, part: int, block: int) -> Tuple[np.ndarray, np.ndarray]:
    info = rsr_host_info(x)
    width = info.last_block_width if block == info.nblocks - 1 else info.k
    return _export(load().rsr_host_export_block, x, part, block, info.rows, width)


def rsr_host_streams(x: int, tile: int = 0) -> dict:
    """Copies of the packed streams of one row tile as numpy arrays: stream (uint16), units (structured),
    blk_unit, and the tile's first row and height."""
    vp, i64 = ctypes.c_void_p, ctypes.c_int64
    pe, pu, pb = vp(), vp(), vp()
    ne, nu, r0, nr = i64(), i64(), i64(), i64()
    _check(load().rsr_host_streams(x, int(tile), ctypes.byref(pe), ctypes.byref(ne), ctypes.byref(pu), ctypes.byref(nu),
                                   ctypes.byref(pb), ctypes.byref(r0), ctypes.byref(nr)))
    info = rsr_host_info(x)

    def view(ptr, count, dtype):
        if count == 0:
            return np.empty(0, dtype=dtype)
        nbytes = count * np.dtype(dtype).itemsize
        buf = (ctypes.c_char * nbytes).from_address(ptr.value)
        return np.frombuffer(buf, dtype=dtype, count=count).copy()

    return {
        "stream": view(pe, ne.value, np.uint16),
        "units": view(pu, nu.value, UNIT_DTYPE),
        "blk_unit": view(pb, info.nblocks + 1, np.uint32),
        "row0": int(r0.value),
        "rows": int(nr.value),
    }
