"""Thin ctypes binding of the C ABI in ``include/adasum.h``: argument marshalling only.

Every function has the name of the C entry point it calls.  PyTorch is used for device memory
and streams; all arithmetic runs in the CUDA library.  There is no CPU fallback: importing this
module raises if the native library has not been built.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "lib", "libadasum_b200.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"native library {LIB_PATH} is missing; build it with "
        "`python -m paper_2006_02924_b200.build` (needs nvcc, targets sm_100a)")

_lib = ctypes.CDLL(LIB_PATH)

ADASUM_F32, ADASUM_F16, ADASUM_BF16, ADASUM_F64 = 0, 1, 2, 3
ADASUM_FLAG_SIMPLE_KERNELS, ADASUM_FLAG_SEPARATE_FINISH, ADASUM_FLAG_LINEAR_ORDER = 1 << 16, 1 << 17, 1 << 18
ADASUM_FLAG_NO_TCGEN05 = 1 << 19
ADASUM_FLAG_TOP_DOWN_HALVES = 1 << 20
ADASUM_FLAG_NO_LEVEL_FUSION = 1 << 21
ADASUM_FLAG_SELFTEST_TIMEOUT = 1 << 22
ADASUM_OK = 0
ADASUM_MAX_WORKERS = 4096
ADASUM_MAX_LEVELS = 12
_DTYPES = {torch.float32: ADASUM_F32, torch.float16: ADASUM_F16, torch.bfloat16: ADASUM_BF16,
           torch.float64: ADASUM_F64}

_i64p = ctypes.POINTER(ctypes.c_int64)
_i32p = ctypes.POINTER(ctypes.c_int32)

_lib.adasum_workspace_bytes.restype = ctypes.c_size_t
_lib.adasum_workspace_bytes.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int,
                                        ctypes.c_uint32]
_lib.adasum_plan_info.restype = ctypes.c_int
_lib.adasum_plan_info.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int,
                                  ctypes.c_uint32, _i32p, _i32p, _i32p]
_lib.adasum_reduce.restype = ctypes.c_int
_lib.adasum_reduce.argtypes = [ctypes.POINTER(ctypes.c_void_p), _i64p, ctypes.c_int32, ctypes.c_int32,
                               ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                               ctypes.c_uint32, ctypes.c_void_p]
_lib.adasum_reduce_ex.restype = ctypes.c_int
_lib.adasum_reduce_ex.argtypes = [ctypes.POINTER(ctypes.c_void_p), _i64p, ctypes.c_int32, ctypes.c_int32,
                                  ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                  ctypes.c_uint32, ctypes.c_void_p]
_lib.adasum_reduce_delta.restype = ctypes.c_int
_lib.adasum_reduce_delta.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_void_p, _i64p, ctypes.c_int32,
                                     ctypes.c_int32, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_size_t, ctypes.c_uint32, ctypes.c_void_p]
_lib.adasum_pair.restype = ctypes.c_int
_lib.adasum_pair.argtypes = [ctypes.c_void_p, ctypes.c_void_p, _i64p, ctypes.c_int32, ctypes.c_int,
                             ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_uint32,
                             ctypes.c_void_p]
_lib.adasum_status_string.restype = ctypes.c_char_p
_lib.adasum_status_string.argtypes = [ctypes.c_int]
_lib.adasum_last_error.restype = ctypes.c_char_p
_lib.adasum_last_error.argtypes = []
_lib.adasum_shutdown.restype = ctypes.c_int
_lib.adasum_shutdown.argtypes = []


class AdasumError(RuntimeError):
    def __init__(self, status: int):
        self.status = int(status)
        detail = _lib.adasum_last_error().decode()
        super().__init__(f"{adasum_status_string(status)}: {detail}" if detail else adasum_status_string(status))


def flags_radix(first: int = 0, later: int = 0) -> int:
    """Value of the ``flags`` argument that fixes the radix of the first / later levels."""
    return (first & 0xFF) | ((later & 0xFF) << 8)


def adasum_status_string(status: int) -> str:
    return _lib.adasum_status_string(int(status)).decode()


def adasum_last_error() -> str:
    return _lib.adasum_last_error().decode()


def adasum_shutdown() -> None:
    status = _lib.adasum_shutdown()
    if status != ADASUM_OK:
        raise AdasumError(status)


def adasum_workspace_bytes(total_elems: int, num_tensors: int, n_workers: int, dtype, flags: int = 0) -> int:
    return int(_lib.adasum_workspace_bytes(int(total_elems), int(num_tensors), int(n_workers),
                                           _dtype_code(dtype), int(flags)))


def adasum_plan_info(total_elems: int, num_tensors: int, n_workers: int, dtype, flags: int = 0) -> dict:
    radices = (ctypes.c_int32 * ADASUM_MAX_LEVELS)()
    levels, launches = ctypes.c_int32(), ctypes.c_int32()
    status = _lib.adasum_plan_info(int(total_elems), int(num_tensors), int(n_workers), _dtype_code(dtype),
                                   int(flags), radices, ctypes.byref(levels), ctypes.byref(launches))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return {"radices": [int(radices[i]) for i in range(levels.value)], "launches": int(launches.value)}


_lib.adasum_device_status.restype = ctypes.c_int
_lib.adasum_device_status.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int, ctypes.c_uint32,
                                      ctypes.c_void_p, ctypes.c_void_p]


def adasum_device_status(total_elems: int, num_tensors: int, n_workers: int, dtype, workspace, flags: int = 0,
                         stream=None) -> int:
    """``adasum_device_status`` of the C ABI: 0, or 7 (ADASUM_ERR_TIMEOUT) if a bounded device-side
    wait of the last reduce on ``workspace`` ran out.  Synchronises the stream."""
    return int(_lib.adasum_device_status(int(total_elems), int(num_tensors), int(n_workers), _dtype_code(dtype),
                                         int(flags), workspace.data_ptr(), _stream_handle(stream)))


def _dtype_code(dtype) -> int:
    if isinstance(dtype, int):
        return dtype
    if isinstance(dtype, str):
        return {"f32": ADASUM_F32, "f16": ADASUM_F16, "bf16": ADASUM_BF16, "f64": ADASUM_F64}[dtype]
    return _DTYPES[dtype]


def _offsets_array(offsets, total: int) -> np.ndarray:
    if offsets is None:
        offsets = [0, total]
    return np.ascontiguousarray(np.asarray(offsets, dtype=np.int64))


def _stream_handle(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _workspace(workspace, need: int, device):
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def adasum_reduce(grads, tensor_offsets=None, out=None, workspace=None, flags: int = 0, stream=None):
    """``adasum_reduce`` of the C ABI.  ``grads``: N CUDA tensors (one fused buffer per worker, same
    dtype and length).  Returns ``out`` (fp32, allocated here if not given)."""
    grads = list(grads)
    first = grads[0]
    total = first.numel()
    offs = _offsets_array(tensor_offsets, total)
    num_tensors = offs.size - 1
    if out is None:
        out = torch.empty(total, dtype=torch.float32, device=first.device)
    need = adasum_workspace_bytes(total, num_tensors, len(grads), first.dtype, flags)
    workspace, ws_ptr, ws_bytes = _workspace(workspace, need, first.device)
    ptrs = (ctypes.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
    with torch.cuda.device(first.device):
        status = _lib.adasum_reduce(ptrs, offs.ctypes.data_as(_i64p), num_tensors, len(grads),
                                    _dtype_code(first.dtype), out.data_ptr(), ws_ptr, ws_bytes, int(flags),
                                    _stream_handle(stream))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return out


def adasum_reduce_ex(grads, tensor_offsets=None, out=None, orthogonality=None, workspace=None, flags: int = 0,
                     stream=None):
    """``adasum_reduce_ex`` of the C ABI: the reduce plus the per-tensor orthogonality measure.
    Returns ``(out, orthogonality)`` (both allocated here if not given)."""
    grads = list(grads)
    first = grads[0]
    total = first.numel()
    offs = _offsets_array(tensor_offsets, total)
    num_tensors = offs.size - 1
    if out is None:
        out = torch.empty(total, dtype=torch.float32, device=first.device)
    if orthogonality is None:
        orthogonality = torch.empty(max(num_tensors, 1), dtype=torch.float32, device=first.device)[:num_tensors]
    need = adasum_workspace_bytes(total, num_tensors, len(grads), first.dtype, flags)
    workspace, ws_ptr, ws_bytes = _workspace(workspace, need, first.device)
    ptrs = (ctypes.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
    with torch.cuda.device(first.device):
        status = _lib.adasum_reduce_ex(ptrs, offs.ctypes.data_as(_i64p), num_tensors, len(grads),
                                       _dtype_code(first.dtype), out.data_ptr(), orthogonality.data_ptr(), ws_ptr,
                                       ws_bytes, int(flags), _stream_handle(stream))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return out, orthogonality


_lib.adasum_reduce_scaled.restype = ctypes.c_int
_lib.adasum_reduce_scaled.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_void_p, _i64p, ctypes.c_int32,
                                      ctypes.c_int32, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                      ctypes.c_void_p, ctypes.c_size_t, ctypes.c_uint32, ctypes.c_void_p]


def adasum_reduce_scaled(grads, scales, tensor_offsets=None, out=None, orthogonality=None, workspace=None,
                         flags: int = 0, stream=None, want_orthogonality: bool = False):
    """``adasum_reduce_scaled`` of the C ABI: the buffers hold ``scales[w, t]`` times worker w's
    gradient for tensor t (a CUDA fp32 tensor of shape [N, num_tensors]); returns the combination of
    the gradients themselves (and the orthogonality measure when asked for)."""
    grads = list(grads)
    first = grads[0]
    total = first.numel()
    offs = _offsets_array(tensor_offsets, total)
    num_tensors = offs.size - 1
    if scales.dtype != torch.float32 or not scales.is_cuda or not scales.is_contiguous():
        raise TypeError("scales must be a contiguous CUDA fp32 tensor")
    if scales.numel() != len(grads) * num_tensors:
        raise ValueError(f"scales has {scales.numel()} entries, need {len(grads)} x {num_tensors}")
    if out is None:
        out = torch.empty(total, dtype=torch.float32, device=first.device)
    if orthogonality is None and want_orthogonality:
        orthogonality = torch.empty(max(num_tensors, 1), dtype=torch.float32, device=first.device)[:num_tensors]
    need = adasum_workspace_bytes(total, num_tensors, len(grads), first.dtype, flags)
    workspace, ws_ptr, ws_bytes = _workspace(workspace, need, first.device)
    ptrs = (ctypes.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
    with torch.cuda.device(first.device):
        status = _lib.adasum_reduce_scaled(ptrs, scales.data_ptr(), offs.ctypes.data_as(_i64p), num_tensors,
                                           len(grads), _dtype_code(first.dtype), out.data_ptr(),
                                           orthogonality.data_ptr() if orthogonality is not None else None, ws_ptr,
                                           ws_bytes, int(flags), _stream_handle(stream))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return (out, orthogonality) if orthogonality is not None else out


_lib.adasum_sharded_gram.restype = ctypes.c_int
_lib.adasum_sharded_gram.argtypes = [ctypes.POINTER(ctypes.c_void_p), _i64p, ctypes.c_int32, ctypes.c_int32,
                                     ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_uint32, ctypes.c_int32,
                                     ctypes.POINTER(ctypes.c_size_t), _i64p, ctypes.c_void_p]
_lib.adasum_sharded_apply.restype = ctypes.c_int
_lib.adasum_sharded_apply.argtypes = [ctypes.POINTER(ctypes.c_void_p), _i64p, ctypes.c_int32, ctypes.c_int32,
                                      ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                      ctypes.c_size_t, ctypes.c_uint32, ctypes.c_int32, ctypes.c_void_p]


def adasum_reduce_delta(currents, start, tensor_offsets=None, out=None, out_dtype=None, orthogonality=None,
                        workspace=None, flags: int = 0, stream=None):
    """``adasum_reduce_delta`` of the C ABI: ``out = start + Adasum_w(currents[w] - start)`` per
    tensor.  ``start=None`` gives the plain reduce with a choice of output type.  ``out`` may be
    ``start`` itself (in-place update) when the types agree.  Returns ``out``."""
    currents = list(currents)
    first = currents[0]
    total = first.numel()
    offs = _offsets_array(tensor_offsets, total)
    num_tensors = offs.size - 1
    if out is None:
        out = torch.empty(total, dtype=out_dtype or torch.float32, device=first.device)
    need = adasum_workspace_bytes(total, num_tensors, len(currents), first.dtype, flags)
    workspace, ws_ptr, ws_bytes = _workspace(workspace, need, first.device)
    ptrs = (ctypes.c_void_p * len(currents))(*[g.data_ptr() for g in currents])
    if start is not None and (start.dtype != first.dtype or start.numel() != total):
        raise ValueError("start must have the type and size of the workers' buffers")
    with torch.cuda.device(first.device):
        status = _lib.adasum_reduce_delta(ptrs, None if start is None else start.data_ptr(),
                                          offs.ctypes.data_as(_i64p), num_tensors, len(currents),
                                          _dtype_code(first.dtype), out.data_ptr(), _dtype_code(out.dtype),
                                          None if orthogonality is None else orthogonality.data_ptr(),
                                          ws_ptr, ws_bytes, int(flags), _stream_handle(stream))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return out


def adasum_sharded_gram(grads, tensor_offsets, workspace, level: int, flags: int = 0, stream=None):
    """``adasum_sharded_gram`` of the C ABI.  Returns this GPU's fp64 Gram sums of ``level`` as a
    float64 view INTO ``workspace`` (add it over the GPUs in place, then call ``adasum_sharded_apply``)."""
    grads = list(grads)
    first = grads[0]
    offs = _offsets_array(tensor_offsets, first.numel())
    ptrs = (ctypes.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
    off, count = ctypes.c_size_t(), ctypes.c_int64()
    with torch.cuda.device(first.device):
        status = _lib.adasum_sharded_gram(ptrs, offs.ctypes.data_as(_i64p), offs.size - 1, len(grads),
                                          _dtype_code(first.dtype), workspace.data_ptr(),
                                          workspace.numel() * workspace.element_size(), int(flags), int(level),
                                          ctypes.byref(off), ctypes.byref(count), _stream_handle(stream))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return workspace.view(torch.uint8)[off.value:off.value + 8 * count.value].view(torch.float64)


def adasum_sharded_apply(grads, tensor_offsets, out, workspace, level: int, orthogonality=None, flags: int = 0,
                         stream=None):
    """``adasum_sharded_apply`` of the C ABI."""
    grads = list(grads)
    first = grads[0]
    offs = _offsets_array(tensor_offsets, first.numel())
    ptrs = (ctypes.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
    with torch.cuda.device(first.device):
        status = _lib.adasum_sharded_apply(ptrs, offs.ctypes.data_as(_i64p), offs.size - 1, len(grads),
                                           _dtype_code(first.dtype), out.data_ptr(),
                                           None if orthogonality is None else orthogonality.data_ptr(),
                                           workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                           int(flags), int(level), _stream_handle(stream))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return out


def adasum_reduce_sharded(grads, tensor_offsets, group=None, out=None, orthogonality=None, workspace=None,
                          flags: int = 0, stream=None):
    """The whole element-sharded reduce on this rank: per level ``adasum_sharded_gram``, a
    ``torch.distributed.all_reduce`` (sum) of the Gram sums over ``group``, ``adasum_sharded_apply``.
    ``grads`` are this rank's slices (see ``include/adasum.h``).  Returns this rank's slice of the result."""
    import torch.distributed as dist

    grads = list(grads)
    first = grads[0]
    total = first.numel()
    offs = _offsets_array(tensor_offsets, total)
    num_tensors = offs.size - 1
    if out is None:
        out = torch.empty(total, dtype=torch.float32, device=first.device)
    need = adasum_workspace_bytes(total, num_tensors, len(grads), first.dtype, flags)
    workspace, _, _ = _workspace(workspace, need, first.device)
    levels = len(adasum_plan_info(total, num_tensors, len(grads), first.dtype, flags)["radices"])
    for level in range(levels):
        sums = adasum_sharded_gram(grads, offs, workspace, level, flags=flags, stream=stream)
        if sums.numel() > 0:
            dist.all_reduce(sums, op=dist.ReduceOp.SUM, group=group)
        adasum_sharded_apply(grads, offs, out, workspace, level, orthogonality=orthogonality, flags=flags,
                             stream=stream)
    return out


def adasum_pair(a, b, tensor_offsets=None, out=None, workspace=None, flags: int = 0, stream=None):
    """``adasum_pair`` of the C ABI: ``out = Adasum(a, b)`` per tensor."""
    total = a.numel()
    offs = _offsets_array(tensor_offsets, total)
    num_tensors = offs.size - 1
    if out is None:
        out = torch.empty(total, dtype=torch.float32, device=a.device)
    need = adasum_workspace_bytes(total, num_tensors, 2, a.dtype, flags)
    workspace, ws_ptr, ws_bytes = _workspace(workspace, need, a.device)
    with torch.cuda.device(a.device):
        status = _lib.adasum_pair(a.data_ptr(), b.data_ptr(), offs.ctypes.data_as(_i64p), num_tensors,
                                  _dtype_code(a.dtype), out.data_ptr(), ws_ptr, ws_bytes, int(flags),
                                  _stream_handle(stream))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return out


def raw():
    """The loaded ``ctypes.CDLL`` (for tests that pass raw pointers)."""
    return _lib


class _LaunchRecord(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("level", ctypes.c_int32), ("radix", ctypes.c_int32),
                ("ms", ctypes.c_float)]


KERNEL_NAMES = {0: "gram_partial", 1: "tree_weights", 2: "weighted_sum", 3: "convert", 4: "fused_small",
                5: "wsum_gram", 6: "short_tensors", 7: "embedding", 8: "embedding_sort", 9: "embedding_sum",
                10: "checkpoint_save", 11: "checkpoint_load", 12: "act_grad", 13: "weight_grad"}

_lib.adasum_profile_enable.restype = ctypes.c_int
_lib.adasum_profile_enable.argtypes = [ctypes.c_int32]
_lib.adasum_profile_collect.restype = ctypes.c_int
_lib.adasum_profile_collect.argtypes = [ctypes.POINTER(_LaunchRecord), ctypes.c_int32, _i32p]


def adasum_profile_enable(max_launches: int) -> None:
    status = _lib.adasum_profile_enable(int(max_launches))
    if status != ADASUM_OK:
        raise AdasumError(status)


def adasum_profile_collect(capacity: int = 4096) -> list[dict]:
    """One dict per kernel launch since ``adasum_profile_enable``: kernel, level, radix, ms."""
    records = (_LaunchRecord * capacity)()
    count = ctypes.c_int32()
    status = _lib.adasum_profile_collect(records, capacity, ctypes.byref(count))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return [{"kernel": KERNEL_NAMES.get(r.kernel, str(r.kernel)), "level": r.level, "radix": r.radix,
             "ms": float(r.ms)} for r in records[:min(count.value, capacity)]]


ADASUM_NOALLOC_MAX_ELEMS = 1 << 26
ADASUM_NOALLOC_MAX_TENSORS = 4096

_lib.adasum_pair_noalloc.restype = ctypes.c_int
_lib.adasum_pair_noalloc.argtypes = [ctypes.c_void_p, ctypes.c_void_p, _i64p, ctypes.c_int32, ctypes.c_int,
                                     ctypes.c_void_p, ctypes.c_void_p]


def adasum_pair_noalloc(a, b, tensor_offsets=None, out=None, stream=None):
    """``adasum_pair_noalloc`` of the C ABI: the pair operator for callers that cannot allocate
    device memory.  The library uses a fixed scratch array of its own instead of a workspace, so
    pass ``out`` to keep this wrapper from allocating either (it allocates ``out`` with torch only
    when none is given)."""
    total = a.numel()
    offs = _offsets_array(tensor_offsets, total)
    if out is None:
        out = torch.empty(total, dtype=torch.float32, device=a.device)
    with torch.cuda.device(a.device):
        status = _lib.adasum_pair_noalloc(a.data_ptr(), b.data_ptr(), offs.ctypes.data_as(_i64p), offs.size - 1,
                                          _dtype_code(a.dtype), out.data_ptr(), _stream_handle(stream))
    if status != ADASUM_OK:
        raise AdasumError(status)
    return out


# ---- producing a worker's gradients in the fused buffer ---------------------------------------------

ADASUM_ACT = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
ADASUM_CHECKPOINT_GROUP = 32

_i64, _i32, _vp, _f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float
_lib.adasum_embedding_forward.restype = ctypes.c_int
_lib.adasum_embedding_forward.argtypes = [_vp, _i64, _i64, _i64, ctypes.c_int, _vp, _i32, _i64, _f32, _vp, _i64,
                                          ctypes.c_int, _vp]
_lib.adasum_embedding_grad_workspace_bytes.restype = ctypes.c_size_t
_lib.adasum_embedding_grad_workspace_bytes.argtypes = [_i64, _i64, _i64]
_lib.adasum_embedding_grad.restype = ctypes.c_int
_lib.adasum_embedding_grad.argtypes = [_vp, _i64, ctypes.c_int, _vp, _i32, _i64, _f32, _vp, _i64, _i64, ctypes.c_int,
                                       _i32, _vp, ctypes.c_size_t, _vp]
_lib.adasum_checkpoint_bytes.restype = ctypes.c_size_t
_lib.adasum_checkpoint_bytes.argtypes = [_i64, _i64]
_lib.adasum_checkpoint_save.restype = ctypes.c_int
_lib.adasum_checkpoint_save.argtypes = [_vp, _i64, _i64, _i64, ctypes.c_int, ctypes.c_int, _vp, _i64, _vp, _vp]
_lib.adasum_checkpoint_load.restype = ctypes.c_int
_lib.adasum_checkpoint_load.argtypes = [_vp, _i64, _i64, _vp, _i64, ctypes.c_int, _vp]
_lib.adasum_checkpoint_act_grad.restype = ctypes.c_int
_lib.adasum_checkpoint_act_grad.argtypes = [_vp, _i64, _i64, ctypes.c_int, _vp, _i64, ctypes.c_int, _vp, _i64, _vp]
_lib.adasum_checkpoint_weight_grad_workspace_bytes.restype = ctypes.c_size_t
_lib.adasum_checkpoint_weight_grad_workspace_bytes.argtypes = [_i64, _i64, _i64, ctypes.c_int]
_lib.adasum_checkpoint_weight_grad.restype = ctypes.c_int
_lib.adasum_checkpoint_weight_grad.argtypes = [_vp, _i64, _i64, _vp, _i64, _i64, ctypes.c_int, _f32, _vp, _vp,
                                               ctypes.c_int, _i32, _vp, ctypes.c_size_t, _vp]


# These calls are outside autograd, as the reduces are: results carry no graph, whatever the arguments require, and a
# tensor that is written in place (out=x, grad_in=grad_out) is not marked as changed.
#
# They sit in a training step's inner loop: their wrappers avoid what costs a microsecond each in Python
# (device objects, context managers, tensors built from keyword-laden factories).

def _matrix(name: str, t, rows=None, cols=None):
    """Checks a CUDA matrix with contiguous rows; returns its row stride in elements."""
    if t.dim() != 2 or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA matrix")
    shape, strides = t.shape, t.stride()
    if (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise ValueError(f"{name} is {tuple(shape)}, need ({rows}, {cols})")
    if strides[1] != 1 and shape[1] > 1:
        raise ValueError(f"{name} must have contiguous rows")
    return strides[0] if shape[0] > 1 else max(strides[0], shape[1])


def _operator_dtype(dtype) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"{dtype}: fp32, fp16 or bf16")
    return code


def _same_device(device: int, *tensors):
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"a tensor is on {t.device}, not on cuda:{device}")


def _operator_call(device: int, stream, function, *args):
    """Calls ``function(*args, stream handle)`` with the tensors' device current, on ``stream`` or that device's
    current one; raises on any status but ADASUM_OK."""
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(device)
    else:
        handle = int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)
    if device == torch._C._cuda_getDevice():
        status = function(*args, handle)
    else:
        with torch.cuda.device(device):
            status = function(*args, handle)
    if status != ADASUM_OK:
        raise AdasumError(status)


def _allocate(like, stream, shape, dtype):
    """A tensor for a call on `stream`."""
    t = like.new_empty(*shape) if dtype is like.dtype else like.new_empty(shape, dtype=dtype)
    return t if stream is None else _hand_over(t, stream)


def _allocate_like(like, stream):
    """A matrix of the same shape and type with contiguous rows."""
    t = torch.empty_like(like)
    return t if stream is None else _hand_over(t, stream)


def _hand_over(t, stream):
    """The caching allocator must not hand a tensor on before the stream that it is used on is done with it."""
    if t.numel() > 0:
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(int(stream), device=t.device)
        # the memory may still be in use on the current stream, from which it was handed out
        stream.wait_stream(torch.cuda.current_stream(t.device))
        t.record_stream(stream)
    return t


def _operator_workspace(like, stream, workspace, need: int):
    if workspace is None:
        return _allocate(like, stream, (max(need, 256),), torch.uint8)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace


def _tokens(tokens):
    if tokens.dtype not in (torch.int32, torch.int64) or not tokens.is_cuda:
        raise TypeError("tokens must be a CUDA tensor of int32 or int64")
    if not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous")


def adasum_embedding_forward(table, tokens, scale: float = 1.0, out=None, out_dtype=None, stream=None):
    """``adasum_embedding_forward`` of the C ABI: ``scale * table[tokens]``, zeros for tokens outside the
    table.  ``tokens`` has any shape; returns ``out`` of shape ``[tokens.numel(), dim]`` (of the table's
    type unless ``out_dtype`` says otherwise)."""
    table_stride = _matrix("table", table)
    _tokens(tokens)
    count = tokens.numel()
    num_rows, dim = table.shape
    if out is None:
        out, out_stride = _allocate(table, stream, (count, dim), out_dtype or table.dtype), dim
    else:
        out_stride = _matrix("out", out, count, dim)
    device = table.get_device()
    _same_device(device, tokens, out)
    _operator_call(device, stream, _lib.adasum_embedding_forward, table.data_ptr(), table_stride, num_rows, dim,
                   _operator_dtype(table.dtype), tokens.data_ptr(), tokens.element_size(), count, scale, out.data_ptr(),
                   out_stride, _operator_dtype(out.dtype))
    return out


def adasum_embedding_grad_workspace_bytes(num_tokens: int, num_rows: int, dim: int) -> int:
    return int(_lib.adasum_embedding_grad_workspace_bytes(int(num_tokens), int(num_rows), int(dim)))


def adasum_embedding_grad(grad_out, tokens, num_rows=None, grad_table=None, grad_dtype=None, scale: float = 1.0,
                          accumulate: bool = False, workspace=None, stream=None):
    """``adasum_embedding_grad`` of the C ABI.  ``grad_out``: ``[tokens.numel(), dim]``.  The gradient goes
    to ``grad_table`` (``[num_rows, dim]`` or flat, contiguous: a tensor's place in a fused buffer), which
    is allocated here (fp32 unless ``grad_dtype`` says otherwise) if only ``num_rows`` is given."""
    _tokens(tokens)
    count = tokens.numel()
    stride = _matrix("grad_out", grad_out, count)
    dim = grad_out.shape[1]
    if grad_table is None:
        if num_rows is None or accumulate:
            raise ValueError("grad_table is missing")
        grad_table = _allocate(grad_out, stream, (num_rows, dim), grad_dtype or torch.float32)
    if not grad_table.is_contiguous():
        raise ValueError("grad_table must be contiguous")
    if num_rows is None:
        num_rows = grad_table.shape[0] if grad_table.dim() == 2 else grad_table.numel() // max(dim, 1)
    if grad_table.numel() != num_rows * dim or (grad_table.dim() == 2 and grad_table.shape[1] != dim):
        raise ValueError(f"grad_table is {tuple(grad_table.shape)}, need ({num_rows}, {dim})")
    workspace = _operator_workspace(grad_out, stream, workspace,
                                    _lib.adasum_embedding_grad_workspace_bytes(count, num_rows, dim))
    device = grad_out.get_device()
    _same_device(device, tokens, grad_table, workspace)
    _operator_call(device, stream, _lib.adasum_embedding_grad, grad_out.data_ptr(), stride,
                   _operator_dtype(grad_out.dtype), tokens.data_ptr(), tokens.element_size(), count, scale,
                   grad_table.data_ptr(), num_rows, dim, _operator_dtype(grad_table.dtype), int(accumulate),
                   workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return grad_table


def adasum_checkpoint_bytes(rows: int, features: int) -> int:
    return int(_lib.adasum_checkpoint_bytes(int(rows), int(features)))


def _checkpoint_size(rows: int, features: int) -> int:
    groups = -(-features // ADASUM_CHECKPOINT_GROUP)
    return rows * groups * (ADASUM_CHECKPOINT_GROUP + 1)


def _checkpoint(device: int, checkpoint, rows: int, features: int):
    if checkpoint.dtype != torch.uint8 or not checkpoint.is_contiguous():
        raise TypeError("checkpoint must be a contiguous tensor of uint8")
    need = _checkpoint_size(rows, features)
    if checkpoint.numel() < need:
        raise ValueError(f"checkpoint has {checkpoint.numel()} bytes, {rows} x {features} needs {need}")
    if checkpoint.get_device() != device:
        raise ValueError(f"checkpoint is on {checkpoint.device}, not on cuda:{device}")
    return checkpoint.data_ptr()


def adasum_checkpoint_save(x, activation: str = "none", out=None, checkpoint=None, want_out: bool = True, stream=None):
    """``adasum_checkpoint_save`` of the C ABI: returns ``(activation(x), checkpoint)``; ``out`` may be ``x``
    itself.  With ``want_out=False`` only the checkpoint is written and the first item is None."""
    stride = _matrix("x", x)
    rows, features = x.shape
    device = x.get_device()
    if checkpoint is None:
        checkpoint = _allocate(x, stream, (_checkpoint_size(rows, features),), torch.uint8)
    out_stride, out_ptr = features, None
    if out is not None:
        out_stride = _matrix("out", out, rows, features)
        if out.dtype != x.dtype:
            raise TypeError("out must have the type of x")
        _same_device(device, out)
        out_ptr = out.data_ptr()
    elif want_out:
        out = _allocate_like(x, stream)
        out_ptr = out.data_ptr()
    _operator_call(device, stream, _lib.adasum_checkpoint_save, x.data_ptr(), stride, rows, features,
                   _operator_dtype(x.dtype), ADASUM_ACT[activation], out_ptr, out_stride,
                   _checkpoint(device, checkpoint, rows, features))
    return out, checkpoint


def adasum_checkpoint_load(checkpoint, rows: int, features: int, dtype=None, out=None, stream=None):
    """``adasum_checkpoint_load`` of the C ABI: the kept values, in ``dtype`` (fp32 by default) or ``out``."""
    if out is None:
        if not checkpoint.is_cuda:
            raise TypeError("checkpoint must be a CUDA tensor")
        out, out_stride = _allocate(checkpoint, stream, (rows, features), dtype or torch.float32), features
    else:
        out_stride = _matrix("out", out, rows, features)
    device = out.get_device()
    _operator_call(device, stream, _lib.adasum_checkpoint_load, _checkpoint(device, checkpoint, rows, features), rows,
                   features, out.data_ptr(), out_stride, _operator_dtype(out.dtype))
    return out


def adasum_checkpoint_act_grad(checkpoint, grad_out, activation: str, grad_in=None, stream=None):
    """``adasum_checkpoint_act_grad`` of the C ABI: ``grad_out * activation'(kept x)``; ``grad_in`` may be
    ``grad_out`` itself."""
    stride = _matrix("grad_out", grad_out)
    rows, features = grad_out.shape
    device = grad_out.get_device()
    if grad_in is None:
        grad_in, in_stride = _allocate_like(grad_out, stream), features
    else:
        in_stride = _matrix("grad_in", grad_in, rows, features)
        if grad_in.dtype != grad_out.dtype:
            raise TypeError("grad_in must have the type of grad_out")
        _same_device(device, grad_in)
    _operator_call(device, stream, _lib.adasum_checkpoint_act_grad, _checkpoint(device, checkpoint, rows, features),
                   rows, features, ADASUM_ACT[activation], grad_out.data_ptr(), stride,
                   _operator_dtype(grad_out.dtype), grad_in.data_ptr(), in_stride)
    return grad_in


def adasum_checkpoint_weight_grad_workspace_bytes(rows: int, features: int, outputs: int, dtype) -> int:
    return int(_lib.adasum_checkpoint_weight_grad_workspace_bytes(int(rows), int(features), int(outputs),
                                                                  _dtype_code(dtype)))


def adasum_checkpoint_weight_grad(checkpoint, grad_out, features=None, grad_weight=None, grad_bias=None,
                                  want_bias: bool = False, grad_dtype=None, scale: float = 1.0,
                                  accumulate: bool = False, workspace=None, stream=None):
    """``adasum_checkpoint_weight_grad`` of the C ABI.  ``grad_out``: ``[rows, outputs]``.  The gradients go to
    ``grad_weight`` (``[outputs, features]`` or flat) and ``grad_bias`` (``[outputs]``), both contiguous;
    what is not given is allocated here (fp32 unless ``grad_dtype`` says otherwise; a bias gradient only
    with ``want_bias``).  Returns ``(grad_weight, grad_bias)``.  fp16 gradients round kept values of fp32 or bf16
    activations to fp16.  A product that the device did not finish (a bounded wait ran out) leaves NaN;
    ``adasum_checkpoint_weight_grad_status`` tells, for a ``workspace`` of the caller's."""
    stride = _matrix("grad_out", grad_out)
    rows, outputs = grad_out.shape
    if grad_weight is None:
        if features is None or accumulate:
            raise ValueError("grad_weight is missing")
        grad_weight = _allocate(grad_out, stream, (outputs, features), grad_dtype or torch.float32)
    if features is None:
        features = grad_weight.shape[1] if grad_weight.dim() == 2 else grad_weight.numel() // max(outputs, 1)
    if not grad_weight.is_contiguous():
        raise ValueError("grad_weight must be contiguous")
    if grad_weight.numel() != outputs * features or (grad_weight.dim() == 2 and grad_weight.shape[1] != features):
        raise ValueError(f"grad_weight is {tuple(grad_weight.shape)}, need ({outputs}, {features})")
    if grad_bias is None and want_bias:
        if accumulate:
            raise ValueError("grad_bias is missing")
        grad_bias = _allocate(grad_out, stream, (outputs,), grad_weight.dtype)
    if grad_bias is not None:
        if grad_bias.dtype != grad_weight.dtype:
            raise TypeError("grad_bias must have the type of grad_weight")
        if not grad_bias.is_contiguous() or grad_bias.numel() != outputs:
            raise ValueError(f"grad_bias must be contiguous and have {outputs} elements")
    code = _operator_dtype(grad_out.dtype)
    workspace = _operator_workspace(grad_out, stream, workspace,
                                    _lib.adasum_checkpoint_weight_grad_workspace_bytes(rows, features, outputs, code))
    device = grad_out.get_device()
    _same_device(device, grad_weight, grad_bias, workspace)
    _operator_call(device, stream, _lib.adasum_checkpoint_weight_grad, _checkpoint(device, checkpoint, rows, features),
                   rows, features, grad_out.data_ptr(), stride, outputs, code, scale, grad_weight.data_ptr(),
                   None if grad_bias is None else grad_bias.data_ptr(), _operator_dtype(grad_weight.dtype),
                   int(accumulate), workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return grad_weight, grad_bias


_lib.adasum_checkpoint_weight_grad_status.restype = ctypes.c_int
_lib.adasum_checkpoint_weight_grad_status.argtypes = [_i64, _i64, _i64, ctypes.c_int, _vp, _vp]


def adasum_checkpoint_weight_grad_status(rows: int, features: int, outputs: int, dtype, workspace, stream=None) -> int:
    """``adasum_checkpoint_weight_grad_status`` of the C ABI: 0, or 7 (ADASUM_ERR_TIMEOUT) if a bounded wait of
    the last weight gradient on ``workspace`` ran out.  Synchronises the stream."""
    return int(_lib.adasum_checkpoint_weight_grad_status(int(rows), int(features), int(outputs), _dtype_code(dtype),
                                                         workspace.data_ptr(), _stream_handle(stream)))


ADASUM_HAND_OVER = {"landed": 1, "multiplied": 2, "added": 3, "ready": 4, "formed": 5, "taken": 6}

_lib.adasum_checkpoint_weight_grad_selftest.restype = ctypes.c_int
_lib.adasum_checkpoint_weight_grad_selftest.argtypes = _lib.adasum_checkpoint_weight_grad.argtypes + [_i32]


def adasum_checkpoint_weight_grad_selftest(hand_over: str, checkpoint, grad_out, grad_weight, grad_bias, workspace):
    """``adasum_checkpoint_weight_grad_selftest`` of the C ABI, on the current stream: the named kind of hand-over
    inside the product never completes, so its bounded waits run out and are reported."""
    rows, outputs = grad_out.shape
    features = grad_weight.shape[1]
    status = _lib.adasum_checkpoint_weight_grad_selftest(
        _checkpoint(grad_out.get_device(), checkpoint, rows, features), rows, features, grad_out.data_ptr(),
        _matrix("grad_out", grad_out), outputs, _operator_dtype(grad_out.dtype), 1.0, grad_weight.data_ptr(),
        None if grad_bias is None else grad_bias.data_ptr(), _operator_dtype(grad_weight.dtype), 0, workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream_handle(None), ADASUM_HAND_OVER[hand_over])
    if status != ADASUM_OK:
        raise AdasumError(status)
