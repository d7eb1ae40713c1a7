"""Thin binding over libqlinear.so (see include/qlinear.h): argument marshalling only, by ctypes and, for the calls on tensors, csrc/native.cpp.

Every arithmetic step runs inside the library's CUDA kernels (or, for pack/unpack, its host
packer).  torch is used for device memory and streams.  There is no CPU fallback: if the shared
library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqlinear.so")

QL_OK = 0
QL_ERR_INVALID_ARG, QL_ERR_UNSUPPORTED, QL_ERR_ALLOC, QL_ERR_CUDA, QL_ERR_DEVICE_TIMEOUT, QL_ERR_ARCH = 1, 2, 3, 4, 5, 6
QL_PATH_GEMV, QL_PATH_GEMM = 1, 2
QL_ACT_IDENTITY, QL_ACT_SILU, QL_ACT_GELU_TANH = 0, 1, 2
ACTIVATIONS = {"identity": QL_ACT_IDENTITY, "silu": QL_ACT_SILU, "gelu_tanh": QL_ACT_GELU_TANH}

EXPORTS = (
    "qlinear_packed_size", "qlinear_pack", "qlinear_unpack", "qlinear_create", "qlinear_forward", "qlinear_forward_group", "qlinear_forward_batch", "qlinear_forward_gated", "qlinear_forward_a8", "qlinear_quantize_activations", "qlinear_kv_append", "qlinear_kv_scores", "qlinear_kv_output", "qlinear_kv_output_uses_tmp", "qlinear_kv_append_heads", "qlinear_kv_scores_heads", "qlinear_kv_output_heads", "qlinear_embed", "qlinear_residual_rmsnorm", "qlinear_rope_qkv",
    "qlinear_path_for", "qlinear_debug_unpack_device", "qlinear_debug_expire_wait", "qlinear_debug_null_launch", "qlinear_device_status", "qlinear_decode_static", "qlinear_destroy",
    "qlinear_status_string", "qlinear_version", "qlinear_debug_plan", "qlinear_debug_plan_kv_output", "qlinear_debug_takes_batch_kernel", "qlinear_debug_kv_hold", "qlinear_debug_route", "qlinear_debug_plan_a8", "qlinear_debug_config_reads",
    "qlinear_rope_tables", "qlinear_paged_page_bytes", "qlinear_paged_create", "qlinear_paged_destroy", "qlinear_paged_device_status", "qlinear_paged_append", "qlinear_paged_read",
    "qlinear_paged_attention_workspace", "qlinear_paged_attention", "qlinear_adjust_logits", "qlinear_debug_paged_ctas",
    "qlinear_paged_fork", "qlinear_paged_release", "qlinear_paged_pages_workspace", "qlinear_paged_reserve", "qlinear_paged_compact", "qlinear_paged_summarise", "qlinear_paged_select",
    "qlinear_paged_attention_selected_workspace", "qlinear_paged_attention_selected", "qlinear_paged_attention_shared_workspace", "qlinear_paged_attention_shared",
)


class QLinearError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (ql_status {status})")


class qlinear_desc(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("K", ctypes.c_int32), ("bits", ctypes.c_int32), ("group", ctypes.c_int32)]


class qlinear_paged_desc(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("h_kv", ctypes.c_int32), ("d_h", ctypes.c_int32)]


class qlinear_rope_scaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("original", ctypes.c_int32), ("factor", ctypes.c_double), ("slow", ctypes.c_double), ("fast", ctypes.c_double)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2505_00232_b200.build` "
            "(nvcc, sm_100a). There is no fallback path.")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32 = ctypes.c_void_p, ctypes.c_int32
    dp = ctypes.POINTER(qlinear_desc)
    lib.qlinear_packed_size.argtypes = [dp]
    lib.qlinear_packed_size.restype = ctypes.c_size_t
    lib.qlinear_pack.argtypes = [dp, vp, vp, vp, ctypes.c_size_t]
    lib.qlinear_pack.restype = ctypes.c_int
    lib.qlinear_unpack.argtypes = [dp, vp, vp, vp]
    lib.qlinear_unpack.restype = ctypes.c_int
    lib.qlinear_create.argtypes = [dp, vp, ctypes.c_int, ctypes.POINTER(vp)]
    lib.qlinear_create.restype = ctypes.c_int
    lib.qlinear_forward.argtypes = [vp, vp, vp, i32, vp]
    lib.qlinear_forward.restype = ctypes.c_int
    lib.qlinear_path_for.argtypes = [vp, i32]
    lib.qlinear_path_for.restype = i32
    lib.qlinear_debug_unpack_device.argtypes = [vp, vp, vp]
    lib.qlinear_debug_unpack_device.restype = ctypes.c_int
    lib.qlinear_forward_group.argtypes = [ctypes.POINTER(vp), ctypes.c_int32, vp, ctypes.POINTER(vp), ctypes.c_int32, vp]
    lib.qlinear_forward_group.restype = ctypes.c_int
    lib.qlinear_forward_batch.argtypes = [ctypes.POINTER(vp), ctypes.c_int32, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.c_int32, vp]
    lib.qlinear_forward_batch.restype = ctypes.c_int
    lib.qlinear_forward_gated.argtypes = [vp, vp, vp, vp, i32, i32, vp]
    lib.qlinear_forward_gated.restype = ctypes.c_int
    lib.qlinear_forward_a8.argtypes = [vp, vp, vp, i32, vp]
    lib.qlinear_forward_a8.restype = ctypes.c_int
    lib.qlinear_quantize_activations.argtypes = [vp, vp, vp, i32, i32, ctypes.c_int, vp]
    lib.qlinear_quantize_activations.restype = ctypes.c_int
    lib.qlinear_kv_append.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp]
    lib.qlinear_kv_append.restype = ctypes.c_int
    lib.qlinear_kv_scores.argtypes = [vp, vp, vp, i32, vp]
    lib.qlinear_kv_scores.restype = ctypes.c_int
    lib.qlinear_kv_output.argtypes = [vp, vp, vp, vp, vp, i32, vp]
    lib.qlinear_kv_output.restype = ctypes.c_int
    lib.qlinear_kv_output_uses_tmp.argtypes = [vp, vp, vp, i32]
    lib.qlinear_kv_output_uses_tmp.restype = i32
    lib.qlinear_embed.argtypes = [vp, vp, ctypes.c_int32, vp, vp]
    lib.qlinear_embed.restype = ctypes.c_int
    lib.qlinear_residual_rmsnorm.argtypes = [vp, vp, vp, ctypes.c_float, ctypes.c_float, vp, vp, i32, i32, ctypes.c_int, vp]
    lib.qlinear_residual_rmsnorm.restype = ctypes.c_int
    lib.qlinear_rope_qkv.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, i32, i32, i32, i32, i32, ctypes.c_int, vp]
    lib.qlinear_rope_qkv.restype = ctypes.c_int
    lib.qlinear_debug_expire_wait.argtypes = [vp, vp]
    lib.qlinear_debug_expire_wait.restype = ctypes.c_int
    lib.qlinear_debug_null_launch.argtypes = [vp, ctypes.c_int32, ctypes.c_int32, vp]
    lib.qlinear_debug_null_launch.restype = ctypes.c_int
    pvp = ctypes.POINTER(ctypes.c_void_p)
    lib.qlinear_kv_append_heads.argtypes = [pvp, pvp, ctypes.c_int32, vp, vp, ctypes.c_int64, ctypes.c_int64, pvp, ctypes.c_int32, ctypes.c_int32, vp]
    lib.qlinear_kv_append_heads.restype = ctypes.c_int
    lib.qlinear_kv_scores_heads.argtypes = [pvp, ctypes.c_int32, vp, vp, ctypes.c_int32, vp]
    lib.qlinear_kv_scores_heads.restype = ctypes.c_int
    lib.qlinear_kv_output_heads.argtypes = [pvp, ctypes.c_int32, vp, pvp, vp, ctypes.c_int32, vp]
    lib.qlinear_kv_output_heads.restype = ctypes.c_int
    lib.qlinear_device_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.qlinear_device_status.restype = ctypes.c_int
    lib.qlinear_decode_static.argtypes = [dp, vp, vp, vp, i32, ctypes.c_int, vp]
    lib.qlinear_decode_static.restype = ctypes.c_int
    lib.qlinear_destroy.argtypes = [vp]
    lib.qlinear_destroy.restype = ctypes.c_int
    lib.qlinear_status_string.argtypes = [ctypes.c_int]
    lib.qlinear_status_string.restype = ctypes.c_char_p
    lib.qlinear_version.restype = ctypes.c_uint32
    lib.qlinear_debug_plan.argtypes = [vp, i32, ctypes.POINTER(i32), i32]
    lib.qlinear_debug_plan.restype = i32
    lib.qlinear_debug_plan_kv_output.argtypes = [vp, i32, ctypes.POINTER(i32), i32]
    lib.qlinear_debug_plan_kv_output.restype = i32
    lib.qlinear_debug_takes_batch_kernel.argtypes = [ctypes.POINTER(vp), i32, i32]
    lib.qlinear_debug_takes_batch_kernel.restype = i32
    lib.qlinear_debug_kv_hold.argtypes = [ctypes.POINTER(vp), i32, vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.qlinear_debug_route.argtypes = [vp, i32, i32, i32, i32, ctypes.POINTER(i32), i32]
    lib.qlinear_debug_route.restype = i32
    lib.qlinear_debug_plan_a8.argtypes = [vp, i32, i32, ctypes.POINTER(i32), i32]
    lib.qlinear_debug_plan_a8.restype = i32
    lib.qlinear_debug_kv_hold.restype = ctypes.c_int
    lib.qlinear_debug_config_reads.restype = ctypes.c_uint32
    i64, f32, size = ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    batch = [vp, i64, i32, vp, vp, i32, i32]                             # table, table_ld, table_width, kv_len, q_start, B, T
    lib.qlinear_rope_tables.argtypes = [vp, vp, i32, i32, i32, ctypes.c_double, ctypes.POINTER(qlinear_rope_scaling), i32, vp]
    lib.qlinear_paged_page_bytes.argtypes = [ctypes.POINTER(qlinear_paged_desc)]
    lib.qlinear_paged_page_bytes.restype = size
    lib.qlinear_paged_create.argtypes = [ctypes.POINTER(qlinear_paged_desc), vp, ctypes.c_int, ctypes.POINTER(vp)]
    lib.qlinear_paged_destroy.argtypes = [vp]
    lib.qlinear_paged_device_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.qlinear_paged_append.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, i32, *batch, vp, vp, i32, i32, i32, vp]
    lib.qlinear_paged_read.argtypes = [vp, *batch, vp, vp, vp]
    lib.qlinear_paged_attention_workspace.argtypes = [vp, i32, i32, i32]
    lib.qlinear_paged_attention_workspace.restype = size
    lib.qlinear_paged_attention.argtypes = [vp, vp, i64, vp, i64, i32, *batch, i32, f32, f32, i32, vp, size, vp]
    lib.qlinear_debug_paged_ctas.argtypes = [vp, i32, ctypes.POINTER(i32)]
    lib.qlinear_debug_paged_ctas.restype = i32
    lib.qlinear_adjust_logits.argtypes = [vp, i64, vp, i64, i32, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, i64, i32, vp]
    lib.qlinear_paged_fork.argtypes = [vp, vp, vp, i64, i32, i32, vp, vp, i32, vp, i64, vp]
    lib.qlinear_paged_release.argtypes = [vp, vp, vp, i64, i32, i32, vp, vp, i32, vp]
    lib.qlinear_paged_reserve.argtypes = [vp, vp, *batch, vp, vp, size, vp]
    lib.qlinear_paged_compact.argtypes = [vp, vp, vp, i64, i32, i32, vp, vp, vp, vp, size, vp]
    lib.qlinear_paged_summarise.argtypes = [vp, *batch, vp, vp, vp]
    lib.qlinear_paged_select.argtypes = [vp, vp, i64, i32, vp, vp, *batch, i32, i32, i32, vp, vp]
    lib.qlinear_paged_attention_selected.argtypes = [vp, vp, i64, vp, i64, i32, vp, i32, *batch, f32, f32, vp, size, vp]
    lib.qlinear_paged_attention_shared.argtypes = [vp, vp, i64, vp, i64, i32, *batch, i32, vp, vp, i32, f32, f32, vp, size, vp]
    lib.qlinear_paged_pages_workspace.argtypes = [vp]
    lib.qlinear_paged_attention_selected_workspace.argtypes = [vp, i32]
    lib.qlinear_paged_attention_shared_workspace.argtypes = [vp, i32, i32, i32, i32, i32, i32]
    for f in ("qlinear_paged_pages_workspace", "qlinear_paged_attention_selected_workspace", "qlinear_paged_attention_shared_workspace"):
        getattr(lib, f).restype = size
    for f in ("qlinear_rope_tables", "qlinear_paged_create", "qlinear_paged_destroy", "qlinear_paged_device_status", "qlinear_paged_append", "qlinear_paged_read", "qlinear_paged_attention", "qlinear_adjust_logits",
              "qlinear_paged_fork", "qlinear_paged_release", "qlinear_paged_reserve", "qlinear_paged_compact", "qlinear_paged_summarise", "qlinear_paged_select", "qlinear_paged_attention_selected",
              "qlinear_paged_attention_shared"):
        getattr(lib, f).restype = ctypes.c_int
    return lib


lib = _load()


def status_string(status: int) -> str:
    return lib.qlinear_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != QL_OK:
        raise QLinearError(status, where)


def _np_ptr(a: np.ndarray) -> ctypes.c_void_p:
    return a.ctypes.data_as(ctypes.c_void_p)


@dataclass(frozen=True)
class Desc:
    N: int
    K: int
    bits: int
    group: int = 0

    def c(self) -> qlinear_desc:
        return qlinear_desc(self.N, self.K, self.bits, self.group)

    @property
    def n_groups(self) -> int:
        return 1 if self.group == 0 else self.K // self.group


# ---------------------------------------------------------------------------- host calls
def qlinear_packed_size(desc: Desc) -> int:
    return int(lib.qlinear_packed_size(ctypes.byref(desc.c())))


def qlinear_pack(desc: Desc, q: np.ndarray, s: np.ndarray) -> np.ndarray:
    """q int8 [N, K] (one integer per byte), s fp16 [N] or [N, K/group] -> packed blob (uint8 array)."""
    q = np.ascontiguousarray(q, dtype=np.int8)
    s = np.ascontiguousarray(s, dtype=np.float16)
    size = qlinear_packed_size(desc)
    if size == 0:
        raise QLinearError(QL_ERR_UNSUPPORTED, "qlinear_packed_size")
    if q.shape != (desc.N, desc.K) or s.size != desc.N * desc.n_groups:
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_pack (shape)")
    out = np.empty(size, dtype=np.uint8)
    _check(lib.qlinear_pack(ctypes.byref(desc.c()), _np_ptr(q), _np_ptr(s), _np_ptr(out), size), "qlinear_pack")
    return out


def qlinear_unpack(desc: Desc, packed: np.ndarray):
    packed = np.ascontiguousarray(packed, dtype=np.uint8)
    if packed.size < qlinear_packed_size(desc) or qlinear_packed_size(desc) == 0:
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_unpack (size)")
    q = np.empty((desc.N, desc.K), dtype=np.int8)
    s = np.empty((desc.N, desc.n_groups), dtype=np.float16)
    _check(lib.qlinear_unpack(ctypes.byref(desc.c()), _np_ptr(packed), _np_ptr(q), _np_ptr(s)), "qlinear_unpack")
    return q, s


# ---------------------------------------------------------------------------- device calls
# A small layer takes the GPU a few microseconds, less than these calls took the host.  So every call on tensors first goes to the module built
# from csrc/native.cpp, which checks the arguments, allocates the outputs and calls the library; it returns None for everything
# that is not the common form of the call (subclasses, tracing, wrong shapes, ...), and the Python below it then does the call, or raises.
# Measured, us per call of the host: QLinear.forward at one token 6.7 -> 3.5 to 4.0 (by machine), qlinear_forward_group of three layers 14.0 -> 5.8,
# qlinear_residual_rmsnorm 11.1 -> 4.3, qlinear_rope_qkv 15.5 -> 4.8, KVCache.output 11.0 -> 5.3.
_half = _raw_stream = _device = _native = _serving = None
_NATIVE_API = ("qlinear_forward", "qlinear_forward_a8", "qlinear_forward_group", "qlinear_forward_gated", "qlinear_residual_rmsnorm", "qlinear_rope_qkv", "qlinear_embed",
               "qlinear_kv_append_heads", "qlinear_kv_scores_heads", "qlinear_kv_output_heads", "qlinear_kv_output", "qlinear_kv_output_uses_tmp")
_SERVING_API = ("qlinear_paged_append", "qlinear_paged_read", "qlinear_paged_attention_workspace", "qlinear_paged_attention", "qlinear_adjust_logits", "qlinear_rope_tables",
                "qlinear_paged_fork", "qlinear_paged_release", "qlinear_paged_pages_workspace", "qlinear_paged_reserve", "qlinear_paged_compact", "qlinear_paged_summarise", "qlinear_paged_select",
                "qlinear_paged_attention_selected_workspace", "qlinear_paged_attention_selected", "qlinear_paged_attention_shared_workspace", "qlinear_paged_attention_shared")


def _bind_torch():
    """torch is imported with the first device object, not with the package (packing needs none of it).  Returns the native module."""
    global _half, _raw_stream, _device, _native, _serving
    import torch
    if _native is None:
        from . import _native as native, build                           # (no fallback: the build makes it beside libqlinear.so)
        if native.built_for != build.installed_torch()[1]:
            raise ImportError(f"_native.so was built for {native.built_for}, not for {build.installed_torch()[1]}: run paper_2505_00232_b200/build.py")
        native.init(_check, *(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in _NATIVE_API))
        native._serving.init(*(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in _SERVING_API))
        _native, _serving = native, native._serving
    # (a torch without CUDA has neither entry point: its own error comes from the calls that need a device)
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)
    _half = torch.float16
    return _native


def _raw(stream):
    return None if stream is None else stream.cuda_stream


def _stream_ptr(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        _bind_torch()
    return _raw_stream(_device())                                        # the current stream of the current device


def _is_out(out, M: int, N: int) -> bool:
    return tuple(out.shape) == (M, N) and out.dtype == _half and out.is_contiguous()


def _is_x(x, K: int) -> bool:
    """A contiguous fp16 CUDA tensor [M, K]."""
    if _half is None:
        _bind_torch()
    shape = x.shape
    return len(shape) == 2 and shape[1] == K and x.dtype == _half and x.is_cuda and x.is_contiguous()


def qlinear_decode_static(desc: Desc, packed, x, out=None, stream=None):
    """Decode (M <= 8) without a handle and without any allocation inside the library: the caller passes the
    packed device tensor, x and (optionally) the output tensor; see include/qlinear.h."""
    import torch
    if (x.dim() != 2 or x.shape[1] != desc.K or x.dtype != torch.float16 or not x.is_cuda or not x.is_contiguous()):
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_decode_static (x must be contiguous fp16 CUDA [M, K])")
    if (not packed.is_cuda or packed.dtype != torch.uint8 or not packed.is_contiguous()
            or packed.numel() < qlinear_packed_size(desc) or packed.device != x.device):
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_decode_static (packed must be a contiguous uint8 CUDA tensor of the packed size)")
    M = x.shape[0]
    if out is None:
        out = torch.empty((M, desc.N), dtype=torch.float16, device=x.device)
    elif out.shape != (M, desc.N) or out.dtype != torch.float16 or not out.is_contiguous() or out.device != x.device:
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_decode_static (bad out tensor)")
    _check(lib.qlinear_decode_static(ctypes.byref(desc.c()), packed.data_ptr(),
                                     x.data_ptr(), out.data_ptr(), M,
                                     x.device.index or 0, _stream_ptr(stream)), "qlinear_decode_static")
    return out


def qlinear_forward_group_raw(lins, x_ptr: int, y_ptrs, M: int, stream=None) -> None:
    """qlinear_forward_group on raw device pointers: the layers `lins` applied to one x."""
    n = len(lins)
    hs = (ctypes.c_void_p * n)(*[l._h for l in lins])
    ys = (ctypes.c_void_p * n)(*map(int, y_ptrs))
    _check(lib.qlinear_forward_group(hs, n, x_ptr, ys, M, _stream_ptr(stream)), "qlinear_forward_group")


def qlinear_forward_batch_raw(lins, x_ptrs, y_ptrs, M: int, stream=None) -> None:
    """qlinear_forward_batch on raw device pointers: layer i applied to its own input x_ptrs[i]."""
    n = len(lins)
    hs = (ctypes.c_void_p * n)(*[l._h for l in lins])
    xs = (ctypes.c_void_p * n)(*map(int, x_ptrs))
    ys = (ctypes.c_void_p * n)(*map(int, y_ptrs))
    _check(lib.qlinear_forward_batch(hs, n, xs, ys, M, _stream_ptr(stream)), "qlinear_forward_batch")


def qlinear_forward_batch(lins, xs, outs=None, stream=None):
    """xs: one fp16 CUDA tensor [M, K] per layer -> list of fp16 [M, N_i] (one launch for M <= 8: up to 4 layers, 8 if they are int8)."""
    import torch
    K, M = lins[0].desc.K, xs[0].shape[0]
    if len(xs) != len(lins):
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_batch (one input per layer)")
    for x in xs:
        if x.dim() != 2 or tuple(x.shape) != (M, K) or x.dtype != torch.float16 or not x.is_cuda or not x.is_contiguous():
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_batch (every x must be contiguous fp16 CUDA [M, K])")
    if outs is None:
        outs = [xs[0].new_empty((M, l.desc.N)) for l in lins]
    for l, o in zip(lins, outs):
        if not _is_out(o, M, l.desc.N):
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_batch (bad out tensor)")
    qlinear_forward_batch_raw(lins, [x.data_ptr() for x in xs], [o.data_ptr() for o in outs], M, stream)
    return outs


def kv_scores_batch(caches, q_rows, stream=None):
    """The score product of up to 8 KV heads in one launch: caches[i].scores(q_rows[i]) for every i (paper Section 3.8)."""
    return qlinear_forward_batch([c.k for c in caches], q_rows, stream=stream)


def qlinear_forward_group(lins, x, outs=None, stream=None):
    """x: fp16 CUDA tensor [M, K] -> list of fp16 [M, N_i], one per layer (one launch for M <= 8)."""
    if outs is None:
        y = (_native or _bind_torch()).forward_group(lins, x, _raw(stream))
        if y is not None:
            return y
    K = lins[0].desc.K
    if not _is_x(x, K):
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_group (x must be contiguous fp16 CUDA [M, K])")
    M = x.shape[0]
    if outs is None:
        outs = [x.new_empty((M, l.desc.N)) for l in lins]
    for l, o in zip(lins, outs):
        if not _is_out(o, M, l.desc.N):
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_group (bad out tensor)")
    qlinear_forward_group_raw(lins, x.data_ptr(), [o.data_ptr() for o in outs], M, stream)
    return outs


def qlinear_forward_gated_raw(gate, up, x_ptr: int, y_ptr: int, M: int, act: str, stream=None) -> None:
    _check(lib.qlinear_forward_gated(gate._h, up._h, x_ptr, y_ptr, M, ACTIVATIONS[act],
                                     _stream_ptr(stream)), "qlinear_forward_gated")


def qlinear_forward_gated(gate, up, x, act: str = "silu", out=None, stream=None):
    """y = act(x . W_gate^T) * (x . W_up^T) as fp16 [M, N], from one fused launch where the shape allows."""
    if act in ACTIVATIONS:
        y = (_native or _bind_torch()).forward_gated(gate._native, up._native, x, ACTIVATIONS[act], out, _raw(stream))
        if y is not None:
            return y
    K, N = gate.desc.K, gate.desc.N
    if not _is_x(x, K):
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_gated (x must be contiguous fp16 CUDA [M, K])")
    if act not in ACTIVATIONS:
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_gated (unknown activation)")
    M = x.shape[0]
    if out is None:
        out = x.new_empty((M, N))
    elif not _is_out(out, M, N):
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_gated (bad out tensor)")
    qlinear_forward_gated_raw(gate, up, x.data_ptr(), out.data_ptr(), M, act, stream)
    return out


def qlinear_quantize_activations(x, stream=None):
    """x fp16 CUDA [M, K] -> (xq int8 [M, K], scale fp32 [M]): the prefill stage's quantisation kernel."""
    import torch
    if x.dim() != 2 or x.dtype != torch.float16 or not x.is_cuda or not x.is_contiguous() or x.shape[1] % 32:
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_quantize_activations (x must be contiguous fp16 CUDA [M, K], K % 32 == 0)")
    M, K = x.shape
    xq = torch.empty((M, K), dtype=torch.int8, device=x.device)
    scale = torch.empty((M,), dtype=torch.float32, device=x.device)
    _check(lib.qlinear_quantize_activations(x.data_ptr(), xq.data_ptr(), scale.data_ptr(),
                                            M, K, x.device.index or 0, _stream_ptr(stream)), "qlinear_quantize_activations")
    return xq, scale


def qlinear_residual_rmsnorm(x, residual, gamma, eps: float, gamma_offset: float = 0.0, h_out=None, y_out=None, want_h=True, stream=None):
    """x, residual (or None) fp16 CUDA [M, K], gamma fp16 [K] -> (h, y): h = x + residual, y = rmsnorm(h) * (gamma_offset + gamma).
    h_out / y_out may be given (h_out may be x or residual: in place); want_h=False skips the h output (h is then None)."""
    hy = (_native or _bind_torch()).residual_rmsnorm(x, residual, gamma, eps, gamma_offset, h_out, y_out, want_h, _raw(stream))
    if hy is not None:
        return hy
    dev = x.get_device()
    def ok(t, shape):
        return t.dtype == _half and t.get_device() == dev and t.is_cuda and t.is_contiguous() and tuple(t.shape) == shape
    if x.dim() != 2 or not ok(x, tuple(x.shape)) or x.shape[1] % 8 or x.shape[1] < 8:
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_residual_rmsnorm (x must be contiguous fp16 CUDA [M, K], K % 8 == 0)")
    M, K = x.shape
    if (residual is not None and not ok(residual, (M, K))) or not ok(gamma, (K,)):
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_residual_rmsnorm (residual [M, K] / gamma [K] fp16 on x's device)")
    if (y_out is not None and not ok(y_out, (M, K))) or (h_out is not None and not ok(h_out, (M, K))):
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_residual_rmsnorm (bad output tensor)")
    if y_out is None:
        y_out = x.new_empty((M, K))
    if h_out is None and want_h:
        h_out = x.new_empty((M, K))
    _check(lib.qlinear_residual_rmsnorm(x.data_ptr(), residual.data_ptr() if residual is not None else None,
                                        gamma.data_ptr(), float(eps), float(gamma_offset),
                                        h_out.data_ptr() if h_out is not None else None, y_out.data_ptr(),
                                        M, K, dev, _stream_ptr(stream)), "qlinear_residual_rmsnorm")
    return h_out, y_out


def qlinear_rope_qkv(q, k, v, pos, cos, sin, B: int, S: int, h_q: int, h_kv: int, d_h: int, stream=None):
    """q fp16 CUDA [B*S, h_q*d_h], k, v [B*S, h_kv*d_h], pos int32 [B*S], cos / sin fp32 [n_pos, d_h/2]
    -> (q_out [B*h_kv, S*h_q/h_kv, d_h], k_out [B*h_kv, S, d_h], v_out [B*h_kv, S, d_h]): rotary embedding + layout change."""
    qkv = (_native or _bind_torch()).rope_qkv(q, k, v, pos, cos, sin, B, S, h_q, h_kv, d_h, _raw(stream))
    if qkv is not None:
        return qkv
    import torch
    T = B * S
    dev = q.get_device()
    def ok(t, dtype, shape):
        return t.dtype == dtype and t.get_device() == dev and t.is_cuda and t.is_contiguous() and tuple(t.shape) == shape
    if h_kv < 1 or h_q % h_kv or d_h % 16 or not ok(q, torch.float16, (T, h_q * d_h)) or not ok(k, torch.float16, (T, h_kv * d_h)) \
            or not ok(v, torch.float16, (T, h_kv * d_h)) or not ok(pos, torch.int32, (T,)) or cos.dim() != 2 \
            or not ok(cos, torch.float32, (cos.shape[0], d_h // 2)) or not ok(sin, torch.float32, tuple(cos.shape)):
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_rope_qkv (shapes / dtypes: see the header)")
    g = h_q // h_kv
    q_out = q.new_empty((B * h_kv, S * g, d_h))
    k_out = q.new_empty((B * h_kv, S, d_h))
    v_out = q.new_empty((B * h_kv, S, d_h))
    p = lambda t: t.data_ptr()
    _check(lib.qlinear_rope_qkv(p(q), p(k), p(v), p(pos), p(cos), p(sin), cos.shape[0], p(q_out), p(k_out), p(v_out), B, S, h_q, h_kv, d_h,
                                dev, _stream_ptr(stream)), "qlinear_rope_qkv")
    return q_out, k_out, v_out


ROPE_SCALINGS = {None: 0, "linear": 1, "ntk": 2, "llama3": 3, "yarn": 4}
_ROPE_TURNS = {3: (1.0, 4.0), 4: (1.0, 32.0)}                            # (slow, fast) that the models with these scalings use


def _on_stream(device, stream):
    """(raw handle, context): the caller's stream, or the current one of the device; what is allocated in the context belongs to it."""
    import torch
    if stream is not None:
        return stream.cuda_stream, torch.cuda.stream(stream)
    if _raw_stream is None:
        _bind_torch()
    return _raw_stream(device.index), torch.cuda.device(device)


def _check_i32(where: str, *numbers) -> None:
    """Refuses what int32_t does not hold: ctypes would pass its lower 32 bits."""
    if not all(-2 ** 31 <= n < 2 ** 31 for n in numbers):
        raise QLinearError(QL_ERR_INVALID_ARG, where + " (a number beyond 32 bits)")


def qlinear_rope_tables(n_pos: int, rot: int, base: float = 10000.0, scaling=None, factor: float = 1.0, original: int = 8192, slow=None, fast=None, first: int = 0, device=None, stream=None):
    """(cos, sin) fp32 CUDA [n_pos, rot / 2] of the positions first .. first + n_pos - 1, with the frequency scaling of a long context (None, "linear", "ntk",
    "llama3", "yarn"; the formulas: include/qlinear.h), for qlinear_rope_qkv and PagedKV.append."""
    import torch
    kind = ROPE_SCALINGS.get(scaling)
    if kind is None or n_pos < 0 or rot < 0:
        raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_rope_tables (unknown scaling or negative size)")
    _check_i32("qlinear_rope_tables", n_pos, rot, original, first)
    turns = _ROPE_TURNS.get(kind, (1.0, 2.0))
    slow, fast = turns[0] if slow is None else slow, turns[1] if fast is None else fast
    if device is not None:
        device = torch.device(device)
        if device.type != "cuda":
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_rope_tables (device must be a CUDA device)")
    y = (_serving or _bind_torch()._serving).rope_tables(n_pos, rot, base, kind, factor, original, slow, fast, first, None if device is None else device.index, _raw(stream))
    if y is not None:
        return y
    s = qlinear_rope_scaling(kind, original, factor, slow, fast)
    if device is None or device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    st, where = _on_stream(device, stream)
    with where:
        cos, sin = (torch.empty((n_pos, rot // 2), dtype=torch.float32, device=device) for _ in range(2))
    _check(lib.qlinear_rope_tables(cos.data_ptr(), sin.data_ptr(), first, n_pos, rot, base, ctypes.byref(s), device.index, st), "qlinear_rope_tables")
    return cos, sin


def qlinear_adjust_logits(logits, tokens=None, start=None, n_prompt=None, repetition=None, presence=None, frequency=None, bias_ids=None, bias_values=None, bias_start=None, mask=None,
                          out=None, stream=None):
    """logits fp16 or fp32 CUDA [rows, vocab] (rows may be strided) -> the same type and shape: penalties for the tokens of every row's history
    (tokens int32 [n], start int32 [rows + 1], n_prompt int32 [rows]; repetition, presence, frequency fp32 [rows]), biases (bias_ids int32 [m], bias_values fp32 [m], bias_start int32
    [rows + 1]), and the mask of allowed tokens (int32 [rows, >= ceil(vocab / 32)], one bit a token).  out may be logits."""
    y = (_serving or _bind_torch()._serving).adjust_logits(logits, tokens, start, n_prompt, repetition, presence, frequency, bias_ids, bias_values, bias_start, mask, out, _raw(stream))
    if y is not None:
        return y
    import torch
    where = "qlinear_adjust_logits"
    def vector(t, dtype, n):
        return t is None or (t.dtype == dtype and t.device == logits.device and t.dim() == 1 and t.is_contiguous() and (n is None or t.shape[0] == n))
    def rows_of(t, dtype):
        return t.dtype == dtype and t.is_cuda and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1)
    if logits.dtype not in (torch.float16, torch.float32) or not rows_of(logits, logits.dtype):
        raise QLinearError(QL_ERR_INVALID_ARG, where + " (logits must be fp16 or fp32 CUDA [rows, vocab])")
    R, V = logits.shape
    _check_i32(where, R, V, *(t.numel() for t in (tokens, bias_ids) if t is not None))
    if (tokens is None) != (start is None) or not vector(tokens, torch.int32, None) or not vector(start, torch.int32, R + 1) or not vector(n_prompt, torch.int32, R) \
            or not all(vector(t, torch.float32, R) for t in (repetition, presence, frequency)):
        raise QLinearError(QL_ERR_INVALID_ARG, where + " (history: int32 tokens, start [rows + 1], n_prompt [rows]; fp32 penalties [rows])")
    if len({bias_ids is None, bias_values is None, bias_start is None}) != 1 or not vector(bias_ids, torch.int32, None) \
            or not vector(bias_values, torch.float32, None if bias_ids is None else bias_ids.shape[0]) or not vector(bias_start, torch.int32, R + 1):
        raise QLinearError(QL_ERR_INVALID_ARG, where + " (biases: int32 ids, fp32 values, int32 start [rows + 1])")
    if mask is not None and (not rows_of(mask, torch.int32) or mask.device != logits.device or mask.shape[0] != R or mask.shape[1] < (V + 31) // 32):
        raise QLinearError(QL_ERR_INVALID_ARG, where + " (mask must be int32 [rows, ceil(vocab / 32)])")
    st, here = _on_stream(logits.device, stream)
    if out is None:
        with here:
            out = torch.empty((R, V), dtype=logits.dtype, device=logits.device)
    elif not rows_of(out, logits.dtype) or tuple(out.shape) != (R, V) or out.device != logits.device:
        raise QLinearError(QL_ERR_INVALID_ARG, where + " (bad out tensor)")
    ptr = lambda t: None if t is None else t.data_ptr()
    count = lambda t: 0 if t is None else t.shape[0]
    ld = lambda t: max(t.stride(0), t.shape[1]) if t.shape[0] <= 1 else t.stride(0)
    _check(lib.qlinear_adjust_logits(ptr(logits), ld(logits), ptr(out), ld(out), R, V, int(logits.dtype == torch.float32), ptr(tokens), count(tokens), ptr(start), ptr(n_prompt),
                                     ptr(repetition), ptr(presence), ptr(frequency), ptr(bias_ids), ptr(bias_values), ptr(bias_start), count(bias_ids),
                                     ptr(mask), 0 if mask is None else ld(mask), logits.device.index, st), where)
    return out


class PagedKV:
    """A paged KV cache held in 4 bits (qlinear_paged_* in include/qlinear.h): the pool of pages, and the calls on a batch of sequences.

    A batch is (page_table int32 [B, pages], kv_len int32 [B], q_start int32 [B + 1]) on the cache's device: the rows q_start[b] .. q_start[b + 1] - 1 of a
    call are the last tokens of sequence b, which has kv_len[b] with them.  Which pages a sequence gets is the caller's business.  Rows of no sequence are left as they
    are in a caller's output, and hold nothing in a new one."""

    def __init__(self, n_pages: int, page_size: int, h_kv: int, d_h: int, device=None):
        import torch
        _bind_torch()
        _check_i32("PagedKV", n_pages, page_size, h_kv, d_h)
        self.n_pages, self.page_size, self.h_kv, self.d_h = n_pages, page_size, h_kv, d_h
        desc = qlinear_paged_desc(n_pages, page_size, h_kv, d_h)
        size = int(lib.qlinear_paged_page_bytes(ctypes.byref(desc)))
        if size == 0:
            raise QLinearError(QL_ERR_UNSUPPORTED, "PagedKV (page_size a power of two from 16 to 1024, d_h 64, 128 or 256)")
        self.pool = torch.zeros((n_pages, size), dtype=torch.uint8, device="cuda" if device is None else device)
        self.device = self.pool.device
        # (the pool's zeros are written on the current stream; calls on others come behind them)
        torch.cuda.current_stream(self.device).synchronize()
        h = ctypes.c_void_p()
        _check(lib.qlinear_paged_create(ctypes.byref(desc), self.pool.data_ptr(), self.device.index, ctypes.byref(h)), "qlinear_paged_create")
        self._h = h
        self._native = (h.value, h_kv, d_h, self.device.index)

    def _rows(self, t, heads, where):
        """(leading dimension of t, its heads): fp16 [T, heads * d_h] or [T, heads, d_h], the elements of a row in order."""
        d = self.d_h
        ok = t.dtype == _half and t.device == self.device and t.dim() in (2, 3) and (t.shape[-1] == d if t.dim() == 3 else t.shape[1] % d == 0)
        ok = ok and t.stride(-1) == 1 and (t.dim() == 2 or t.shape[1] == 1 or t.stride(1) == d)
        n = 0 if not ok else t.shape[1] if t.dim() == 3 else t.shape[1] // d
        if not ok or n < 1 or (heads is not None and n != heads):
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (rows must be fp16 CUDA [T, heads * d_h] or [T, heads, d_h] on the cache's device)")
        return (max(t.stride(0), n * d) if t.shape[0] <= 1 else t.stride(0)), n

    def _batch(self, page_table, kv_len, q_start, T, where):
        import torch
        ok = all(t.dtype == torch.int32 and t.device == self.device for t in (page_table, kv_len, q_start)) and page_table.dim() == 2
        B, W = page_table.shape if ok else (0, 0)
        if not ok or tuple(kv_len.shape) != (B,) or tuple(q_start.shape) != (B + 1,) or not kv_len.is_contiguous() or not q_start.is_contiguous() or (W > 1 and page_table.stride(1) != 1):
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (int32 page_table [B, pages], kv_len [B], q_start [B + 1] on the cache's device)")
        _check_i32(where, B, W, T)
        return page_table.data_ptr() if page_table.numel() else None, max(page_table.stride(0), W) if B <= 1 else page_table.stride(0), W, kv_len.data_ptr(), q_start.data_ptr(), B, T

    def append(self, k, v, page_table, kv_len, q_start, q=None, cos=None, sin=None, interleaved: bool = False, q_out=None, stream=None):
        """Writes the keys and values of the batch's new tokens to their pages, queries and keys turned by the tables on the way; returns the turned queries, shaped like q (None without)."""
        y = _serving.paged_append(self._native, k, v, page_table, kv_len, q_start, q, cos, sin, interleaved, q_out, _raw(stream))
        if y is not None:
            return y if q is not None else None
        import torch
        where = "qlinear_paged_append"
        T = k.shape[0]
        k_ld, _ = self._rows(k, self.h_kv, where)
        v_ld, _ = self._rows(v, self.h_kv, where)
        batch = self._batch(page_table, kv_len, q_start, T, where)
        if v.shape[0] != T or (q is not None and q.shape[0] != T):
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (q, k and v differ in rows)")
        rot = n_pos = 0
        if (cos is None) != (sin is None):
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (cos and sin come together)")
        if cos is not None:
            if any(t.dtype != torch.float32 or t.device != self.device or t.dim() != 2 or not t.is_contiguous() for t in (cos, sin)) or cos.shape != sin.shape:
                raise QLinearError(QL_ERR_INVALID_ARG, where + " (cos, sin must be contiguous fp32 CUDA [n_pos, rot / 2])")
            n_pos, rot = cos.shape[0], 2 * cos.shape[1]
            _check_i32(where, n_pos, rot)
        st, here = _on_stream(self.device, stream)
        q_ld = out_ld = h_q = 0
        if q is not None:
            q_ld, h_q = self._rows(q, None, where)
            _check_i32(where, h_q)
            if q_out is None:
                with here:
                    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            out_ld, n = self._rows(q_out, h_q, where)
            if q_out.shape != q.shape:
                raise QLinearError(QL_ERR_INVALID_ARG, where + " (bad q_out tensor)")
        elif q_out is not None:
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (q_out without q)")
        ptr = lambda t: None if t is None else t.data_ptr()
        _check(lib.qlinear_paged_append(self._h, ptr(q), q_ld, k.data_ptr(), k_ld, v.data_ptr(), v_ld, ptr(q_out), out_ld, h_q, *batch, ptr(cos), ptr(sin), n_pos, rot, int(bool(interleaved)), st), where)
        return q_out

    def read(self, page_table, kv_len, q_start, T: int, stream=None):
        """(k, v) fp16 [T, h_kv, d_h]: what the cache holds of the batch's T rows (zeros where the table gives them no page)."""
        y = _serving.paged_read(self._native, page_table, kv_len, q_start, T, _raw(stream))
        if y is not None:
            return y
        import torch
        where = "qlinear_paged_read"
        if T < 0:
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (negative T)")
        batch = self._batch(page_table, kv_len, q_start, T, where)
        st, here = _on_stream(self.device, stream)
        with here:
            k, v = (torch.empty((T, self.h_kv, self.d_h), dtype=torch.float16, device=self.device) for _ in range(2))
        _check(lib.qlinear_paged_read(self._h, *batch, k.data_ptr(), v.data_ptr(), st), where)
        return k, v

    def attention(self, q, page_table, kv_len, q_start, max_q: int, scale=None, softcap: float = 0.0, window: int = 0, out=None, stream=None):
        """q fp16 [T, h_q * d_h] or [T, h_q, d_h] -> fp16 [T, h_q, d_h]: causal attention of the batch's rows over their sequences in the cache; no sequence
        has more than max_q rows.  scale None: 1 / sqrt(d_h)."""
        scale = self.d_h ** -0.5 if scale is None else scale
        y = _serving.paged_attention(self._native, q, page_table, kv_len, q_start, max_q, scale, softcap, window, out, _raw(stream))
        if y is not None:
            return y
        import torch
        where = "qlinear_paged_attention"
        q_ld, h_q = self._rows(q, None, where)
        T = q.shape[0]
        batch = self._batch(page_table, kv_len, q_start, T, where)
        _check_i32(where, h_q, max_q, window)
        if h_q % self.h_kv or max_q < 0:
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (query heads a multiple of the KV heads, max_q >= 0)")
        st, here = _on_stream(self.device, stream)
        size = lib.qlinear_paged_attention_workspace(self._h, h_q, batch[5], max_q)
        with here:
            if out is None:
                out = torch.empty((T, h_q, self.d_h), dtype=torch.float16, device=self.device)
            work = torch.empty(size, dtype=torch.uint8, device=self.device)
        out_ld, n = self._rows(out, h_q, where)
        if out.shape[0] != T:
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (bad out tensor)")
        _check(lib.qlinear_paged_attention(self._h, q.data_ptr(), q_ld, out.data_ptr(), out_ld, h_q, *batch, max_q, scale, softcap, window, work.data_ptr(), size, st), where)
        return out

    def _ints(self, where, *tensors):
        """The addresses of int32 vectors (or None) on the cache's device, of the length that comes with each (None: any)."""
        import torch
        for t, n in tensors:
            if t is not None and (t.dtype != torch.int32 or t.device != self.device or t.dim() != 1 or not t.is_contiguous() or (n is not None and t.shape[0] != n) or t.shape[0] > 2 ** 31 - 1):
                raise QLinearError(QL_ERR_INVALID_ARG, where + " (int32 CUDA vectors of the right lengths on the cache's device)")
        return [None if t is None else t.data_ptr() for t, _ in tensors]

    def _table(self, table, where):
        """(address, leading dimension, columns, rows) of a page table."""
        import torch
        if table.dtype != torch.int32 or table.device != self.device or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (page_table int32 [rows, pages] on the cache's device)")
        n, W = table.shape
        _check_i32(where, n, W)
        return table.data_ptr() if table.numel() else None, max(table.stride(0), W) if n <= 1 else table.stride(0), W, n

    def _bounds(self, bounds, where):
        import torch
        ok = len(bounds) == 2 and all(t.device == self.device and t.is_contiguous() for t in bounds) and bounds[0].dtype == torch.int8 and bounds[1].dtype == torch.float32
        if not ok or tuple(bounds[0].shape) != (self.n_pages, self.h_kv, 2, self.d_h) or tuple(bounds[1].shape) != (self.n_pages, self.h_kv):
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (bounds: what key_bounds returns)")
        return bounds[0].data_ptr(), bounds[1].data_ptr()

    def fork(self, refs, page_table, parents, lengths, out=None, stream=None):
        """parents, lengths int32 [n] -> int32 [n, pages]: rows with the pages of the first lengths[i] tokens of row parents[i], -1 behind them; refs (int32 [n_pages], how many entries of the caller's page tables hold a
        page) counts the new entries.  out: rows to write them to, which hold no pages; they and page_table have no entry in common."""
        y = _serving.paged_fork(self._native, refs, page_table, parents, lengths, out, self.n_pages, _raw(stream))
        if y is not None:
            return y
        import torch
        where, n = "qlinear_paged_fork", parents.shape[0]
        table = self._table(page_table, where)
        at = self._ints(where, (refs, self.n_pages), (parents, n), (lengths, n))
        _check_i32(where, n)
        st, here = _on_stream(self.device, stream)
        if out is None:
            with here:
                out = torch.empty((n, table[2]), dtype=torch.int32, device=self.device)
        to = self._table(out, where)
        if to[2:] != (table[2], n):
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (bad out tensor)")
        _check(lib.qlinear_paged_fork(self._h, at[0], *table, at[1], at[2], n, to[0], to[1], st), where)
        return out

    def release(self, refs, page_table, rows, keep=None, stream=None) -> None:
        """Rows `rows` (int32 [n]) of the page table give back their pages behind their first keep[i] tokens (None: all of them)."""
        if _serving.paged_release(self._native, refs, page_table, rows, keep, self.n_pages, _raw(stream)) is not None:
            return
        where, n = "qlinear_paged_release", rows.shape[0]
        table = self._table(page_table, where)
        at = self._ints(where, (refs, self.n_pages), (rows, n), (keep, n))
        _check_i32(where, n)
        _check(lib.qlinear_paged_release(self._h, at[0], *table, at[1], at[2], n, _on_stream(self.device, stream)[0]), where)

    def reserve(self, refs, page_table, kv_len, q_start, T: int, stream=None):
        """Gives every sequence of the batch pages of its own for its T new rows, before they are appended: free ones where the page table has none, copies (in this cache's pool) where others hold the page too.  Returns int32 [1]: 0,
        or how many pages the pool is short of, in which case nothing has changed."""
        y = _serving.paged_reserve(self._native, refs, page_table, kv_len, q_start, T, self.n_pages, _raw(stream))
        if y is not None:
            return y
        import torch
        where = "qlinear_paged_reserve"
        batch = self._batch(page_table, kv_len, q_start, T, where)
        at = self._ints(where, (refs, self.n_pages))
        st, here = _on_stream(self.device, stream)
        size = lib.qlinear_paged_pages_workspace(self._h)
        with here:
            missing = torch.empty(1, dtype=torch.int32, device=self.device)
            work = torch.empty(size, dtype=torch.uint8, device=self.device)
        _check(lib.qlinear_paged_reserve(self._h, at[0], *batch, missing.data_ptr(), work.data_ptr(), size, st), where)
        return missing

    def compact(self, refs, page_table, bounds=None, stream=None):
        """Moves the live pages (refs > 0) to the front of the pool, with their entries of the page table, refs and (what key_bounds returns) summaries.  Returns int32 [n_pages]: where each page is now, -1 for free ones."""
        y = _serving.paged_compact(self._native, refs, page_table, None if bounds is None else bounds[0], None if bounds is None else bounds[1], self.n_pages, _raw(stream))
        if y is not None:
            return y
        import torch
        where = "qlinear_paged_compact"
        table = self._table(page_table, where)
        at = self._ints(where, (refs, self.n_pages))
        b = (None, None) if bounds is None else self._bounds(bounds, where)
        st, here = _on_stream(self.device, stream)
        size = lib.qlinear_paged_pages_workspace(self._h)
        with here:
            moved = torch.empty(self.n_pages, dtype=torch.int32, device=self.device)
            work = torch.empty(size, dtype=torch.uint8, device=self.device)
        _check(lib.qlinear_paged_compact(self._h, at[0], *table, *b, moved.data_ptr(), work.data_ptr(), size, st), where)
        return moved

    def key_bounds(self):
        """(int8 [n_pages, h_kv, 2, d_h], fp32 [n_pages, h_kv]), zeros: what `summarise` keeps of every page, the largest and the smallest key element per channel and the unit that they are held in."""
        import torch
        return (torch.zeros((self.n_pages, self.h_kv, 2, self.d_h), dtype=torch.int8, device=self.device), torch.zeros((self.n_pages, self.h_kv), dtype=torch.float32, device=self.device))

    def summarise(self, bounds, page_table, kv_len, q_start, T: int, stream=None) -> None:
        """Brings the summaries of the pages that the batch's T new rows lie in up to date, after they have been appended."""
        if _serving.paged_summarise(self._native, bounds[0], bounds[1], page_table, kv_len, q_start, T, self.n_pages, _raw(stream)) is not None:
            return
        where = "qlinear_paged_summarise"
        batch = self._batch(page_table, kv_len, q_start, T, where)
        _check(lib.qlinear_paged_summarise(self._h, *batch, *self._bounds(bounds, where), _on_stream(self.device, stream)[0]), where)

    def select(self, q, bounds, page_table, kv_len, q_start, budget: int, first: int = 1, recent: int = 1, out=None, stream=None):
        """q fp16 [T, h_q * d_h] or [T, h_q, d_h] -> int32 [T, h_kv, budget]: for every row and KV head the columns of its page table row that promise the largest scores by their summaries, the `first`
        first and the `recent` last ones always among them; ascending, -1 behind them."""
        y = _serving.paged_select(self._native, q, bounds[0], bounds[1], page_table, kv_len, q_start, budget, first, recent, out, self.n_pages, _raw(stream))
        if y is not None:
            return y
        import torch
        where = "qlinear_paged_select"
        q_ld, h_q = self._rows(q, None, where)
        T = q.shape[0]
        batch = self._batch(page_table, kv_len, q_start, T, where)
        _check_i32(where, h_q, budget, first, recent)
        if h_q % self.h_kv or budget < 1:
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (query heads a multiple of the KV heads, budget >= 1)")
        b = self._bounds(bounds, where)
        st, here = _on_stream(self.device, stream)
        if out is None:
            with here:
                out = torch.empty((T, self.h_kv, budget), dtype=torch.int32, device=self.device)
        elif out.dtype != torch.int32 or out.device != self.device or tuple(out.shape) != (T, self.h_kv, budget) or not out.is_contiguous():
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (bad out tensor)")
        _check(lib.qlinear_paged_select(self._h, q.data_ptr(), q_ld, h_q, *b, *batch, budget, first, recent, out.data_ptr(), st), where)
        return out

    def attention_selected(self, q, pages, page_table, kv_len, q_start, scale=None, softcap: float = 0.0, out=None, stream=None):
        """q fp16 [T, h_q * d_h] or [T, h_q, d_h] -> fp16 [T, h_q, d_h]: causal attention over the columns of the page table that pages (int32 [T, h_kv, budget], as `select` returns it) lists for each
        row and KV head.  scale None: 1 / sqrt(d_h)."""
        scale = self.d_h ** -0.5 if scale is None else scale
        y = _serving.paged_attention_selected(self._native, q, pages, page_table, kv_len, q_start, scale, softcap, out, _raw(stream))
        if y is not None:
            return y
        import torch
        where = "qlinear_paged_attention_selected"
        q_ld, h_q = self._rows(q, None, where)
        T = q.shape[0]
        batch = self._batch(page_table, kv_len, q_start, T, where)
        if h_q % self.h_kv:
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (query heads a multiple of the KV heads)")
        if pages.dtype != torch.int32 or pages.device != self.device or pages.dim() != 3 or tuple(pages.shape[:2]) != (T, self.h_kv) or not pages.is_contiguous():
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (pages must be contiguous int32 [T, h_kv, budget] on the cache's device)")
        _check_i32(where, h_q, pages.shape[2])
        st, here = _on_stream(self.device, stream)
        size = lib.qlinear_paged_attention_selected_workspace(self._h, h_q)
        with here:
            if out is None:
                out = torch.empty((T, h_q, self.d_h), dtype=torch.float16, device=self.device)
            work = torch.empty(size, dtype=torch.uint8, device=self.device)
        out_ld, n = self._rows(out, h_q, where)
        if out.shape[0] != T:
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (bad out tensor)")
        _check(lib.qlinear_paged_attention_selected(self._h, q.data_ptr(), q_ld, out.data_ptr(), out_ld, h_q, pages.data_ptr() if pages.numel() else None, pages.shape[2], *batch, scale, softcap, work.data_ptr(), size, st), where)
        return out

    def attention_shared(self, q, page_table, kv_len, q_start, max_q: int, group_start, prefix_len, scale=None, softcap: float = 0.0, out=None, stream=None):
        """`attention` (without a window) of a batch of which sequences share their beginning: the sequences group_start[g] .. group_start[g + 1] - 1 (int32 [groups + 1]) have the same first prefix_len[g] (int32 [groups])
        tokens, which are read and multiplied once for all of them."""
        scale = self.d_h ** -0.5 if scale is None else scale
        y = _serving.paged_attention_shared(self._native, q, page_table, kv_len, q_start, max_q, group_start, prefix_len, scale, softcap, out, _raw(stream))
        if y is not None:
            return y
        import torch
        where = "qlinear_paged_attention_shared"
        q_ld, h_q = self._rows(q, None, where)
        T, G = q.shape[0], prefix_len.shape[0]
        batch = self._batch(page_table, kv_len, q_start, T, where)
        groups = self._ints(where, (group_start, G + 1), (prefix_len, G))
        _check_i32(where, h_q, max_q, G)
        if h_q % self.h_kv or max_q < 0:
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (query heads a multiple of the KV heads, max_q >= 0)")
        st, here = _on_stream(self.device, stream)
        size = lib.qlinear_paged_attention_shared_workspace(self._h, h_q, batch[2], batch[5], T, max_q, G)
        with here:
            if out is None:
                out = torch.empty((T, h_q, self.d_h), dtype=torch.float16, device=self.device)
            work = torch.empty(size, dtype=torch.uint8, device=self.device)
        out_ld, n = self._rows(out, h_q, where)
        if out.shape[0] != T:
            raise QLinearError(QL_ERR_INVALID_ARG, where + " (bad out tensor)")
        _check(lib.qlinear_paged_attention_shared(self._h, q.data_ptr(), q_ld, out.data_ptr(), out_ld, h_q, *batch, max_q, *groups, G, scale, softcap, work.data_ptr(), size, st), where)
        return out

    def device_status(self):
        detail = ctypes.c_uint32(0)
        st = lib.qlinear_paged_device_status(self._h, ctypes.byref(detail))
        return int(st), int(detail.value)

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib.qlinear_paged_destroy(self._h)
            self._h = None
            self._native = (0, 0, 0, 0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class QLinear:
    """One quantised linear layer resident on a GPU: owns the packed device tensor and the handle."""

    def __init__(self, desc: Desc, packed, device=None):
        import torch
        _bind_torch()
        self.desc = desc
        if isinstance(packed, np.ndarray):
            dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
            packed = torch.from_numpy(np.ascontiguousarray(packed, dtype=np.uint8)).to(dev)
        if not packed.is_cuda or packed.dtype != torch.uint8 or not packed.is_contiguous():
            raise QLinearError(QL_ERR_INVALID_ARG, "QLinear (packed must be a contiguous uint8 CUDA tensor)")
        if packed.numel() < qlinear_packed_size(desc):
            raise QLinearError(QL_ERR_INVALID_ARG, "QLinear (packed blob too small)")
        self.packed = packed                      # keeps the device memory alive
        self.device = packed.device
        h = ctypes.c_void_p()
        _check(lib.qlinear_create(ctypes.byref(desc.c()), packed.data_ptr(),
                                  self.device.index or 0, ctypes.byref(h)), "qlinear_create")
        self._h = h
        self._native = (h.value, desc.K, desc.N)

    @classmethod
    def from_weights(cls, q: np.ndarray, s: np.ndarray, bits: int, group: int = 0, device=None) -> "QLinear":
        desc = Desc(int(q.shape[0]), int(q.shape[1]), bits, group)
        return cls(desc, qlinear_pack(desc, q, s), device)

    def forward(self, x, out=None, stream=None):
        """x: fp16 CUDA tensor [M, K] -> y fp16 [M, N] (qlinear_forward on the current stream)."""
        y = _native.forward(self._native, x, out, _raw(stream))
        if y is not None:
            return y
        if not _is_x(x, self.desc.K):
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward (x must be contiguous fp16 CUDA [M, K])")
        M = x.shape[0]
        if out is None:
            out = x.new_empty((M, self.desc.N))
        elif not _is_out(out, M, self.desc.N):
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward (bad out tensor)")
        self.forward_raw(x.data_ptr(), out.data_ptr(), M, stream)
        return out

    def forward_a8(self, x, out=None, stream=None):
        """The decode call with int8 activations quantised inside the kernel (qlinear_forward_a8), M <= 8."""
        y = _native.forward_a8(self._native, x, out, _raw(stream))
        if y is not None:
            return y
        if not _is_x(x, self.desc.K):
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_a8 (x must be contiguous fp16 CUDA [M, K])")
        M = x.shape[0]
        if out is None:
            out = x.new_empty((M, self.desc.N))
        elif not _is_out(out, M, self.desc.N):
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_forward_a8 (bad out tensor)")
        _check(lib.qlinear_forward_a8(self._h, x.data_ptr(), out.data_ptr(), M, _stream_ptr(stream)),
               "qlinear_forward_a8")
        return out

    def forward_a8_raw(self, x_ptr: int, y_ptr: int, M: int, stream=None) -> None:
        _check(lib.qlinear_forward_a8(self._h, x_ptr, y_ptr, M, _stream_ptr(stream)), "qlinear_forward_a8")

    def forward_raw(self, x_ptr: int, y_ptr: int, M: int, stream=None) -> None:
        _check(lib.qlinear_forward(self._h, x_ptr, y_ptr, M, _stream_ptr(stream)),
               "qlinear_forward")

    def embed(self, ids, out=None, stream=None):
        """ids: int32 CUDA tensor [n] -> fp16 [n, K], the dequantised rows ids of the table (qlinear_embed)."""
        y = _native.embed(self._native, ids, out, _raw(stream))
        if y is not None:
            return y
        import torch
        if ids.dim() != 1 or ids.dtype != torch.int32 or not ids.is_cuda or not ids.is_contiguous():
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_embed (ids must be a contiguous int32 CUDA vector)")
        n = ids.shape[0]
        if out is None:
            out = torch.empty((n, self.desc.K), dtype=torch.float16, device=ids.device)
        elif out.shape != (n, self.desc.K) or out.dtype != torch.float16 or not out.is_contiguous():
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_embed (bad out tensor)")
        _check(lib.qlinear_embed(self._h, ids.data_ptr(), n, out.data_ptr(),
                                 _stream_ptr(stream)), "qlinear_embed")
        return out

    def path_for(self, M: int) -> int:
        return int(lib.qlinear_path_for(self._h, M))

    def debug_unpack(self, stream=None):
        import torch
        q = torch.empty((self.desc.N, self.desc.K), dtype=torch.int8, device=self.device)
        _check(lib.qlinear_debug_unpack_device(self._h, q.data_ptr(), _stream_ptr(stream)),
               "qlinear_debug_unpack_device")
        return q

    def debug_expire_wait(self, stream=None) -> None:
        """Runs the kernels' bounded wait on a barrier nothing completes (about a second); see device_status."""
        _check(lib.qlinear_debug_expire_wait(self._h, _stream_ptr(stream)), "qlinear_debug_expire_wait")

    def debug_null_launch(self, grid: int = 1, block: int = 32, stream=None) -> None:
        """Launches a kernel that does nothing (what a dependent launch costs on this machine)."""
        _check(lib.qlinear_debug_null_launch(self._h, grid, block, _stream_ptr(stream)), "qlinear_debug_null_launch")

    def device_status(self):
        detail = ctypes.c_uint32(0)
        st = lib.qlinear_device_status(self._h, ctypes.byref(detail))
        return int(st), int(detail.value)

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib.qlinear_destroy(self._h)
            self._h = self._native = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVCache:
    """One KV head's cache held as two int8 weight blobs (see include/qlinear.h, qlinear_kv_append): argument
    marshalling only -- the blobs start as the packed form of zero weights, every later byte is written by the library."""

    def __init__(self, cache_size: int, d_h: int, device="cuda:0"):
        import torch
        self.cache_size, self.d_h, self.length = cache_size, d_h, 0
        kd, vd = Desc(cache_size, d_h, 8, 0), Desc(d_h, cache_size, 8, 0)
        self.k = QLinear(kd, qlinear_pack(kd, np.zeros((cache_size, d_h), np.int8), np.zeros((cache_size, 1), np.float16)), device)
        self.v = QLinear(vd, qlinear_pack(vd, np.zeros((d_h, cache_size), np.int8), np.ones((d_h, 1), np.float16)), device)
        self.v_scale = torch.zeros((cache_size,), dtype=torch.float16, device=device)

    def append(self, k_new, v_new, stream=None):
        """k_new, v_new: fp16 CUDA [n_new, d_h], written to positions length .. length + n_new - 1."""
        import torch
        for t in (k_new, v_new):
            if t.dim() != 2 or t.shape[1] != self.d_h or t.dtype != torch.float16 or not t.is_cuda or not t.is_contiguous():
                raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_kv_append (k_new, v_new must be contiguous fp16 CUDA [n, d_h])")
        n = k_new.shape[0]
        if v_new.shape[0] != n:
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_kv_append (k_new and v_new differ in length)")
        _check(lib.qlinear_kv_append(self.k._h, self.v._h, k_new.data_ptr(), v_new.data_ptr(),
                                     self.v_scale.data_ptr(), self.length, n, _stream_ptr(stream)), "qlinear_kv_append")
        self.length += n

    def scores(self, q_rows, stream=None):
        """q_rows fp16 [R, d_h] -> fp16 [R, cache_size] (positions beyond `length` score 0)."""
        y = _native.kv_scores_one(self.k._native, q_rows, None, _raw(stream))
        if y is not None:
            return y
        if not _is_x(q_rows, self.d_h):
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_kv_scores (q_rows must be contiguous fp16 CUDA [R, d_h])")
        out = q_rows.new_empty((q_rows.shape[0], self.cache_size))
        _check(lib.qlinear_kv_scores(self.k._h, q_rows.data_ptr(), out.data_ptr(), q_rows.shape[0],
                                     _stream_ptr(stream)), "qlinear_kv_scores")
        return out

    def output(self, prob, stream=None):
        """prob fp16 [R, cache_size] -> fp16 [R, d_h]."""
        y = _native.kv_output(self.v._native, self.v_scale, prob, _raw(stream))
        if y is not None:
            return y
        if not _is_x(prob, self.cache_size):
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_kv_output (prob must be contiguous fp16 CUDA [R, cache_size])")
        tmp = prob.new_empty(prob.shape)
        out = prob.new_empty((prob.shape[0], self.d_h))
        _check(lib.qlinear_kv_output(self.v._h, prob.data_ptr(), self.v_scale.data_ptr(),
                                     tmp.data_ptr(), out.data_ptr(), prob.shape[0], _stream_ptr(stream)),
               "qlinear_kv_output")
        return out


class KVHeads:
    """The caches of all KV heads of one attention layer (n_heads <= 16 KVCache objects of equal shape), driven through
    the calls that serve every head in one launch (qlinear_kv_*_heads in include/qlinear.h): argument marshalling only."""

    def __init__(self, n_heads: int, cache_size: int, d_h: int, device="cuda:0"):
        self.heads = [KVCache(cache_size, d_h, device) for _ in range(n_heads)]
        self.n, self.cache_size, self.d_h, self.length = n_heads, cache_size, d_h, 0
        arr = ctypes.c_void_p * n_heads
        self._hk = arr(*[c.k._h for c in self.heads])
        self._hv = arr(*[c.v._h for c in self.heads])
        self._vs = arr(*[c.v_scale.data_ptr() for c in self.heads])
        self._native = (n_heads, cache_size, d_h, ctypes.addressof(self._hk), ctypes.addressof(self._hv), ctypes.addressof(self._vs))

    def append_raw(self, k_ptr: int, v_ptr: int, head_stride: int, token_stride: int, n_new: int, stream=None) -> None:
        _check(lib.qlinear_kv_append_heads(self._hk, self._hv, self.n, k_ptr, v_ptr, head_stride, token_stride,
                                           self._vs, self.length, n_new, _stream_ptr(stream)), "qlinear_kv_append_heads")
        self._appended(n_new)

    def _appended(self, n_new: int) -> None:
        self.length += n_new
        for c in self.heads:
            c.length = self.length

    def append(self, k_new, v_new, stream=None):
        """k_new, v_new: fp16 CUDA [n_heads, n_new, d_h] (the k_out / v_out of qlinear_rope_qkv)."""
        n_new = _native.kv_append(self._native, self.length, k_new, v_new, _raw(stream))
        if n_new is not None:
            return self._appended(n_new)
        import torch
        for t in (k_new, v_new):
            if t.dim() != 3 or t.shape[0] != self.n or t.shape[2] != self.d_h or t.dtype != torch.float16 or not t.is_cuda or not t.is_contiguous():
                raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_kv_append_heads (k_new, v_new must be contiguous fp16 CUDA [n_heads, n_new, d_h])")
        if k_new.shape != v_new.shape:
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_kv_append_heads (k_new and v_new differ in shape)")
        n_new = k_new.shape[1]
        self.append_raw(k_new.data_ptr(), v_new.data_ptr(), n_new * self.d_h, self.d_h, n_new, stream)

    def scores_raw(self, q_ptr: int, out_ptr: int, R: int, stream=None) -> None:
        _check(lib.qlinear_kv_scores_heads(self._hk, self.n, q_ptr, out_ptr, R, _stream_ptr(stream)),
               "qlinear_kv_scores_heads")

    def scores(self, q_rows, stream=None):
        """q_rows fp16 [n_heads, R, d_h] -> fp16 [n_heads, R, cache_size]."""
        y = _native.kv_scores(self._native, q_rows, _raw(stream))
        if y is not None:
            return y
        import torch
        if q_rows.dim() != 3 or q_rows.shape[0] != self.n or q_rows.shape[2] != self.d_h or q_rows.dtype != torch.float16 or not q_rows.is_cuda or not q_rows.is_contiguous():
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_kv_scores_heads (q_rows must be contiguous fp16 CUDA [n_heads, R, d_h])")
        out = q_rows.new_empty((self.n, q_rows.shape[1], self.cache_size))
        self.scores_raw(q_rows.data_ptr(), out.data_ptr(), q_rows.shape[1], stream)
        return out

    def output_raw(self, prob_ptr: int, out_ptr: int, R: int, stream=None) -> None:
        _check(lib.qlinear_kv_output_heads(self._hv, self.n, prob_ptr, self._vs, out_ptr, R, _stream_ptr(stream)),
               "qlinear_kv_output_heads")

    def output(self, prob, stream=None):
        """prob fp16 [n_heads, R, cache_size] -> fp16 [n_heads, R, d_h]."""
        y = _native.kv_output_heads(self._native, prob, _raw(stream))
        if y is not None:
            return y
        import torch
        if prob.dim() != 3 or prob.shape[0] != self.n or prob.shape[2] != self.cache_size or prob.dtype != torch.float16 or not prob.is_cuda or not prob.is_contiguous():
            raise QLinearError(QL_ERR_INVALID_ARG, "qlinear_kv_output_heads (prob must be contiguous fp16 CUDA [n_heads, R, cache_size])")
        out = prob.new_empty((self.n, prob.shape[1], self.d_h))
        self.output_raw(prob.data_ptr(), out.data_ptr(), prob.shape[1], stream)
        return out
