"""GB300 fused attention (prefill + Flash Decode): thin Python binding of ``libloomattn.so``.

Every function here only marshals arguments (tensor data pointers, sizes, the current
CUDA stream) into the C ABI declared in ``include/loom_attn.h``; all computation runs
in the library's CUDA kernels.  There is no fallback: if the compiled library is
missing, every call raises.  (Where ``_binding.so`` was built, the training and serving
entry points marshal their common case there.)

Two layers:

* ``capi()`` returns the ``ctypes.CDLL`` with argument types declared -- the raw C ABI,
  taking integer device pointers.
* Functions with the C names (``loom_attn_fwd``, ``loom_attn_decode``, ...) that take
  torch tensors, check their dtype/device/layout, and raise ``LoomError`` on a non-OK
  status.
"""
from __future__ import annotations

import ctypes
import functools
import operator
import os
import threading

__all__ = [
    "LoomError", "capi", "library_path", "STATUS",
    "loom_attn_fwd", "loom_attn_decode", "loom_attn_decode_noalloc", "loom_attn_decode_workspace_bytes",
    "loom_attn_decode_num_splits", "loom_attn_check_error", "loom_status_string",
    "loom_debug_set_timeout_ns", "loom_debug_inject", "loom_model_fwd_plan",
    "loom_model_fwd_time_us", "loom_model_decode_time_us", "FwdPlan", "loom_debug_prefill_design",
    "loom_model_fwd_plan_variant", "loom_model_heg_pipe", "loom_model_fwd_time_us_design",
    "loom_attn_decode_paged", "loom_attn_fwd_varlen", "loom_gemm_bf16", "loom_gemm_bf16_bt", "loom_gemm_tile_n", "loom_gemm_splits", "loom_gemm_cta_pair", "loom_model_gemm_time_us", "loom_debug_gemm_tile_n",
    "loom_debug_gemm_splits", "loom_debug_gemm_cta_pair", "loom_model_decode_cluster_time_us",
    "loom_attn_decode_form", "loom_decode_max_clusters", "loom_decode_persistent_slots", "loom_debug_decode_form",
    "loom_model_decode_persistent_time_us", "loom_model_decode_tc_time_us", "DECODE_SPLIT_MERGE", "DECODE_PERSISTENT", "DECODE_CLUSTER",
    "loom_debug_prefill_slots", "loom_debug_decode_stage_plan", "loom_debug_gemm_stages",
    "loom_debug_gemm_order", "loom_debug_decode_tensor_cores", "loom_attn_fwd_cluster",
    "loom_attn_bwd", "loom_attn_bwd_workspace_bytes", "loom_attn_bwd_varlen", "loom_attn_bwd_varlen_workspace_bytes",
    "loom_attn_bwd_plan", "loom_qkv_norm_rope", "loom_qkv_norm_rope_cache", "loom_qkv_norm_rope_bwd", "loom_qkv_norm_rope_bwd_workspace_bytes",
    "loom_attn_chunk_paged", "loom_attn_chunk_paged_workspace_bytes", "loom_paged_plan",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libloomattn.so")
_lock = threading.Lock()
_lib = None

STATUS = {
    0: "LOOM_OK", 1: "LOOM_ERR_INVALID_ARG", 2: "LOOM_ERR_UNSUPPORTED", 3: "LOOM_ERR_MISALIGNED",
    4: "LOOM_ERR_WORKSPACE", 5: "LOOM_ERR_CUDA", 6: "LOOM_ERR_TIMEOUT",
}


class FwdPlan(ctypes.Structure):
    """Mirror of ``loom_fwd_plan`` (include/loom_attn.h)."""
    _fields_ = [(n, ctypes.c_int) for n in ("design", "bm", "bn", "q_tiles", "s_buffers", "kv_slots",
                                             "b_lm", "b_ms", "smem_bytes", "tmem_cols")] + \
               [(n, ctypes.c_double) for n in ("t_load_ns", "t_mma_ns", "t_softmax_ns", "t_iter_ns")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class LoomError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)}")


def library_path() -> str:
    return _LIB_PATH


def capi() -> ctypes.CDLL:
    """The compiled library with its C signatures declared (raises if it is missing)."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(_LIB_PATH):
                raise RuntimeError(
                    f"{_LIB_PATH} is missing: build it with paper_2609_29219_gb300.build.build() "
                    "(there is no fallback implementation)")
            lib = ctypes.CDLL(_LIB_PATH)
            vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
            lib.loom_attn_fwd.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, f32, vp]
            lib.loom_attn_fwd.restype = i32
            lib.loom_attn_decode_num_splits.argtypes = [i32, i32, i32, i32, i32]
            lib.loom_attn_decode_num_splits.restype = i32
            lib.loom_attn_decode_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
            lib.loom_attn_decode_workspace_bytes.restype = sz
            lib.loom_attn_decode.argtypes = [vp, vp, vp, vp, vp, vp, vp, sz, i32, i32, i32, i32, i32,
                                             f32, i32, vp]
            lib.loom_attn_decode.restype = i32
            lib.loom_attn_decode_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, f32, i32,
                                                     vp]
            lib.loom_attn_decode_noalloc.restype = i32
            lib.loom_attn_check_error.argtypes = [vp]
            lib.loom_attn_check_error.restype = i32
            lib.loom_status_string.argtypes = [i32]
            lib.loom_status_string.restype = ctypes.c_char_p
            lib.loom_debug_set_timeout_ns.argtypes = [ctypes.c_uint64]
            lib.loom_debug_set_timeout_ns.restype = None
            lib.loom_debug_inject.argtypes = [i32]
            lib.loom_debug_inject.restype = None
            lib.loom_debug_prefill_design.argtypes = [i32]
            lib.loom_debug_prefill_design.restype = None
            lib.loom_model_fwd_plan.argtypes = [i32, ctypes.POINTER(FwdPlan)]
            lib.loom_model_fwd_plan.restype = i32
            lib.loom_model_fwd_plan_variant.argtypes = [i32, i32, ctypes.POINTER(FwdPlan)]
            lib.loom_model_fwd_plan_variant.restype = i32
            lib.loom_model_heg_pipe.argtypes = [ctypes.c_double] * 3 + [i32, i32]
            lib.loom_model_heg_pipe.restype = ctypes.c_double
            lib.loom_model_fwd_time_us.argtypes = [i32, i32, i32, i32, i32, i32]
            lib.loom_model_fwd_time_us.restype = ctypes.c_double
            lib.loom_model_fwd_time_us_design.argtypes = [i32] * 7
            lib.loom_model_fwd_time_us_design.restype = ctypes.c_double
            lib.loom_attn_decode_paged.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, i32, i32, i32, i32,
                                                   i32, i32, i32, i32, f32, i32, vp]
            lib.loom_attn_decode_paged.restype = i32
            lib.loom_attn_fwd_varlen.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32,
                                                 i32, f32, vp]
            lib.loom_attn_fwd_varlen.restype = i32
            lib.loom_gemm_bf16.argtypes = [vp, vp, vp, i32, i32, i32, vp]
            lib.loom_gemm_bf16.restype = i32
            lib.loom_gemm_bf16_bt.argtypes = [vp, vp, vp, i32, i32, i32, vp]
            lib.loom_gemm_bf16_bt.restype = i32
            lib.loom_gemm_tile_n.argtypes = [i32, i32, i32]
            lib.loom_gemm_tile_n.restype = i32
            lib.loom_gemm_splits.argtypes = [i32, i32, i32]
            lib.loom_gemm_splits.restype = i32
            lib.loom_gemm_cta_pair.argtypes = [i32, i32, i32]
            lib.loom_gemm_cta_pair.restype = i32
            lib.loom_model_gemm_time_us.argtypes = [i32] * 6
            lib.loom_model_gemm_time_us.restype = ctypes.c_double
            lib.loom_debug_gemm_tile_n.argtypes = [i32]
            lib.loom_debug_gemm_tile_n.restype = None
            lib.loom_debug_gemm_splits.argtypes = [i32]
            lib.loom_debug_gemm_splits.restype = None
            lib.loom_debug_gemm_cta_pair.argtypes = [i32]
            lib.loom_debug_gemm_cta_pair.restype = None
            lib.loom_model_decode_time_us.argtypes = [i32, i32, i32, i32, i32, i32, i32]
            lib.loom_model_decode_time_us.restype = ctypes.c_double
            lib.loom_model_decode_cluster_time_us.argtypes = [i32] * 8
            lib.loom_model_decode_cluster_time_us.restype = ctypes.c_double
            lib.loom_model_decode_persistent_time_us.argtypes = [i32] * 7
            lib.loom_model_decode_persistent_time_us.restype = ctypes.c_double
            lib.loom_model_decode_tc_time_us.argtypes = [i32] * 7
            lib.loom_model_decode_tc_time_us.restype = ctypes.c_double
            lib.loom_attn_fwd_cluster.argtypes = [i32] * 7
            lib.loom_attn_fwd_cluster.restype = i32
            lib.loom_attn_decode_form.argtypes = [i32] * 7 + [ctypes.POINTER(i32)]
            lib.loom_attn_decode_form.restype = i32
            lib.loom_decode_max_clusters.argtypes = [i32, i32, i32]
            lib.loom_decode_max_clusters.restype = i32
            lib.loom_decode_persistent_slots.argtypes = [i32, i32]
            lib.loom_decode_persistent_slots.restype = i32
            lib.loom_debug_decode_form.argtypes = [i32, i32]
            lib.loom_debug_decode_form.restype = None
            lib.loom_debug_prefill_slots.argtypes = [i32, i32]
            lib.loom_debug_prefill_slots.restype = i32
            lib.loom_debug_decode_stage_plan.argtypes = [i32, i32, i32]
            lib.loom_debug_decode_stage_plan.restype = i32
            lib.loom_debug_gemm_stages.argtypes = [i32]
            lib.loom_debug_gemm_stages.restype = None
            lib.loom_debug_gemm_order.argtypes = [i32, i32]
            lib.loom_debug_gemm_order.restype = None
            lib.loom_debug_decode_tensor_cores.argtypes = [i32]
            lib.loom_debug_decode_tensor_cores.restype = None
            i64 = ctypes.c_int64
            lib.loom_attn_bwd.argtypes = [vp] * 11 + [sz] + [i32] * 7 + [f32, vp]
            lib.loom_attn_bwd.restype = i32
            lib.loom_attn_bwd_workspace_bytes.argtypes = [i32] * 6
            lib.loom_attn_bwd_workspace_bytes.restype = sz
            lib.loom_attn_bwd_varlen.argtypes = [vp] * 13 + [sz] + [i32] * 9 + [f32, vp]
            lib.loom_attn_bwd_varlen.restype = i32
            lib.loom_attn_bwd_varlen_workspace_bytes.argtypes = [i32] * 6
            lib.loom_attn_bwd_varlen_workspace_bytes.restype = sz
            lib.loom_attn_bwd_plan.argtypes = [i32] * 8 + [vp]
            lib.loom_attn_bwd_plan.restype = i32
            norm = [vp, vp, i32, vp, vp, i32, i32, i32, vp]  # the weights, the tables and the positions
            lib.loom_qkv_norm_rope.argtypes = [vp, i64] + norm + [vp] * 3 + [i32] * 5 + [f32, vp]
            lib.loom_qkv_norm_rope.restype = i32
            lib.loom_qkv_norm_rope_cache.argtypes = [vp, i64] + norm + [vp] * 4 + [i32] * 7 + [f32, vp]
            lib.loom_qkv_norm_rope_cache.restype = i32
            lib.loom_qkv_norm_rope_bwd.argtypes = [vp] * 4 + [i64] + norm + [vp, i64, vp, vp, vp, sz] + [i32] * 5 + [f32, vp]
            lib.loom_qkv_norm_rope_bwd.restype = i32
            axes = norm + [i64, i32, vp]  # and the axes of the positions
            lib.loom_qkv_norm_rope_axes.argtypes = [vp, i64] + axes + [vp] * 3 + [i32] * 5 + [f32, vp]
            lib.loom_qkv_norm_rope_axes.restype = i32
            lib.loom_qkv_norm_rope_axes_cache.argtypes = [vp, i64] + axes + [vp] * 4 + [i32] * 7 + [f32, vp]
            lib.loom_qkv_norm_rope_axes_cache.restype = i32
            lib.loom_qkv_norm_rope_axes_bwd.argtypes = [vp] * 4 + [i64] + axes + [vp, i64, vp, vp, vp, sz] + [i32] * 5 + [f32, vp]
            lib.loom_qkv_norm_rope_axes_bwd.restype = i32
            lib.loom_attn_chunk_paged.argtypes = [vp] * 9 + [sz] + [i32] * 10 + [f32, vp]
            lib.loom_attn_chunk_paged.restype = i32
            lib.loom_attn_chunk_paged_workspace_bytes.argtypes = [i32] * 5
            lib.loom_attn_chunk_paged_workspace_bytes.restype = sz
            lib.loom_paged_plan.argtypes = [vp] * 11 + [i32] * 5 + [vp]
            lib.loom_paged_plan.restype = i32
            lib.loom_qkv_norm_rope_bwd_workspace_bytes.argtypes = [i32]
            lib.loom_qkv_norm_rope_bwd_workspace_bytes.restype = sz
            _lib = lib
    return _lib


# ------------------------------------------------------------------ marshalling helpers
# A decode step or a small prefill takes the device 5 to 10 us, so what these helpers cost per
# argument is what such a call costs.  GB300 host, us per call before and after: prefill of 128
# rows 16.4 -> 10.8, one decode step 15.3 -> 10.8, GEMM of 16 rows 15.0 -> 9.2.  Most of it was
# torch.cuda.current_stream (2.0; the raw stream 0.1), the outputs' torch.empty (3.7 between
# two launches; 1.7 by the call below), and the checks, lock and import statement per argument
# (0.45; 0.3 in one expression).
_torch_mod = None
_bf16 = _f32 = _i32 = _u8 = None  # torch's types


_empty_strided_cuda = None
_fast = None  # the compiled binding, where it can be used
_current_device = None  # torch's: the index of the current device
# Whether there is more than one: with one GPU every CUDA tensor is on it, and devices are not
# compared (GB300 host: 0.1 us a tensor).
_several = False


def _torch():
    global _torch_mod, _empty_strided_cuda, _bf16, _f32, _i32, _u8, _fast, _current_device, _several
    if _torch_mod is None:
        import torch
        try:  # what torch's generated code allocates by: no dispatch, on the current device
            from torch._C._dynamo.guards import _empty_strided_cuda as call
            if all(hasattr(torch._C, n) for n in ("_cuda_getDevice", "_len_torch_dispatch_stack",
                                                  "_len_torch_function_stack", "_get_deterministic_algorithms")):
                _empty_strided_cuda = call
        except ImportError:
            pass
        _bf16, _f32, _i32, _u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _several = torch.cuda.device_count() > 1
        _torch_mod = torch
        _fast = _compiled_binding(torch)
    return _torch_mod


def _compiled_binding(torch):
    """The compiled binding (csrc/binding.cpp), or None where it was not built, or for another torch."""
    try:
        from . import _binding
    except ImportError:
        return None
    if not torch.__version__.startswith(_binding.torch_version):
        return None
    lib = capi()
    _binding.set_up(
        tuple(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in (
            "loom_attn_bwd", "loom_attn_bwd_workspace_bytes", "loom_attn_bwd_varlen", "loom_attn_bwd_varlen_workspace_bytes",
            "loom_qkv_norm_rope", "loom_qkv_norm_rope_cache", "loom_qkv_norm_rope_bwd",
            "loom_qkv_norm_rope_bwd_workspace_bytes", "loom_qkv_norm_rope_axes", "loom_qkv_norm_rope_axes_cache",
            "loom_qkv_norm_rope_axes_bwd", "loom_attn_chunk_paged", "loom_attn_chunk_paged_workspace_bytes", "loom_paged_plan")))
    return _binding


def _fast_result(r, where):
    """The compiled binding's outputs; it returned a status where the C call refused."""
    if type(r) is tuple:
        return r
    raise LoomError(r, where)


def _new(shape, strides, dtype, t, like=False, stream=None):
    """An uninitialised contiguous tensor (strides: its strides) on CUDA tensor t's device
    (like: of t's shape and type), for a call on the stream.  It passes torch's dispatcher by
    only where nobody would miss the call: no dispatch or function mode, no deterministic mode
    (which fills new tensors), no subclass of Tensor."""
    if stream is not None and not _is_current(stream, t):
        return _new_on(stream, shape, dtype, t, like)
    if _direct(t):
        return _empty_strided_cuda(shape, strides, dtype)
    torch = _torch_mod
    return torch.empty_like(t) if like else torch.empty(shape, dtype=dtype, device=t.device)


def _is_current(stream, t):
    """Whether the stream given is the current one of tensor t's device."""
    return _stream_ptr(stream, t.device) == _stream_of(None, t)


def _new_on(stream, shape, dtype, t, like=False):
    """_new for a call on a stream given.  The allocator must know that the tensor is that stream's:
    memory of the current stream may still be in use by what is queued there, and is handed out again there
    as soon as the tensor is gone (scratch: when the call returns), whatever this stream does.  It is noted as
    used on the current stream too, where a program that waits for this one may read it."""
    torch = _torch_mod
    if not isinstance(stream, torch.cuda.Stream):
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        # (0 and 1: the default stream's handles)
        stream = torch.cuda.ExternalStream(handle, t.device) if handle > 1 else torch.cuda.default_stream(t.device)
    if stream.device != t.device:
        raise ValueError(f"the stream is of {stream.device}, the tensors are on {t.device}")
    with torch.cuda.stream(stream):
        new = torch.empty_like(t) if like else torch.empty(shape, dtype=dtype, device=t.device)
    new.record_stream(torch.cuda.current_stream(t.device))
    return new


def _direct(t):
    """Whether new tensors on tensor t's device may pass the dispatcher by (see _new).  t is a call's first
    tensor, which is on the current device."""
    c = _torch_mod._C
    return (_empty_strided_cuda is not None and type(t) is _torch_mod.Tensor and not c._len_torch_dispatch_stack()
            and not c._len_torch_function_stack() and not c._get_deterministic_algorithms())


def _maker(t, stream):
    """What makes uninitialised contiguous tensors on tensor t's device, of (shape, strides, type):
    _new for a call that makes several (GB300 host: 0.9 us a tensor, 1.3 by _new)."""
    if stream is not None and not _is_current(stream, t):
        return lambda shape, strides, dtype: _new_on(stream, shape, dtype, t)
    if _direct(t):
        return _empty_strided_cuda
    return lambda shape, strides, dtype: _torch_mod.empty(shape, dtype=dtype, device=t.device)


def _workspace(need, t, stream):
    """Scratch of a decode call."""
    if stream is not None and not _is_current(stream, t):
        return _new_on(stream, (max(need, 16),), _u8, t)
    return _torch_mod.empty(max(need, 16), dtype=_u8, device=t.device)


def _on_current(t, name):
    """The device index of a call's first tensor: where the kernels run, so it must be the current one."""
    d = t.get_device()
    if d != _current_device():
        raise ValueError(f"{name} is on cuda:{d}, which is not the current device")
    return d


def _together(first, *others):
    """Whether a call's tensors (those that there are) are on the first's device."""
    d = first.get_device()
    return all(t is None or t.get_device() == d for t in others)


def _ptr(t, name, dtype, ndim, dev=None):
    """_dev_ptr of a tensor that passes its checks, in one expression (it names what fails)."""
    if (isinstance(t, _torch_mod.Tensor) and t.is_cuda and t.dtype is dtype and t.dim() == ndim
            and t.is_contiguous() and (dev is None or t.get_device() == dev)):
        return t.data_ptr()
    return _dev_ptr(t, name, dtype, ndim, dev)


def _dev_ptr(t, name, dtype=None, ndim=None, dev=None):
    """Pointer of a contiguous CUDA tensor (dev: on that device), or what it is not."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got shape {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dev is not None and t.get_device() != dev:
        raise ValueError(f"{name} is on cuda:{t.get_device()}, the call's first tensor on cuda:{dev}")
    return t.data_ptr()


def _stream_of(stream, t):
    """The given stream, or the current one of tensor t's device, as an integer."""
    if stream is None:
        raw = getattr(_torch_mod._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(t.get_device())
    return _stream_ptr(stream, t.device)


def _stream_ptr(stream, device):
    torch = _torch()
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(status: int, where: str):
    if status:
        raise LoomError(status, where)


# ------------------------------------------------------------------ C-ABI functions
# stream: None (the current one), a torch stream or a handle.  Outputs and scratch that a call on
# a stream given allocates belong to that stream, as under torch.cuda.stream.
def loom_attn_fwd(q, k, v, o=None, lse=None, *, causal=False, scale=None, stream=None,
                  return_lse=False):
    """Prefill attention.  q [B,Hq,Sq,D], k/v [B,Hkv,Skv,D] bf16 CUDA tensors.

    Writes ``o`` ([B,Hq,Sq,D] bf16, allocated if None) and, if given (or
    ``return_lse``), ``lse`` ([B,Hq,Sq] fp32).  Returns ``o`` or ``(o, lse)``.
    """
    torch = _torch()
    bf16 = torch.bfloat16
    qp = _ptr(q, "q", bf16, 4)
    dev = _on_current(q, "q") if _several else None
    kp = _ptr(k, "k", bf16, 4, dev)
    vp_ = _ptr(v, "v", bf16, 4, dev)
    B, Hq, Sq, D = q.shape
    Bk, Hkv, Skv, Dk = k.shape
    if v.shape != k.shape or Bk != B or Dk != D:
        raise ValueError("q/k/v shapes disagree")
    if o is None:
        o = _new((B, Hq, Sq, D), (Hq * Sq * D, Sq * D, D, 1), bf16, q, True, stream)
    if o.shape != q.shape:
        raise ValueError("o must have q's shape")
    op = _ptr(o, "o", bf16, 4, dev)
    if lse is None and return_lse:
        lse = _new((B, Hq, Sq), (Hq * Sq, Sq, 1), torch.float32, q, stream=stream)
    lp = None
    if lse is not None:
        if tuple(lse.shape) != (B, Hq, Sq):
            raise ValueError("lse must be [B, Hq, Sq]")
        lp = _dev_ptr(lse, "lse", torch.float32, None, dev)
    if scale is None:
        scale = D ** -0.5
    st = (_lib or capi()).loom_attn_fwd(qp, kp, vp_, op, lp, B, Hq, Hkv, Sq, Skv, D, int(bool(causal)), float(scale),
                                        _stream_of(stream, q))
    _check(st, "loom_attn_fwd")
    return (o, lse) if (return_lse or lse is not None) else o


def loom_attn_decode_num_splits(B, Hq, Hkv, Skv, D) -> int:
    return int(capi().loom_attn_decode_num_splits(B, Hq, Hkv, Skv, D))


def loom_attn_decode_workspace_bytes(B, Hq, Hkv, Skv, D, num_splits=0) -> int:
    return int(capi().loom_attn_decode_workspace_bytes(B, Hq, Hkv, Skv, D, num_splits))


def _decode_operands(q, k_cache, v_cache, seqlens_k, o, lse, return_lse, stream):
    """Pointers and sizes of the contiguous decode entry points' tensor arguments, outputs, and the device."""
    torch = _torch()
    bf16 = torch.bfloat16
    qp = _ptr(q, "q", bf16, 4)
    dev = _on_current(q, "q") if _several else None
    kp = _ptr(k_cache, "k_cache", bf16, 4, dev)
    vp_ = _ptr(v_cache, "v_cache", bf16, 4, dev)
    B, Hq, Sq, D = q.shape
    Bk, Hkv, Skv, Dk = k_cache.shape
    if Sq != 1 or v_cache.shape != k_cache.shape or Bk != B or Dk != D:
        raise ValueError("decode takes q [B,Hq,1,D] and k/v caches [B,Hkv,Skv,D]")
    sp = None
    if seqlens_k is not None:
        if tuple(seqlens_k.shape) != (B,):
            raise ValueError("seqlens_k must be [B]")
        sp = _ptr(seqlens_k, "seqlens_k", torch.int32, 1, dev)
    if o is None:
        o = _new((B, Hq, 1, D), (Hq * D, D, D, 1), bf16, q, True, stream)
    op = _ptr(o, "o", bf16, 4, dev)
    if lse is None and return_lse:
        lse = _new((B, Hq), (Hq, 1), torch.float32, q, stream=stream)
    lp = None
    if lse is not None:
        if lse.numel() != B * Hq:
            raise ValueError("lse must hold B*Hq values")
        lp = _dev_ptr(lse, "lse", torch.float32, None, dev)
    return (qp, kp, vp_, sp, op, lp), (B, Hq, Hkv, Skv, D), o, lse, dev


def loom_attn_decode(q, k_cache, v_cache, seqlens_k=None, o=None, lse=None, workspace=None, *,
                     scale=None, num_splits=0, stream=None, return_lse=False):
    """Flash Decode.  q [B,Hq,1,D], k_cache/v_cache [B,Hkv,Skv,D] bf16, seqlens_k [B] int32.

    ``workspace`` is a CUDA uint8 tensor of at least ``loom_attn_decode_workspace_bytes``
    bytes (allocated here if None).  Returns ``o`` or ``(o, lse)``.
    """
    torch = _torch()
    (qp, kp, vp_, sp, op, lp), (B, Hq, Hkv, Skv, D), o, lse, dev = _decode_operands(
        q, k_cache, v_cache, seqlens_k, o, lse, return_lse, stream)
    if workspace is None:
        need = loom_attn_decode_workspace_bytes(B, Hq, Hkv, Skv, D, num_splits)
        workspace = _workspace(need, q, stream)
    wp = _dev_ptr(workspace, "workspace", None, None, dev)
    if scale is None:
        scale = D ** -0.5
    st = (_lib or capi()).loom_attn_decode(qp, kp, vp_, sp, op, lp, wp, workspace.numel() * workspace.element_size(),
                                           B, Hq, Hkv, Skv, D, float(scale), int(num_splits), _stream_of(stream, q))
    _check(st, "loom_attn_decode")
    return (o, lse) if (return_lse or lse is not None) else o


def loom_attn_decode_noalloc(q, k_cache, v_cache, seqlens_k=None, o=None, lse=None, *, scale=None,
                             num_splits=0, stream=None, return_lse=False):
    """Flash Decode with the partials in the library's built-in scratch array (no
    workspace argument, no device allocation by the library).  Arguments and results as
    ``loom_attn_decode``; problems whose partials exceed the array raise LOOM_ERR_WORKSPACE."""
    (qp, kp, vp_, sp, op, lp), (B, Hq, Hkv, Skv, D), o, lse, _ = _decode_operands(
        q, k_cache, v_cache, seqlens_k, o, lse, return_lse, stream)
    if scale is None:
        scale = D ** -0.5
    st = (_lib or capi()).loom_attn_decode_noalloc(qp, kp, vp_, sp, op, lp, B, Hq, Hkv, Skv, D, float(scale),
                                                   int(num_splits), _stream_of(stream, q))
    _check(st, "loom_attn_decode_noalloc")
    return (o, lse) if (return_lse or lse is not None) else o


def loom_attn_fwd_varlen(q, k, v, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, o=None, lse=None, *, causal=False,
                         scale=None, stream=None, return_lse=False):
    """Prefill over a ragged batch.  q [total_q, Hq, D], k/v [total_k, Hkv, D] bf16;
    cu_seqlens_q / cu_seqlens_k [B + 1] int32 on the device; max_seqlen_q an int.
    Returns ``o`` ([total_q, Hq, D]) or ``(o, lse)`` with lse [Hq, total_q]."""
    torch = _torch()
    bf16 = torch.bfloat16
    qp = _ptr(q, "q", bf16, 3)
    dev = _on_current(q, "q") if _several else None
    kp = _ptr(k, "k", bf16, 3, dev)
    vp_ = _ptr(v, "v", bf16, 3, dev)
    total_q, Hq, D = q.shape
    total_k, Hkv, Dk = k.shape
    if v.shape != k.shape or Dk != D:
        raise ValueError("varlen prefill takes q [total_q, Hq, D] and k/v [total_k, Hkv, D]")
    cqp = _ptr(cu_seqlens_q, "cu_seqlens_q", torch.int32, 1, dev)
    ckp = _ptr(cu_seqlens_k, "cu_seqlens_k", torch.int32, 1, dev)
    if cu_seqlens_q.numel() != cu_seqlens_k.numel() or cu_seqlens_q.numel() < 2:
        raise ValueError("cu_seqlens_q and cu_seqlens_k must both be [B + 1]")
    B = cu_seqlens_q.numel() - 1
    if o is None:
        o = _new((total_q, Hq, D), (Hq * D, D, 1), bf16, q, True, stream)
    op = _ptr(o, "o", bf16, 3, dev)
    if lse is None and return_lse:
        lse = _new((Hq, total_q), (total_q, 1), torch.float32, q, stream=stream)
    lp = None
    if lse is not None:
        if lse.numel() != Hq * total_q:
            raise ValueError("lse must hold Hq*total_q values")
        lp = _dev_ptr(lse, "lse", torch.float32, None, dev)
    if scale is None:
        scale = D ** -0.5
    st = (_lib or capi()).loom_attn_fwd_varlen(qp, kp, vp_, op, lp, cqp, ckp, B, Hq, Hkv, total_q, total_k,
                                               int(max_seqlen_q), D, int(bool(causal)), float(scale),
                                               _stream_of(stream, q))
    _check(st, "loom_attn_fwd_varlen")
    return (o, lse) if (return_lse or lse is not None) else o


def loom_attn_decode_paged(q, k_cache, v_cache, block_table, seqlens_k, o=None, lse=None, workspace=None, *,
                           scale=None, num_splits=0, stream=None, return_lse=False, layout="nhd"):
    """Flash Decode over a paged cache.  q [B,Hq,1,D]; k_cache/v_cache bf16, [num_pages,
    page_size, Hkv, D] (layout "nhd") or [num_pages, Hkv, page_size, D] (layout "hnd");
    block_table [B, max_pages] int32; seqlens_k [B] int32 (all on the device).  Returns
    ``o`` or ``(o, lse)``."""
    torch = _torch()
    bf16 = torch.bfloat16
    qp = _ptr(q, "q", bf16, 4)
    dev = _on_current(q, "q") if _several else None
    kp = _ptr(k_cache, "k_cache", bf16, 4, dev)
    vp_ = _ptr(v_cache, "v_cache", bf16, 4, dev)
    B, Hq, Sq, D = q.shape
    if layout not in ("nhd", "hnd"):
        raise ValueError("layout is 'nhd' or 'hnd'")
    if layout == "nhd":
        num_pages, page_size, Hkv, Dk = k_cache.shape
    else:
        num_pages, Hkv, page_size, Dk = k_cache.shape
    if Sq != 1 or v_cache.shape != k_cache.shape or Dk != D:
        raise ValueError("paged decode takes q [B,Hq,1,D] and two caches of one shape")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = block_table.shape[1]
    tp = _ptr(block_table, "block_table", torch.int32, 2, dev)
    if tuple(seqlens_k.shape) != (B,):
        raise ValueError("seqlens_k must be [B]")
    sp = _ptr(seqlens_k, "seqlens_k", torch.int32, 1, dev)
    if o is None:
        o = _new((B, Hq, 1, D), (Hq * D, D, D, 1), bf16, q, True, stream)
    op = _ptr(o, "o", bf16, 4, dev)
    if lse is None and return_lse:
        lse = _new((B, Hq), (Hq, 1), torch.float32, q, stream=stream)
    lp = None
    if lse is not None:
        if lse.numel() != B * Hq:
            raise ValueError("lse must hold B*Hq values")
        lp = _dev_ptr(lse, "lse", torch.float32, None, dev)
    Skv = max_pages * page_size
    if workspace is None:
        need = loom_attn_decode_workspace_bytes(B, Hq, Hkv, Skv, D, num_splits)
        workspace = _workspace(need, q, stream)
    wp = _dev_ptr(workspace, "workspace", None, None, dev)
    if scale is None:
        scale = D ** -0.5
    st = (_lib or capi()).loom_attn_decode_paged(
        qp, kp, vp_, tp, sp, op, lp, wp, workspace.numel() * workspace.element_size(), B, Hq, Hkv, num_pages, page_size,
        max_pages, 0 if layout == "nhd" else 1, D, float(scale), int(num_splits), _stream_of(stream, q))
    _check(st, "loom_attn_decode_paged")
    return (o, lse) if (return_lse or lse is not None) else o


def loom_attn_chunk_paged_workspace_bytes(B, Hq, Hkv, total_q, D) -> int:
    return int(capi().loom_attn_chunk_paged_workspace_bytes(B, Hq, Hkv, total_q, D))


@functools.lru_cache(maxsize=256)
def _chunk_need(device, *sizes):  # (the devices' SMs may differ)
    return capi().loom_attn_chunk_paged_workspace_bytes(*sizes)


def loom_attn_chunk_paged(q, k_cache, v_cache, block_table, cu_seqlens_q, seqlens_k, o=None, lse=None, workspace=None, *,
                          causal=True, scale=None, stream=None, return_lse=False, layout="nhd"):
    """Attention of each sequence's new tokens over its keys in a paged cache (theirs among them).

    q [total_q, Hq, D]: the new tokens, packed; k_cache/v_cache bf16, [num_pages, page_size, Hkv, D]
    (layout "nhd") or [num_pages, Hkv, page_size, D] ("hnd"); block_table [B, max_pages], cu_seqlens_q
    [B + 1] and seqlens_k [B] int32, all on the device.  Tokens from cu_seqlens_q[B] on are padding, whose
    rows are left as they were.  ``workspace``: a CUDA uint8 tensor of at least
    ``loom_attn_chunk_paged_workspace_bytes`` bytes (allocated here if None).  Returns ``o``
    ([total_q, Hq, D]) or ``(o, lse)`` with lse [Hq, total_q]."""
    _torch()
    if layout not in ("nhd", "hnd"):
        raise ValueError("layout is 'nhd' or 'hnd'")
    if _fast is not None and o is None and lse is None and workspace is None and stream is None:
        r = _fast.chunk(q, k_cache, v_cache, block_table, cu_seqlens_q, seqlens_k, causal, scale, layout == "hnd", bool(return_lse))
        if r is not None:
            r = _fast_result(r, "loom_attn_chunk_paged")
            return r if return_lse else r[0]
    qp = _ptr(q, "q", _bf16, 3)
    dev = _on_current(q, "q") if _several else None
    kp = _ptr(k_cache, "k_cache", _bf16, 4, dev)
    vp_ = _ptr(v_cache, "v_cache", _bf16, 4, dev)
    total_q, Hq, D = q.shape
    if layout == "nhd":
        num_pages, page_size, Hkv, Dk = k_cache.shape
    else:
        num_pages, Hkv, page_size, Dk = k_cache.shape
    if v_cache.shape != k_cache.shape or Dk != D:
        raise ValueError("the chunk's attention takes q [total_q, Hq, D] and two caches of one shape")
    tp = _ptr(block_table, "block_table", _i32, 2, dev)
    cp = _ptr(cu_seqlens_q, "cu_seqlens_q", _i32, 1, dev)
    sp = _ptr(seqlens_k, "seqlens_k", _i32, 1, dev)
    B, max_pages = block_table.shape
    if cu_seqlens_q.shape[0] != B + 1 or seqlens_k.shape[0] != B:
        raise ValueError("block_table, cu_seqlens_q and seqlens_k must be [B, max_pages], [B + 1] and [B]")
    if max(B, max_pages) > 0x7fffffff:  # (the C call's numbers have 32 bits)
        raise LoomError(2, "loom_attn_chunk_paged")
    if o is None:
        o = _new((total_q, Hq, D), (Hq * D, D, 1), _bf16, q, True, stream)
    elif o.shape != q.shape:
        raise ValueError("o must have q's shape")
    op = _ptr(o, "o", _bf16, 3, dev)
    if lse is None and return_lse:
        lse = _new((Hq, total_q), (total_q, 1), _f32, q, stream=stream)
    lp = None
    if lse is not None:
        lp = _ptr(lse, "lse", _f32, 2, dev)
        if tuple(lse.shape) != (Hq, total_q):
            raise ValueError("lse must be [Hq, total_q]")
    if workspace is None:
        wbytes = _chunk_need(q.get_device(), B, Hq, Hkv, total_q, D)
        workspace = _new((max(wbytes, 16),), (1,), _u8, q, stream=stream)
        wp = workspace.data_ptr()
    else:
        wp = _dev_ptr(workspace, "workspace", None, None, dev)
        wbytes = workspace.numel() * workspace.element_size()
    st = (_lib or capi()).loom_attn_chunk_paged(
        qp, kp, vp_, tp, cp, sp, op, lp, wp, wbytes, B, Hq, Hkv, total_q, num_pages, page_size, max_pages,
        0 if layout == "nhd" else 1, D, 1 if causal else 0, D ** -0.5 if scale is None else float(scale), _stream_of(stream, q))
    _check(st, "loom_attn_chunk_paged")
    return (o, lse) if lse is not None else o


def loom_paged_plan(new_lens, lens, block_table, free_pages, free_count, num_tokens, page_size, seqlens_k=None,
                    free_count_out=None, cu_seqlens=None, positions=None, slots=None, granted=None, *, stream=None):
    """A serving step's bookkeeping on the device, from the requests' lengths.

    new_lens and lens [B] int32: the tokens that each request brings to the step (negative: it is over,
    and its pages go back to the list) and those that it has in the cache; block_table [B, max_pages]
    int32, updated with the pages taken; free_pages [num_pages] int32 with free_count [1] int32 of
    them free; num_tokens: the tokens that the step has room for (those past the last request's are padding).
    A request that the table, the tokens or the free pages have no room for is refused whole.

    Writes and returns ``cu_seqlens`` [B + 1], ``seqlens_k`` [B] (may be lens), ``positions`` and ``slots``
    [num_tokens] and ``granted`` [B] (allocated if None); the free pages that are left go to
    ``free_count_out`` (None: to free_count)."""
    _torch()
    if _fast is not None and cu_seqlens is None and positions is None and slots is None and stream is None:
        r = _fast.plan(new_lens, lens, block_table, free_pages, free_count, free_count if free_count_out is None else free_count_out,
                       seqlens_k, granted, num_tokens, page_size)
        if r is not None:
            return _fast_result(r, "loom_paged_plan")
    T, page_size = operator.index(num_tokens), operator.index(page_size)  # (no fraction is cut off)
    if T < 0:
        raise ValueError("num_tokens must not be negative")
    if max(T, abs(page_size)) > 0x7fffffff:  # (the C call's numbers have 32 bits)
        raise ValueError("num_tokens and page_size must be below 2^31")
    np_ = _ptr(new_lens, "new_lens", _i32, 1)
    dev = _on_current(new_lens, "new_lens") if _several else None
    B = new_lens.shape[0]
    lp, tp = _ptr(lens, "lens", _i32, 1, dev), _ptr(block_table, "block_table", _i32, 2, dev)
    fp, cp = _ptr(free_pages, "free_pages", _i32, 1, dev), _ptr(free_count, "free_count", _i32, 1, dev)
    if lens.shape[0] != B or block_table.shape[0] != B or free_count.shape[0] != 1:
        raise ValueError("new_lens, lens, block_table and free_count must be [B], [B], [B, max_pages] and [1]")
    if max(*block_table.shape, free_pages.shape[0]) > 0x7fffffff:
        raise LoomError(2, "loom_paged_plan")
    if free_count_out is None:
        free_count_out = free_count
    outs = []
    for t, name, n in ((free_count_out, "free_count_out", 1), (cu_seqlens, "cu_seqlens", B + 1), (seqlens_k, "seqlens_k", B),
                       (positions, "positions", T), (slots, "slots", T), (granted, "granted", B)):
        if t is None:
            t = _new((n,), (1,), _i32, new_lens, stream=stream)
        elif _ptr(t, name, _i32, 1, dev) is None or t.shape[0] != n:
            raise ValueError(f"{name} must be [{n}]")
        outs.append(t)
    st = (_lib or capi()).loom_paged_plan(
        np_, lp, tp, fp, cp, *(t.data_ptr() for t in outs), B, T, free_pages.shape[0], page_size, block_table.shape[1],
        _stream_of(stream, new_lens))
    _check(st, "loom_paged_plan")
    return tuple(outs[1:])


@functools.lru_cache(maxsize=256)
def _bwd_need(varlen, *sizes):
    lib = capi()
    return (lib.loom_attn_bwd_varlen_workspace_bytes if varlen else lib.loom_attn_bwd_workspace_bytes)(*sizes)


@functools.lru_cache(maxsize=4)
def _norm_bwd_need(D):
    return capi().loom_qkv_norm_rope_bwd_workspace_bytes(D)


# The checks of the entry points below take most of a small call's time if each tensor goes through
# _ptr, so they are one expression that names nothing, and what fails it is looked at again by name;
# and the common case goes through the compiled binding.  GB300 host, us per call with _ptr / one
# expression / compiled (the C call in it): backward of 128 rows 25.0 / 19.9 / 9 (4), norm and
# rotation 17.6 / 14.7 / 5.4 (2), into a cache 14.4 / 12.9 / 3.8 (2), its gradients 27.2 / 22.1 /
# 8 (3).
def _bwd_checked(do, q, k, v, o, lse, dlse, dq, dk, dv, ndim):
    """The backward entry points' tensors, named if they are not what they should be."""
    _dev_ptr(q, "q", _bf16, ndim)
    dev = q.get_device()
    for t, name in ((k, "k"), (v, "v"), (do, "do"), (o, "o")):
        _dev_ptr(t, name, _bf16, ndim, dev)
    if v.shape != k.shape or k.shape[-1] != q.shape[-1] or (ndim == 4 and k.shape[0] != q.shape[0]):
        raise ValueError("q/k/v shapes disagree")
    for t, name in ((do, "do"), (o, "o")):
        if t.shape != q.shape:
            raise ValueError(f"{name} must have q's shape")
    if lse is None:
        raise TypeError("lse is needed: call the forward pass with return_lse=True")
    _dev_ptr(lse, "lse", _f32, None, dev)
    if dlse is not None:
        _dev_ptr(dlse, "dlse", _f32, None, dev)
        if dlse.shape != lse.shape:
            raise ValueError("dlse must have lse's shape")
    for t, like, name in ((dq, q, "dq"), (dk, k, "dk"), (dv, v, "dv")):
        if t is not None:
            _dev_ptr(t, name, _bf16, ndim, dev)
            if t.shape != like.shape:
                raise ValueError(f"{name} must have {name[1]}'s shape")


def _bwd_fine(do, q, k, v, o, lse, dlse, qs, ks):
    try:
        return (q.is_cuda and q.dtype is _bf16 and q.is_contiguous() and do.is_cuda and do.dtype is _bf16 and do.is_contiguous()
                and o.is_cuda and o.dtype is _bf16 and o.is_contiguous() and k.is_cuda and k.dtype is _bf16
                and k.is_contiguous() and v.is_cuda and v.dtype is _bf16 and v.is_contiguous() and lse.is_cuda
                and lse.dtype is _f32 and lse.is_contiguous() and do.shape == qs and o.shape == qs and v.shape == ks
                and (dlse is None or (dlse.is_cuda and dlse.dtype is _f32 and dlse.is_contiguous() and dlse.shape == lse.shape))
                and (not _several or _together(q, do, k, v, o, lse, dlse)))
    except AttributeError:
        return False


def loom_attn_bwd_workspace_bytes(B, Hq, Hkv, Sq, Skv, D) -> int:
    return int(capi().loom_attn_bwd_workspace_bytes(B, Hq, Hkv, Sq, Skv, D))


def loom_attn_bwd_varlen_workspace_bytes(B, Hq, Hkv, total_q, total_k, D) -> int:
    return int(capi().loom_attn_bwd_varlen_workspace_bytes(B, Hq, Hkv, total_q, total_k, D))


def loom_attn_bwd_plan(B, Hq, Hkv, Sq, Skv, D, causal=False, ragged=False) -> dict:
    """How ``loom_attn_bwd`` (ragged: ``loom_attn_bwd_varlen``, Sq and Skv the totals) deals its work: the
    shares of the items of 128 keys and of 128 query rows, and the planes of kv and of query heads whose
    items are dealt together (0: ragged)."""
    plan = (ctypes.c_int * 4)()
    _check(capi().loom_attn_bwd_plan(B, Hq, Hkv, Sq, Skv, D, int(bool(causal)), int(bool(ragged)), plan), "loom_attn_bwd_plan")
    return dict(zip(("kv_shares", "q_shares", "kv_block", "q_block"), plan))


def loom_attn_bwd(do, q, k, v, o, lse, dq=None, dk=None, dv=None, workspace=None, *, causal=False, scale=None, dlse=None,
                  stream=None):
    """Gradients of ``loom_attn_fwd``.  do and o [B,Hq,Sq,D], q, k, v as the forward call had them,
    lse [B,Hq,Sq] as it returned it; dlse: the gradient of lse, or None.

    ``workspace`` is a CUDA uint8 tensor of at least ``loom_attn_bwd_workspace_bytes`` bytes
    (allocated here if None).  Writes and returns ``dq, dk, dv`` (allocated if None)."""
    _torch()
    if _fast is not None and dq is None and dk is None and dv is None and workspace is None and stream is None:
        r = _fast.attn_bwd(do, q, k, v, o, lse, dlse, causal, scale)
        if r is not None:
            return _fast_result(r, "loom_attn_bwd")
    try:
        qs, ks = q.shape, k.shape
        B, Hq, Sq, D = qs
        Bk, Hkv, Skv, Dk = ks
        fine = Bk == B and Dk == D
    except (AttributeError, ValueError):
        fine = False
    if not fine or dq is not None or dk is not None or dv is not None or not _bwd_fine(do, q, k, v, o, lse, dlse, qs, ks):
        _bwd_checked(do, q, k, v, o, lse, dlse, dq, dk, dv, 4)
    if tuple(lse.shape) != (B, Hq, Sq):
        raise ValueError("lse must be [B, Hq, Sq]")
    dev = _on_current(q, "q") if _several else None
    new = _maker(q, stream)
    if dq is None:
        dq = new(tuple(qs), (Hq * Sq * D, Sq * D, D, 1), _bf16)
    if dk is None:
        dk = new(tuple(ks), (Hkv * Skv * D, Skv * D, D, 1), _bf16)
    if dv is None:
        dv = new(tuple(ks), (Hkv * Skv * D, Skv * D, D, 1), _bf16)
    if workspace is None:
        wbytes = _bwd_need(False, B, Hq, Hkv, Sq, Skv, D)
        workspace = new((max(wbytes, 16),), (1,), _u8)
        wp = workspace.data_ptr()
    else:
        wp = _dev_ptr(workspace, "workspace", None, None, dev)
        wbytes = workspace.numel() * workspace.element_size()
    st = (_lib or capi()).loom_attn_bwd(
        do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
        None if dlse is None else dlse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), wp, wbytes, B, Hq, Hkv, Sq, Skv,
        D, 1 if causal else 0, D ** -0.5 if scale is None else float(scale), _stream_of(stream, q))
    if st:
        raise LoomError(st, "loom_attn_bwd")
    return dq, dk, dv


def loom_attn_bwd_varlen(do, q, k, v, o, lse, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k, dq=None, dk=None,
                         dv=None, workspace=None, *, causal=False, scale=None, dlse=None, stream=None):
    """Gradients of ``loom_attn_fwd_varlen``.  do, o and q [total_q, Hq, D], k and v [total_k, Hkv, D],
    lse (and dlse) [Hq, total_q]; cu_seqlens_q / cu_seqlens_k [B + 1] int32 on the device; the
    longest lengths as ints.  Writes and returns ``dq, dk, dv`` (allocated if None)."""
    _torch()
    if _fast is not None and dq is None and dk is None and dv is None and workspace is None and stream is None:
        r = _fast.attn_bwd_varlen(do, q, k, v, o, lse, dlse, causal, scale, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k)
        if r is not None:
            return _fast_result(r, "loom_attn_bwd_varlen")
    try:
        qs, ks = q.shape, k.shape
        total_q, Hq, D = qs
        total_k, Hkv, Dk = ks
        fine = Dk == D
    except (AttributeError, ValueError):
        fine = False
    if not fine or dq is not None or dk is not None or dv is not None or not _bwd_fine(do, q, k, v, o, lse, dlse, qs, ks):
        _bwd_checked(do, q, k, v, o, lse, dlse, dq, dk, dv, 3)
    if lse.numel() != Hq * total_q:
        raise ValueError("lse must hold Hq*total_q values")
    dev = _on_current(q, "q") if _several else None
    cqp, ckp = _ptr(cu_seqlens_q, "cu_seqlens_q", _i32, 1, dev), _ptr(cu_seqlens_k, "cu_seqlens_k", _i32, 1, dev)
    B = cu_seqlens_q.shape[0] - 1
    if cu_seqlens_k.shape[0] != B + 1 or B < 1:
        raise ValueError("cu_seqlens_q and cu_seqlens_k must both be [B + 1]")
    new = _maker(q, stream)
    if dq is None:
        dq = new(tuple(qs), (Hq * D, D, 1), _bf16)
    if dk is None:
        dk = new(tuple(ks), (Hkv * D, D, 1), _bf16)
    if dv is None:
        dv = new(tuple(ks), (Hkv * D, D, 1), _bf16)
    if workspace is None:
        wbytes = _bwd_need(True, B, Hq, Hkv, total_q, total_k, D)
        workspace = new((max(wbytes, 16),), (1,), _u8)
        wp = workspace.data_ptr()
    else:
        wp = _dev_ptr(workspace, "workspace", None, None, dev)
        wbytes = workspace.numel() * workspace.element_size()
    st = (_lib or capi()).loom_attn_bwd_varlen(
        do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
        None if dlse is None else dlse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), cqp, ckp, wp, wbytes, B, Hq, Hkv,
        total_q, total_k, int(max_seqlen_q), int(max_seqlen_k), D, 1 if causal else 0, D ** -0.5 if scale is None else float(scale),
        _stream_of(stream, q))
    if st:
        raise LoomError(st, "loom_attn_bwd_varlen")
    return dq, dk, dv


def _row_matrix(t, name, width, dev=None):
    """Pointer and row distance of a bf16 CUDA matrix whose rows are contiguous (dev: on that device)."""
    if not isinstance(t, _torch_mod.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype is not _bf16:
        raise TypeError(f"{name} must be {_bf16}, got {t.dtype}")
    if t.dim() != 2 or t.shape[1] != width or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be [T, {width}] with contiguous rows, got shape {tuple(t.shape)}")
    if dev is not None and t.get_device() != dev:
        raise ValueError(f"{name} is on cuda:{t.get_device()}, the call's first tensor on cuda:{dev}")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else width


def _norm_checked(qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, positions):
    """The norm-and-rotation entry points' shared tensors, named if they are not what they should be."""
    dev = qkv.get_device() if isinstance(qkv, _torch_mod.Tensor) and qkv.is_cuda else None
    for t, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        _dev_ptr(t, name, None, 1, dev)
        if t.dtype not in (_bf16, _f32):
            raise TypeError(f"{name} must be {_bf16} or {_f32}, got {t.dtype}")
    if k_weight.dtype is not q_weight.dtype:
        raise TypeError("q_weight and k_weight must have one type")
    if k_weight.shape != q_weight.shape:
        raise ValueError("q_weight and k_weight must both be [D]")
    _dev_ptr(cos, "cos", _f32, 2, dev), _dev_ptr(sin, "sin", _f32, 2, dev)
    if cos.shape != sin.shape:
        raise ValueError("cos and sin must both be [positions, rotary_dim / 2]")
    _row_matrix(qkv, "qkv", (num_heads + 2 * num_kv_heads) * q_weight.shape[0])
    if positions is not None:
        _dev_ptr(positions, "positions", _i32, 1, dev)
        if positions.shape[0] != qkv.shape[0]:
            raise ValueError("positions must be [T]")


@functools.lru_cache(maxsize=64)
def _axis_array(pair_axis):
    return (ctypes.c_int * len(pair_axis))(*pair_axis)


def _axes_operands(qkv, cos, positions, pair_axis):
    """The C arguments of positions on several axes, from positions on."""
    if positions is None:
        raise TypeError("positions are needed with pair_axis")
    _dev_ptr(positions, "positions", _i32, 2, qkv.get_device())
    if positions.shape[1] != qkv.shape[0]:
        raise ValueError("positions must be [axes, T] with pair_axis")
    axes = _axis_array(tuple(map(operator.index, pair_axis)))  # (a copy: what it was given may change)
    if len(axes) != cos.shape[1]:
        raise ValueError(f"pair_axis must name an axis for each of the {cos.shape[1]} pairs that the tables have")
    if not all(0 <= a < positions.shape[0] for a in axes):
        raise ValueError(f"pair_axis names an axis that positions do not have ({positions.shape[0]} axes)")
    return positions.data_ptr(), positions.shape[1], positions.shape[0], axes


def _norm_operands(qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, positions, interleaved, pair_axis=None):
    """What the norm-and-rotation entry points share: (T, D, the device's index, qkv's row distance, and
    the C arguments from q_weight to positions, or to pair_axis)."""
    _torch()
    if pair_axis is not None:
        T, D, dev, row, norm = _norm_operands(qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, None, interleaved)
        return T, D, dev, row, norm[:-1] + _axes_operands(qkv, cos, positions, pair_axis)
    try:
        T, W = qkv.shape
        D, = q_weight.shape
        P, half = cos.shape
        wt = q_weight.dtype
        stride, inner = qkv.stride()
        fine = (qkv.is_cuda and qkv.dtype is _bf16 and inner == 1 and W == (num_heads + 2 * num_kv_heads) * D
                and q_weight.is_cuda and (wt is _bf16 or wt is _f32) and q_weight.is_contiguous()
                and k_weight.is_cuda and k_weight.dtype is wt and k_weight.is_contiguous() and k_weight.shape[0] == D
                and k_weight.dim() == 1 and cos.is_cuda and cos.dtype is _f32 and cos.is_contiguous() and sin.is_cuda
                and sin.dtype is _f32 and sin.is_contiguous() and sin.shape == cos.shape
                and (positions is None or (positions.is_cuda and positions.dtype is _i32 and positions.is_contiguous()
                                           and positions.dim() == 1 and positions.shape[0] == T))
                and (not _several or _together(qkv, q_weight, k_weight, cos, sin, positions)))
    except (AttributeError, ValueError):
        fine = False
    if not fine:
        _norm_checked(qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, positions)
    return T, D, _on_current(qkv, "qkv") if _several else None, stride if T > 1 else W, (
        q_weight.data_ptr(), k_weight.data_ptr(), 1 if wt is _f32 else 0, cos.data_ptr(), sin.data_ptr(), P, 2 * half,
        1 if interleaved else 0, None if positions is None else positions.data_ptr())


def _check_tables(T, seq_len, cos, positions):
    """Without positions, the tables must have a row for each that is implied."""
    if positions is None and T and (seq_len or T) > cos.shape[0]:
        raise ValueError(f"cos and sin have {cos.shape[0]} rows, positions go up to {(seq_len or T) - 1}")


def loom_qkv_norm_rope(qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, positions=None, q=None, k=None, v=None, *,
                       seq_len=0, eps=1e-6, interleaved=False, pair_axis=None, stream=None):
    """RMS norm of each query and key head, the position rotation, and the split of a packed projection.

    qkv [T, (num_heads + 2 num_kv_heads) D] bf16 (its rows may lie further apart); q_weight, k_weight
    [D] bf16 or fp32; cos, sin [positions, rotary_dim / 2] fp32; positions [T] int32 (None: t, or t %
    seq_len).  Writes and returns ``q, k, v`` (allocated if None): [T, H, D], or with ``seq_len``
    [T / seq_len, H, seq_len, D], as the ragged and the dense prefill take them.

    ``pair_axis``, a sequence of rotary_dim / 2 whole numbers: positions are [axes, T] (at most four axes)
    and pair i of a head turns by its token's position on axis pair_axis[i]."""
    _torch()
    if _fast is not None and q is None and k is None and v is None and stream is None:
        r = _fast.norm_rope(qkv, q_weight, k_weight, cos, sin, positions, interleaved, eps, num_heads, num_kv_heads, seq_len,
                            pair_axis)
        if r is not None:
            return _fast_result(r, "loom_qkv_norm_rope")
    num_heads, num_kv_heads, seq_len = int(num_heads), int(num_kv_heads), int(seq_len)
    T, D, dev, row, norm = _norm_operands(qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, positions, interleaved,
                                          pair_axis)
    S = seq_len
    if S < 0 or (S and T % S):
        raise ValueError("T must be a multiple of seq_len")
    _check_tables(T, S, cos, positions)
    if S:
        qs, ks = (T // S, num_heads, S, D), (T // S, num_kv_heads, S, D)
        qst, kst = (num_heads * S * D, S * D, D, 1), (num_kv_heads * S * D, S * D, D, 1)
    else:
        qs, ks, qst, kst = (T, num_heads, D), (T, num_kv_heads, D), (num_heads * D, D, 1), (num_kv_heads * D, D, 1)
    for t, name, shape in ((q, "q", qs), (k, "k", ks), (v, "v", ks)) if q is not None or k is not None or v is not None else ():
        if t is not None and (_dev_ptr(t, name, _bf16, None, dev) is None or tuple(t.shape) != shape):
            raise ValueError(f"{name} must be {list(shape)}")
    new = _maker(qkv, stream)
    if q is None:
        q = new(qs, qst, _bf16)
    if k is None:
        k = new(ks, kst, _bf16)
    if v is None:
        v = new(ks, kst, _bf16)
    lib = _lib or capi()
    st = (lib.loom_qkv_norm_rope if pair_axis is None else lib.loom_qkv_norm_rope_axes)(
        qkv.data_ptr(), row, *norm, q.data_ptr(), k.data_ptr(), v.data_ptr(), T, S, num_heads, num_kv_heads, D, float(eps),
        _stream_of(stream, qkv))
    if st:
        raise LoomError(st, "loom_qkv_norm_rope")
    return q, k, v


def _cache_checked(k_cache, v_cache, positions, slots):
    """The caches and slots of the cache form, named if they are not what they should be."""
    _dev_ptr(k_cache, "k_cache", _bf16, 4), _dev_ptr(v_cache, "v_cache", _bf16, 4)
    if v_cache.shape != k_cache.shape:
        raise ValueError("the caches must have one shape")
    if positions is None or slots is None:
        raise TypeError("positions and slots are needed")
    _dev_ptr(slots, "slots", _i32, 1)


def loom_qkv_norm_rope_cache(qkv, q_weight, k_weight, cos, sin, positions, slots, k_cache, v_cache, num_heads, q=None, *,
                             layout="nhd", eps=1e-6, interleaved=False, pair_axis=None, stream=None):
    """``loom_qkv_norm_rope`` for serving: k and v go to their rows of the caches, q is returned.

    positions and slots [T] int32: token t's row is slots[t] % page_size of page slots[t] //
    page_size (a slot outside the cache, such as -1, is not written).  k_cache, v_cache [num_pages,
    page_size, Hkv, D] (layout "nhd") or [num_pages, Hkv, page_size, D] ("hnd"; also a contiguous
    cache [B, Hkv, capacity, D], whose slots are b * capacity + position).  Returns q [T, num_heads, D].
    ``pair_axis``: positions on several axes, as ``loom_qkv_norm_rope``."""
    if layout not in ("nhd", "hnd"):
        raise ValueError("layout is 'nhd' or 'hnd'")
    _torch()
    if _fast is not None and q is None and stream is None:
        r = _fast.norm_rope_cache(qkv, q_weight, k_weight, cos, sin, positions, interleaved, eps, num_heads, slots, k_cache,
                                  v_cache, layout == "hnd", pair_axis)
        if r is not None:
            return _fast_result(r, "loom_qkv_norm_rope_cache")[0]
    try:
        cs = k_cache.shape
        pages, a, b, Dk = cs
        fine = (k_cache.is_cuda and k_cache.dtype is _bf16 and k_cache.is_contiguous() and v_cache.is_cuda
                and v_cache.dtype is _bf16 and v_cache.is_contiguous() and v_cache.shape == cs and positions is not None
                and slots.is_cuda and slots.dtype is _i32 and slots.is_contiguous() and slots.dim() == 1)
    except (AttributeError, ValueError):
        fine = False
    if not fine:
        _cache_checked(k_cache, v_cache, positions, slots)
    num_heads = int(num_heads)
    page_size, Hkv = (a, b) if layout == "nhd" else (b, a)
    T, D, dev, row, norm = _norm_operands(qkv, q_weight, k_weight, cos, sin, num_heads, Hkv, positions, interleaved, pair_axis)
    if _several and not _together(qkv, k_cache, v_cache, slots):
        for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache"), (slots, "slots")):
            _dev_ptr(t, name, dev=dev)
    if Dk != D or slots.shape[0] != T:
        raise ValueError("the caches must have the weights' D, and slots be [T]")
    if q is None:
        q = _new((T, num_heads, D), (num_heads * D, D, 1), _bf16, qkv, stream=stream)
    elif _dev_ptr(q, "q", _bf16, 3, dev) is None or tuple(q.shape) != (T, num_heads, D):
        raise ValueError(f"q must be {[T, num_heads, D]}")
    lib = _lib or capi()
    st = (lib.loom_qkv_norm_rope_cache if pair_axis is None else lib.loom_qkv_norm_rope_axes_cache)(
        qkv.data_ptr(), row, *norm, slots.data_ptr(), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), pages, page_size,
        0 if layout == "nhd" else 1, T, num_heads, Hkv, D, float(eps), _stream_of(stream, qkv))
    if st:
        raise LoomError(st, "loom_qkv_norm_rope_cache")
    return q


def loom_qkv_norm_rope_bwd_workspace_bytes(D) -> int:
    return int(capi().loom_qkv_norm_rope_bwd_workspace_bytes(D))


def loom_qkv_norm_rope_bwd(dq, dk, dv, qkv, q_weight, k_weight, cos, sin, positions=None, dqkv=None, dq_weight=None,
                           dk_weight=None, workspace=None, *, eps=1e-6, interleaved=False, pair_axis=None, stream=None):
    """Gradients of ``loom_qkv_norm_rope``: dq, dk, dv laid out as it returned q, k, v ([T, H, D] or
    [B, H, seq_len, D]), the rest as the forward call had it.  Writes and returns ``dqkv`` (like qkv;
    its rows may lie further apart), ``dq_weight`` and ``dk_weight`` ([D] fp32), allocated if None.
    ``workspace``: a CUDA uint8 tensor of ``loom_qkv_norm_rope_bwd_workspace_bytes(D)`` bytes."""
    _torch()
    if _fast is not None and dqkv is None and dq_weight is None and dk_weight is None and workspace is None and stream is None:
        r = _fast.norm_rope_bwd(qkv, q_weight, k_weight, cos, sin, positions, interleaved, eps, dq, dk, dv, pair_axis)
        if r is not None:
            return _fast_result(r, "loom_qkv_norm_rope_bwd")
    try:
        qs, ks = dq.shape, dk.shape
        ndim, Hq, Hkv = len(qs), qs[1], ks[1]
        fine = (dq.is_cuda and dq.dtype is _bf16 and dq.is_contiguous() and dk.is_cuda and dk.dtype is _bf16
                and dk.is_contiguous() and dv.is_cuda and dv.dtype is _bf16 and dv.is_contiguous() and dv.shape == ks)
    except (AttributeError, IndexError):
        fine = False
    if not fine:
        dims = 4 if isinstance(dq, _torch_mod.Tensor) and dq.dim() == 4 else 3
        for t, n in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
            _dev_ptr(t, n, _bf16, dims)
    T, D, dev, row, norm = _norm_operands(qkv, q_weight, k_weight, cos, sin, Hq, Hkv, positions, interleaved, pair_axis)
    S = qs[2] if ndim == 4 else 0
    if (not fine or tuple(qs) != ((qs[0], Hq, S, D) if ndim == 4 else (T, Hq, D)) or (qs[0] * S if ndim == 4 else T) != T
            or tuple(ks) != (qs[0], Hkv, *qs[2:])):
        raise ValueError("dq, dk and dv must be laid out as q, k and v of the forward call")
    _check_tables(T, S, cos, positions)
    if _several and not _together(qkv, dq, dk, dv):
        for t, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
            _dev_ptr(t, name, dev=dev)
    width = (Hq + 2 * Hkv) * D
    new = _maker(qkv, stream)
    if dqkv is None:
        dqkv, drow = new((T, width), (width, 1), _bf16), width
    else:
        drow = _row_matrix(dqkv, "dqkv", width, dev)[1]
        if dqkv.shape[0] != T:
            raise ValueError(f"dqkv must be {[T, width]}")
    if dq_weight is None:
        dq_weight = new((D,), (1,), _f32)
    elif _dev_ptr(dq_weight, "dq_weight", _f32, None, dev) is None or tuple(dq_weight.shape) != (D,):
        raise ValueError("dq_weight must be [D]")
    if dk_weight is None:
        dk_weight = new((D,), (1,), _f32)
    elif _dev_ptr(dk_weight, "dk_weight", _f32, None, dev) is None or tuple(dk_weight.shape) != (D,):
        raise ValueError("dk_weight must be [D]")
    if workspace is None:
        wbytes = _norm_bwd_need(D)
        workspace = new((max(wbytes, 16),), (1,), _u8)
        wp = workspace.data_ptr()
    else:
        wp = _dev_ptr(workspace, "workspace", None, None, dev)
        wbytes = workspace.numel() * workspace.element_size()
    lib = _lib or capi()
    st = (lib.loom_qkv_norm_rope_bwd if pair_axis is None else lib.loom_qkv_norm_rope_axes_bwd)(
        dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), qkv.data_ptr(), row, *norm, dqkv.data_ptr(), drow, dq_weight.data_ptr(),
        dk_weight.data_ptr(), wp, wbytes, T, S, Hq, Hkv, D, float(eps), _stream_of(stream, qkv))
    if st:
        raise LoomError(st, "loom_qkv_norm_rope_bwd")
    return dqkv, dq_weight, dk_weight


def loom_attn_check_error(stream=None, device=None):
    """Synchronise and raise ``LoomError`` if a kernel abandoned a bounded wait."""
    st = capi().loom_attn_check_error(_stream_ptr(stream, device))
    _check(st, "loom_attn_check_error")


def loom_status_string(status: int) -> str:
    return capi().loom_status_string(int(status)).decode()


def loom_debug_set_timeout_ns(ns: int):
    capi().loom_debug_set_timeout_ns(int(ns))


def loom_debug_inject(mode: int):
    capi().loom_debug_inject(int(mode))


def loom_debug_prefill_design(design: int):
    capi().loom_debug_prefill_design(int(design))


def loom_model_fwd_plan(D: int) -> dict:
    plan = FwdPlan()
    _check(capi().loom_model_fwd_plan(int(D), ctypes.byref(plan)), "loom_model_fwd_plan")
    return plan.as_dict()


def loom_model_fwd_plan_variant(D: int, design: int):
    """Best plan of one prefill design (1, 2 or 3), or None if the design is infeasible at D."""
    plan = FwdPlan()
    st = capi().loom_model_fwd_plan_variant(int(D), int(design), ctypes.byref(plan))
    if st == 2:  # LOOM_ERR_UNSUPPORTED
        return None
    _check(st, "loom_model_fwd_plan_variant")
    return plan.as_dict()


def loom_model_heg_pipe(l: float, m: float, s: float, b_lm: int, b_ms: int) -> float:
    return float(capi().loom_model_heg_pipe(float(l), float(m), float(s), int(b_lm), int(b_ms)))


def loom_gemm_bf16(a, b, c=None, *, stream=None, b_transposed=False):
    """C = A B (bf16, fp32 accumulation): a [M, K] and b [K, N] bf16 CUDA tensors, or with
    ``b_transposed`` b [N, K] and C = A b^T (a linear layer's weight); writes and returns c
    ([M, N] bf16, allocated if None)."""
    torch = _torch()
    bf16 = torch.bfloat16
    ap = _ptr(a, "a", bf16, 2)
    dev = _on_current(a, "a") if _several else None
    bp = _ptr(b, "b", bf16, 2, dev)
    M, K = a.shape
    if b_transposed:
        N, K2 = b.shape
    else:
        K2, N = b.shape
    if K2 != K:
        raise ValueError(f"a is [M, {K}] but b has {K2} along K")
    if c is None:
        c = _new((M, N), (N, 1), bf16, a, stream=stream)
    cp = _ptr(c, "c", bf16, 2, dev)
    if tuple(c.shape) != (M, N):
        raise ValueError("c must be [M, N]")
    lib = _lib or capi()
    fn = lib.loom_gemm_bf16_bt if b_transposed else lib.loom_gemm_bf16
    _check(fn(ap, bp, cp, M, N, K, _stream_of(stream, a)), "loom_gemm_bf16")
    return c


def loom_gemm_tile_n(M, N, K) -> int:
    return int(capi().loom_gemm_tile_n(M, N, K))


def loom_gemm_splits(M, N, K) -> int:
    return int(capi().loom_gemm_splits(M, N, K))


def loom_model_gemm_time_us(M, N, K, tile_n, splits, num_sms) -> float:
    return float(capi().loom_model_gemm_time_us(M, N, K, tile_n, splits, num_sms))


def loom_debug_gemm_tile_n(tile_n: int):
    capi().loom_debug_gemm_tile_n(int(tile_n))


def loom_debug_gemm_splits(splits: int):
    capi().loom_debug_gemm_splits(int(splits))


def loom_gemm_cta_pair(M, N, K) -> int:
    return int(capi().loom_gemm_cta_pair(M, N, K))


def loom_debug_gemm_cta_pair(mode: int):
    capi().loom_debug_gemm_cta_pair(int(mode))


def loom_model_fwd_time_us_design(design, B, Hq, Sq, Skv, D, causal) -> float:
    """Modeled prefill time (us) with one design forced; negative if the design is infeasible."""
    return float(capi().loom_model_fwd_time_us_design(design, B, Hq, Sq, Skv, D, int(bool(causal))))


def loom_model_fwd_time_us(B, Hq, Sq, Skv, D, causal) -> float:
    return float(capi().loom_model_fwd_time_us(B, Hq, Sq, Skv, D, int(bool(causal))))


def loom_model_decode_time_us(splits, B, Hq, Hkv, Skv, D, num_sms) -> float:
    return float(capi().loom_model_decode_time_us(splits, B, Hq, Hkv, Skv, D, num_sms))


def loom_model_decode_cluster_time_us(splits, cluster, B, Hq, Hkv, Skv, D, clusters) -> float:
    return float(capi().loom_model_decode_cluster_time_us(splits, cluster, B, Hq, Hkv, Skv, D, clusters))


def loom_attn_fwd_cluster(B, Hq, Hkv, Sq, Skv, D, causal=False) -> int:
    """CTAs per cluster that share a work item of ``loom_attn_fwd`` with these sizes (1: none
    do; 0: invalid sizes or no device)."""
    return int(capi().loom_attn_fwd_cluster(B, Hq, Hkv, Sq, Skv, D, int(bool(causal))))


DECODE_SPLIT_MERGE, DECODE_PERSISTENT, DECODE_CLUSTER = 1, 2, 3


def loom_attn_decode_form(B, Hq, Hkv, Skv, D, num_splits=0, paged=False):
    """(form, cluster size) a decode call with these sizes runs: DECODE_SPLIT_MERGE,
    DECODE_PERSISTENT or DECODE_CLUSTER (with its cluster size; 0 otherwise); form -1 on
    invalid sizes."""
    cs = ctypes.c_int(0)
    f = int(capi().loom_attn_decode_form(B, Hq, Hkv, Skv, D, num_splits, int(bool(paged)), ctypes.byref(cs)))
    return f, int(cs.value)


def loom_model_decode_persistent_time_us(splits, B, Hq, Hkv, Skv, D, ctas) -> float:
    return float(capi().loom_model_decode_persistent_time_us(splits, B, Hq, Hkv, Skv, D, ctas))


def loom_model_decode_tc_time_us(splits, B, Hq, Hkv, Skv, D, num_sms) -> float:
    return float(capi().loom_model_decode_tc_time_us(splits, B, Hq, Hkv, Skv, D, num_sms))


def loom_decode_persistent_slots(D, G) -> int:
    return int(capi().loom_decode_persistent_slots(D, G))


def loom_decode_max_clusters(D, G, cluster) -> int:
    return int(capi().loom_decode_max_clusters(D, G, cluster))


def loom_debug_decode_form(form: int, cluster: int = 0) -> None:
    """Pin the Flash Decode form (DECODE_*; 0: the model's) and the cluster size (0: the model's)."""
    capi().loom_debug_decode_form(int(form), int(cluster))


def loom_debug_prefill_slots(D: int, slots: int) -> bool:
    """Pin the two-tile prefill's K/V ring depth (0: the model's); False if not compiled."""
    return bool(capi().loom_debug_prefill_slots(int(D), int(slots)))


def loom_debug_decode_stage_plan(tokens: int, stages: int = 0, ctas_per_sm: int = 0) -> bool:
    """Pin the decode split kernel's stage plan (tokens 0: the model's); False if not compiled."""
    return bool(capi().loom_debug_decode_stage_plan(int(tokens), int(stages), int(ctas_per_sm)))


def loom_debug_gemm_stages(stages: int) -> None:
    """Pin the GEMM's K-stage ring depth where a neighbour is compiled (0: the model's)."""
    capi().loom_debug_gemm_stages(int(stages))


def loom_debug_decode_tensor_cores(mode) -> None:
    """Split kernel of the split + merge decode on a contiguous cache: 1 / True (default)
    tensor cores, persistent; 2 tensor cores, one CTA per split; 0 / False CUDA cores."""
    capi().loom_debug_decode_tensor_cores(int(mode))


def loom_debug_gemm_order(group_rows: int = 0, k_alternate: int = 0) -> None:
    """Pin the GEMM's tile order: tile rows per group (0: the default) and the CTA-pair
    kernel's alternating K direction (-1: off; 0, 1: on)."""
    capi().loom_debug_gemm_order(int(group_rows), int(k_alternate))
