"""Thin ctypes binding over libvfm.so: argument marshalling only.

Every step of the path runs in the HIP kernels of the library; this module
turns torch tensors (device memory) and host int32 arrays into the pointers and
sizes the C ABI takes (include/vfm.h).  There is no fallback: if the library
is not built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import types
from typing import Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# VFM_LIB may point at another build of the library (same C ABI).
LIB_PATH = os.environ.get("VFM_LIB") or os.path.join(_HERE, "libvfm.so")

VFM_BF16 = 0
VFM_F32 = 1
VFM_MAX_SEQS = 256

EXPORTS = ("vfm_rope3d", "vfm_qknorm_rope3d", "vfm_qknorm_rope3d_bwd", "vfm_attn_fwd", "vfm_attn_bwd_workspace_size", "vfm_attn_bwd", "vfm_attn_bwd_noalloc", "vfm_xattn_fwd", "vfm_xattn_bwd_workspace_size", "vfm_xattn_bwd", "vfm_tattn_fwd", "vfm_tattn_bwd",
           "vfm_fp8_pack_sizes", "vfm_fp8_pack", "vfm_attn_fwd_fp8", "vfm_strerror", "vfm_last_hip_error", "vfm_schedule_units",
           "vfm_attn_fwd_tile_rows", "vfm_cattn_fwd_workspace_size", "vfm_cattn_fwd", "vfm_cattn_bwd_workspace_size", "vfm_cattn_bwd",
           "vfm_kv4_append", "vfm_kv4_gather", "vfm_kv4_attn_workspace_size", "vfm_kv4_attn")

_lib = None
_calls = None                # the library's functions as the wrappers call them (load_library)
_torch = None                # both set when the library is loaded


class VfmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libvfm status {status}: {message}")
        self.status = status


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """dlopen libvfm.so and declare the C signatures.  Raises if it is missing."""
    global _lib, _calls, _torch
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it first (python -m paper_2503_12964_amd.build); "
            "there is no CPU fallback")
    # The library and PyTorch must share ONE HIP runtime: the tensors and streams handed over
    # belong to PyTorch's.  libvfm.so asks for the runtime by its soname; with PyTorch (which
    # ships its own copy under that soname) loaded first, the dynamic linker gives the library
    # that copy.  Loaded the other way round, the library would bring in the system's copy as a
    # second runtime in the process, and a second runtime finds no device.
    import torch
    _torch = torch
    lib = ctypes.CDLL(path)
    c_int, c_float, c_void_p, c_size_t = ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
    p_i32 = ctypes.POINTER(ctypes.c_int32)
    lib.vfm_rope3d.restype = c_int
    lib.vfm_rope3d.argtypes = [c_void_p, p_i32, p_i32, c_int, c_int, c_int, c_int, c_int, c_int, c_int,
                               c_float, c_int, c_int, c_void_p]
    lib.vfm_qknorm_rope3d.restype = c_int
    lib.vfm_qknorm_rope3d.argtypes = [c_void_p, c_void_p, c_float, c_void_p, p_i32, p_i32, c_int, c_int, c_int,
                                      c_int, c_int, c_int, c_int, c_float, c_int, c_void_p]
    lib.vfm_qknorm_rope3d_bwd.restype = c_int
    lib.vfm_qknorm_rope3d_bwd.argtypes = [c_void_p, c_void_p, c_float, c_void_p, c_void_p, c_void_p, p_i32, p_i32,
                                          c_int, c_int, c_int, c_int, c_int, c_int, c_int, c_float, c_int,
                                          c_void_p]
    lib.vfm_attn_fwd.restype = c_int
    lib.vfm_attn_fwd.argtypes = [c_void_p, c_void_p, c_void_p, p_i32, c_int, c_int, c_int, c_int, c_float,
                                 c_void_p, c_void_p, c_int, c_void_p]
    lib.vfm_attn_bwd_workspace_size.restype = c_size_t
    lib.vfm_attn_bwd_workspace_size.argtypes = [c_int, c_int, c_int]
    lib.vfm_attn_bwd.restype = c_int
    lib.vfm_attn_bwd.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, p_i32, c_int,
                                 c_int, c_int, c_int, c_float, c_void_p, c_void_p, c_void_p, c_void_p,
                                 c_size_t, c_int, c_void_p]
    lib.vfm_attn_bwd_noalloc.restype = c_int
    lib.vfm_attn_bwd_noalloc.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, p_i32, c_int,
                                         c_int, c_int, c_int, c_float, c_void_p, c_void_p, c_void_p, c_int,
                                         c_void_p]
    lib.vfm_xattn_fwd.restype = c_int
    lib.vfm_xattn_fwd.argtypes = [c_void_p, c_void_p, c_void_p, p_i32, p_i32, c_int, c_int, c_int, c_int, c_int,
                                  c_float, c_void_p, c_void_p, c_int, c_void_p]
    lib.vfm_xattn_bwd_workspace_size.restype = c_size_t
    lib.vfm_xattn_bwd_workspace_size.argtypes = [c_int, c_int, c_int, c_int]
    lib.vfm_xattn_bwd.restype = c_int
    lib.vfm_xattn_bwd.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, p_i32, p_i32, c_int,
                                  c_int, c_int, c_int, c_int, c_float, c_void_p, c_void_p, c_void_p, c_void_p,
                                  c_size_t, c_int, c_void_p]
    lib.vfm_tattn_fwd.restype = c_int
    lib.vfm_tattn_fwd.argtypes = [c_void_p, c_void_p, c_void_p, p_i32, p_i32, c_int, c_int, c_int, c_int, c_float,
                                  c_void_p, c_int, c_void_p]
    lib.vfm_tattn_bwd.restype = c_int
    lib.vfm_tattn_bwd.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, p_i32, p_i32, c_int, c_int, c_int, c_int,
                                  c_float, c_void_p, c_void_p, c_void_p, c_int, c_void_p]
    p_size = ctypes.POINTER(c_size_t)
    lib.vfm_fp8_pack_sizes.restype = c_int
    lib.vfm_fp8_pack_sizes.argtypes = [p_i32, c_int, c_int, c_int, c_int, p_size, p_size, p_size, p_size]
    lib.vfm_fp8_pack.restype = c_int
    lib.vfm_fp8_pack.argtypes = [c_void_p, c_void_p, c_void_p, p_i32, c_int, c_int, c_int, c_int, c_float,
                                 c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_void_p]
    lib.vfm_attn_fwd_fp8.restype = c_int
    lib.vfm_attn_fwd_fp8.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, p_i32, c_int, c_int, c_int, c_int,
                                     c_void_p, c_void_p, c_void_p]
    lib.vfm_strerror.restype = ctypes.c_char_p
    lib.vfm_strerror.argtypes = [c_int]
    lib.vfm_schedule_units.restype = c_int
    lib.vfm_schedule_units.argtypes = [p_i32, c_int, c_int, c_int, c_int, p_i32, c_int, ctypes.POINTER(c_int)]
    lib.vfm_attn_fwd_tile_rows.restype = c_int
    lib.vfm_attn_fwd_tile_rows.argtypes = [p_i32, c_int, c_int, c_int, c_int, ctypes.POINTER(c_int)]
    lib.vfm_last_hip_error.restype = ctypes.c_char_p
    lib.vfm_last_hip_error.argtypes = []
    c_i64 = ctypes.c_int64
    causal_sizes = [p_i32, p_i32, c_int, c_int, c_int, c_int, c_int, c_int]
    rows3 = [c_void_p, c_i64, c_void_p, c_i64, c_void_p, c_i64]          # three tensors with their token strides
    lib.vfm_cattn_fwd_workspace_size.restype = c_size_t
    lib.vfm_cattn_fwd_workspace_size.argtypes = causal_sizes
    lib.vfm_cattn_fwd.restype = c_int
    lib.vfm_cattn_fwd.argtypes = [*rows3, *causal_sizes, c_float, c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_void_p]
    lib.vfm_cattn_bwd_workspace_size.restype = c_size_t
    lib.vfm_cattn_bwd_workspace_size.argtypes = causal_sizes
    lib.vfm_cattn_bwd.restype = c_int
    lib.vfm_cattn_bwd.argtypes = [*rows3, c_void_p, c_void_p, c_void_p, *causal_sizes, c_float, *rows3, c_void_p, c_size_t,
                                  c_int, c_void_p]
    cache = [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int]       # k4, v4, k_scales, v_scales, n_pages, page_size
    lib.vfm_kv4_append.restype = c_int
    lib.vfm_kv4_append.argtypes = [c_void_p, c_i64, c_void_p, c_i64, p_i32, c_int, c_int, c_void_p, c_void_p, c_int, *cache,
                                   c_int, c_int, c_int, c_void_p]
    lib.vfm_kv4_gather.restype = c_int
    lib.vfm_kv4_gather.argtypes = [*cache, c_void_p, c_int, p_i32, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_int, c_void_p]
    lib.vfm_kv4_attn_workspace_size.restype = c_size_t
    lib.vfm_kv4_attn_workspace_size.argtypes = [p_i32, c_int, c_int, c_int, c_int, c_int]
    lib.vfm_kv4_attn.restype = c_int
    lib.vfm_kv4_attn.argtypes = [c_void_p, c_i64, *cache, c_void_p, c_int, c_void_p, p_i32, c_int, c_int, c_int, c_int, c_int,
                                 c_float, c_void_p, c_void_p, c_void_p, c_size_t, c_int, c_void_p]
    # The same functions taking a host int32 array as the address of its first element (a plain int, which the
    # wrappers below pass: see _host_i32); the library's own keep refusing anything but an int32 array or pointer.
    lib.by_address = types.SimpleNamespace()
    for name in EXPORTS:
        typed, fn = getattr(lib, name), lib[name]
        fn.restype, fn.argtypes = typed.restype, [c_void_p if t is p_i32 else t for t in typed.argtypes]
        setattr(lib.by_address, name, fn)
    if path == LIB_PATH:
        _lib, _calls = lib, lib.by_address
    return lib


def strerror(status: int) -> str:
    return load_library().vfm_strerror(int(status)).decode()


def vfm_last_hip_error() -> str:
    return load_library().vfm_last_hip_error().decode()


VFM_ERR_LAUNCH = 8


def _check(status: int) -> None:
    if status != 0:
        text = strerror(status)
        if status == VFM_ERR_LAUNCH:
            text += " (" + vfm_last_hip_error() + ")"
        raise VfmError(status, text)


def vfm_schedule_units(cu_seqlens, n_heads: int, rows_per_tile: int) -> np.ndarray:
    """(head, first packed row, rows) of every workgroup of a launch that cuts rows_per_tile-row
    tiles from the clips; head -1 marks grid padding.  Host only."""
    lib = load_library().by_address
    cu = _host_i32(cu_seqlens)
    n = ctypes.c_int(0)
    st = lib.vfm_schedule_units(_i32_ptr(cu), int(cu.size - 1), int(cu[-1]), int(n_heads), int(rows_per_tile),
                                None, 0, ctypes.byref(n))
    if st not in (0, 2):          # SHAPE only says "capacity too small" here
        _check(st)
    units = np.zeros((max(n.value, 1), 3), dtype=np.int32)
    _check(lib.vfm_schedule_units(_i32_ptr(cu), int(cu.size - 1), int(cu[-1]), int(n_heads), int(rows_per_tile),
                                  _i32_ptr(units), int(units.shape[0]), ctypes.byref(n)))
    return units[:n.value]


def vfm_attn_fwd_tile_rows(cu_seqlens, head_dim: int, run: int = 0) -> int:
    """Query rows per workgroup the forward uses for run `run` of these clips.  Host only."""
    lib = load_library().by_address
    cu = _host_i32(cu_seqlens)
    rows = ctypes.c_int(0)
    _check(lib.vfm_attn_fwd_tile_rows(_i32_ptr(cu), int(cu.size - 1), int(cu[-1]), int(head_dim), int(run),
                                      ctypes.byref(rows)))
    return rows.value


# What a call costs here is what bounds the smallest steps: the argument handling of one call took 7 to 9 us beside the
# 4 to 5 us of the native call and its launch (current_stream() alone 2.6 us, a ctypes pointer to an array 1.2), now 2 to 4.
_I32 = np.dtype(np.int32)


def _host_i32(a) -> np.ndarray:
    if type(a) is np.ndarray and a.dtype is _I32 and a.ndim and a.flags.c_contiguous:
        return a
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _i32_ptr(a: np.ndarray) -> int:
    """Address of the first element; the caller keeps the array alive over the native call."""
    return a.__array_interface__["data"][0]


def _stream_ptr(stream) -> int:
    if stream is None:
        try:
            c = _torch._C
            return c._cuda_getCurrentRawStream(c._cuda_getDevice())
        except AttributeError:      # another PyTorch: the public way, slower
            stream = _torch.cuda.current_stream()
    return int(getattr(stream, "cuda_stream", stream))


def _dev(t, name: str) -> int:
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    return t.data_ptr()


def _dtype_code(t) -> int:
    dt = t.dtype
    if dt is _torch.bfloat16:
        return VFM_BF16
    if dt is _torch.float32:
        return VFM_F32
    raise ValueError(f"unsupported dtype {dt}")


def vfm_rope3d(x, thw, cu_seqlens, dims: Sequence[int], theta: float = 10000.0,
               inverse: bool = False, stream=None):
    """In-place 3D RoPE on x[total, heads, head_dim] (device, bf16).  Returns x."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    g = _host_i32(thw).reshape(-1)
    total, heads, hd = x.shape
    _check(lib.vfm_rope3d(_dev(x, "x"), _i32_ptr(g), _i32_ptr(cu), int(cu.size - 1), int(total), int(heads),
                          int(hd), int(dims[0]), int(dims[1]), int(dims[2]), float(theta), int(bool(inverse)),
                          _dtype_code(x), _stream_ptr(stream)))
    return x


def vfm_qknorm_rope3d(x, gain, eps: float, thw, cu_seqlens, dims: Sequence[int], theta: float = 10000.0,
                      y=None, stream=None):
    """y = RoPE3D(gain * x / sqrt(mean_d x^2 + eps)) per (token, head); y=None works in place on x."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    g = _host_i32(thw).reshape(-1)
    total, heads, hd = x.shape
    y = x if y is None else y
    _check(lib.vfm_qknorm_rope3d(_dev(x, "x"), _dev(gain, "gain"), float(eps), _dev(y, "y"), _i32_ptr(g),
                                 _i32_ptr(cu), cu.size - 1, total, heads, hd,
                                 int(dims[0]), int(dims[1]), int(dims[2]), float(theta), _dtype_code(x),
                                 _stream_ptr(stream)))
    return y


def vfm_qknorm_rope3d_bwd(x, gain, eps: float, dy, thw, cu_seqlens, dims: Sequence[int],
                          theta: float = 10000.0, dx=None, dgain=None, stream=None) -> Tuple:
    """dx (bf16, shape of x; may be dy itself) and dgain (fp32 [head_dim]) given the forward's input x."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    g = _host_i32(thw).reshape(-1)
    total, heads, hd = x.shape
    dx = _torch.empty_like(x) if dx is None else dx
    dgain = _torch.empty(hd, dtype=_torch.float32, device=x.device) if dgain is None else dgain
    _check(lib.vfm_qknorm_rope3d_bwd(_dev(x, "x"), _dev(gain, "gain"), float(eps), _dev(dy, "dy"), _dev(dx, "dx"),
                                     _dev(dgain, "dgain"), _i32_ptr(g), _i32_ptr(cu), int(cu.size - 1),
                                     int(total), int(heads), int(hd), int(dims[0]), int(dims[1]), int(dims[2]),
                                     float(theta), _dtype_code(x), _stream_ptr(stream)))
    return dx, dgain


def vfm_attn_fwd(q, k, v, cu_seqlens, scale: float, out=None, lse=None, stream=None) -> Tuple:
    """out[total, heads, head_dim] (bf16) and lse[heads, total] (fp32) for packed q, k, v."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    total, heads, hd = q.shape
    if out is None:
        out = _torch.empty_like(q)
    if lse is None:
        lse = _torch.empty((heads, total), dtype=_torch.float32, device=q.device)
    _check(lib.vfm_attn_fwd(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _i32_ptr(cu), int(cu.size - 1), int(total),
                            int(heads), int(hd), float(scale), _dev(out, "out"), _dev(lse, "lse"),
                            _dtype_code(q), _stream_ptr(stream)))
    return out, lse


def vfm_attn_bwd_workspace_size(total_tokens: int, n_heads: int, head_dim: int) -> int:
    return int(load_library().vfm_attn_bwd_workspace_size(int(total_tokens), int(n_heads), int(head_dim)))


def vfm_attn_bwd(q, k, v, out, lse, dout, cu_seqlens, scale: float, dq=None, dk=None, dv=None,
                 workspace=None, stream=None) -> Tuple:
    """dq, dk, dv (bf16, shape of q) given the forward's out and lse."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    total, heads, hd = q.shape
    dq = _torch.empty_like(q) if dq is None else dq
    dk = _torch.empty_like(k) if dk is None else dk
    dv = _torch.empty_like(v) if dv is None else dv
    if workspace is None:
        need = vfm_attn_bwd_workspace_size(total, heads, hd)
        workspace = _torch.empty(max(need, 256), dtype=_torch.uint8, device=q.device)
    _check(lib.vfm_attn_bwd(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"), _dev(lse, "lse"),
                            _dev(dout, "dout"), _i32_ptr(cu), cu.size - 1, total, heads, hd,
                            float(scale), _dev(dq, "dq"), _dev(dk, "dk"), _dev(dv, "dv"),
                            _dev(workspace, "workspace"), int(workspace.numel() * workspace.element_size()),
                            _dtype_code(q), _stream_ptr(stream)))
    return dq, dk, dv


def vfm_attn_bwd_noalloc(q, k, v, out, lse, dout, cu_seqlens, scale: float, dq, dk, dv, stream=None) -> Tuple:
    """vfm_attn_bwd without a workspace (the library's built-in scratch holds the statistics).
    The caller passes every output; nothing is allocated here or in the library."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    total, heads, hd = q.shape
    _check(lib.vfm_attn_bwd_noalloc(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"), _dev(lse, "lse"),
                                    _dev(dout, "dout"), _i32_ptr(cu), int(cu.size - 1), int(total), int(heads),
                                    int(hd), float(scale), _dev(dq, "dq"), _dev(dk, "dk"), _dev(dv, "dv"),
                                    _dtype_code(q), _stream_ptr(stream)))
    return dq, dk, dv


def vfm_xattn_fwd(q, k, v, cu_seqlens_q, cu_seqlens_kv, scale: float, out=None, lse=None, stream=None) -> Tuple:
    """Cross-attention: out[total_q, heads, head_dim] (bf16), lse[heads, total_q] (fp32)."""
    lib = _calls or load_library().by_address
    cq, ck = _host_i32(cu_seqlens_q), _host_i32(cu_seqlens_kv)
    if cq.size != ck.size:
        raise ValueError("cu_seqlens_q and cu_seqlens_kv must have the same length")
    total_q, heads, hd = q.shape
    if out is None:
        out = _torch.empty_like(q)
    if lse is None:
        lse = _torch.empty((heads, total_q), dtype=_torch.float32, device=q.device)
    _check(lib.vfm_xattn_fwd(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _i32_ptr(cq), _i32_ptr(ck), cq.size - 1,
                             int(total_q), int(k.shape[0]), int(heads), int(hd), float(scale), _dev(out, "out"),
                             _dev(lse, "lse"), _dtype_code(q), _stream_ptr(stream)))
    return out, lse


def vfm_xattn_bwd_workspace_size(total_q: int, total_kv: int, n_heads: int, head_dim: int) -> int:
    return int(load_library().vfm_xattn_bwd_workspace_size(int(total_q), int(total_kv), int(n_heads), int(head_dim)))


def vfm_xattn_bwd(q, k, v, out, lse, dout, cu_seqlens_q, cu_seqlens_kv, scale: float, dq=None, dk=None,
                  dv=None, workspace=None, stream=None) -> Tuple:
    """Cross-attention gradients: dq (shape of q), dk, dv (shape of k)."""
    lib = _calls or load_library().by_address
    cq, ck = _host_i32(cu_seqlens_q), _host_i32(cu_seqlens_kv)
    if cq.size != ck.size:
        raise ValueError("cu_seqlens_q and cu_seqlens_kv must have the same length")
    total_q, heads, hd = q.shape
    dq = _torch.empty_like(q) if dq is None else dq
    dk = _torch.empty_like(k) if dk is None else dk
    dv = _torch.empty_like(v) if dv is None else dv
    if workspace is None:
        need = vfm_xattn_bwd_workspace_size(total_q, int(k.shape[0]), heads, hd)
        workspace = _torch.empty(max(need, 256), dtype=_torch.uint8, device=q.device)
    _check(lib.vfm_xattn_bwd(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(out, "out"), _dev(lse, "lse"),
                             _dev(dout, "dout"), _i32_ptr(cq), _i32_ptr(ck), cq.size - 1, int(total_q),
                             int(k.shape[0]), int(heads), int(hd), float(scale), _dev(dq, "dq"), _dev(dk, "dk"),
                             _dev(dv, "dv"), _dev(workspace, "workspace"),
                             int(workspace.numel() * workspace.element_size()), _dtype_code(q),
                             _stream_ptr(stream)))
    return dq, dk, dv


def vfm_tattn_fwd(q, k, v, thw, cu_seqlens, scale: float, out=None, stream=None):
    """Temporal attention (one sequence per pixel across a clip's frames): out, shape of q."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    g = _host_i32(thw).reshape(-1)
    total, heads, hd = q.shape
    out = _torch.empty_like(q) if out is None else out
    _check(lib.vfm_tattn_fwd(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _i32_ptr(g), _i32_ptr(cu), int(cu.size - 1),
                             int(total), int(heads), int(hd), float(scale), _dev(out, "out"), _dtype_code(q),
                             _stream_ptr(stream)))
    return out


def vfm_tattn_bwd(q, k, v, dout, thw, cu_seqlens, scale: float, dq=None, dk=None, dv=None, stream=None) -> Tuple:
    """Temporal attention gradients dq, dk, dv (shape of q)."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    g = _host_i32(thw).reshape(-1)
    total, heads, hd = q.shape
    dq = _torch.empty_like(q) if dq is None else dq
    dk = _torch.empty_like(k) if dk is None else dk
    dv = _torch.empty_like(v) if dv is None else dv
    _check(lib.vfm_tattn_bwd(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _dev(dout, "dout"), _i32_ptr(g), _i32_ptr(cu),
                             cu.size - 1, total, heads, hd, float(scale), _dev(dq, "dq"),
                             _dev(dk, "dk"), _dev(dv, "dv"), _dtype_code(q), _stream_ptr(stream)))
    return dq, dk, dv


def vfm_fp8_pack_sizes(cu_seqlens, n_heads: int, head_dim: int) -> Tuple[int, int, int, int]:
    """Bytes of the packed q8, k8, vT8 and scales buffers for these clips."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    a, b, c, d = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib.vfm_fp8_pack_sizes(_i32_ptr(cu), int(cu.size - 1), int(cu[-1]), int(n_heads), int(head_dim),
                                  ctypes.byref(a), ctypes.byref(b), ctypes.byref(c), ctypes.byref(d)))
    return int(a.value), int(b.value), int(c.value), int(d.value)


def vfm_fp8_pack(q, k, v, cu_seqlens, scale: float, q8=None, k8=None, vT8=None, scales=None, stream=None) -> Tuple:
    """Quantise bf16 q, k, v to E4M3 tiles with power-of-two scales, in the packed layout
    vfm_attn_fwd_fp8 reads (uint8 device buffers q8, k8, vT8 and the scales buffer).  q also
    carries scale * log2(e) (scale = softmax scale)."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    total, heads, hd = q.shape
    nq, nk, nv, ns = vfm_fp8_pack_sizes(cu, heads, hd)
    q8 = _torch.empty(max(nq, 16), dtype=_torch.uint8, device=q.device) if q8 is None else q8
    k8 = _torch.empty(max(nk, 16), dtype=_torch.uint8, device=q.device) if k8 is None else k8
    vT8 = _torch.empty(max(nv, 16), dtype=_torch.uint8, device=q.device) if vT8 is None else vT8
    scales = _torch.empty(max(ns, 16), dtype=_torch.uint8, device=q.device) if scales is None else scales
    _check(lib.vfm_fp8_pack(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _i32_ptr(cu), int(cu.size - 1), int(total),
                            int(heads), int(hd), float(scale), _dev(q8, "q8"), _dev(k8, "k8"), _dev(vT8, "vT8"),
                            _dev(scales, "scales"), _dtype_code(q), _stream_ptr(stream)))
    return q8, k8, vT8, scales


def vfm_attn_fwd_fp8(q8, k8, vT8, scales, cu_seqlens, n_heads: int, head_dim: int, out=None, lse=None,
                     stream=None) -> Tuple:
    """FP8 attention forward on packed operands: out (bf16 [total, heads, head_dim]) and lse (fp32)."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    total = int(cu[-1])
    if out is None:
        out = _torch.empty((total, n_heads, head_dim), dtype=_torch.bfloat16, device=q8.device)
    if lse is None:
        lse = _torch.empty((n_heads, total), dtype=_torch.float32, device=q8.device)
    _check(lib.vfm_attn_fwd_fp8(_dev(q8, "q8"), _dev(k8, "k8"), _dev(vT8, "vT8"), _dev(scales, "scales"), _i32_ptr(cu),
                                int(cu.size - 1), total, int(n_heads), int(head_dim), _dev(out, "out"),
                                _dev(lse, "lse"), _stream_ptr(stream)))
    return out, lse


# ---- causal attention with grouped heads, 4-bit key/value cache
# What a call costs here bounds the smallest steps (a token of one sequence: 11 us on the GPU), so each argument is looked at once:
# its device (which also tells a host tensor), type, shape and order, and what a wrapper allocates itself is not looked at.
def _current_device() -> int:
    try:
        return _torch._C._cuda_getDevice()
    except AttributeError:      # another PyTorch
        return _torch.cuda.current_device()


def _elsewhere(t, name: str, here: int):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    raise ValueError(f"{name} lives on {t.device}, the current device is cuda:{here}")


def _rows(t, name: str, here: int, shape):
    """Address and token stride of a bf16 tensor of this shape, [tokens, heads, head_dim], whose tokens may lie apart."""
    if t.get_device() != here:
        _elsewhere(t, name, here)
    if t.dtype is not _torch.bfloat16 or t.shape != shape:
        raise ValueError(f"{name} must be bfloat16 of shape {tuple(shape)}, not {t.dtype} of {tuple(t.shape)}")
    n, heads, hd = shape
    if t.is_contiguous():
        return t.data_ptr(), heads * hd
    row, head, elem = t.stride()
    if (elem != 1 and hd > 1) or (head != hd and heads > 1):
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    return t.data_ptr(), row if n > 1 else heads * hd


def _like(t, name: str, here: int, shape, dtype) -> int:
    """Address of a contiguous tensor of exactly this shape and type."""
    if t.get_device() != here:
        _elsewhere(t, name, here)
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, {dtype} of shape {tuple(shape)}, not {t.dtype} of {tuple(t.shape)}")
    return t.data_ptr()


def _new(shape, dtype, like, stream, result=True):
    """A tensor for the kernels of this call, from the memory of the stream that they run on: what the current stream has freed may
    still be in use by work in front of it.  A result lives on until the current stream, where the caller goes on, is done with it too."""
    here = s = None
    if stream is not None:
        here = _torch.cuda.current_stream()
        s = stream if hasattr(stream, "cuda_stream") else _torch.cuda.ExternalStream(int(stream))
    if s is None or s.cuda_stream == here.cuda_stream:
        if like.dtype is dtype and like.shape == shape and like.is_contiguous():
            return _torch.empty_like(like)          # (a third less than the general call)
        return _torch.empty(shape, dtype=dtype, device=like.device)
    with _torch.cuda.stream(s):
        t = _torch.empty(shape, dtype=dtype, device=like.device)
    if result and t.numel():
        t.record_stream(here)
    return t


def _out_lse(q, shape, out, lse, here: int, stream):
    """out and lse of a forward, and their addresses."""
    total, heads, _ = shape
    if out is None:
        out = _new(shape, _torch.bfloat16, q, stream)
        po = out.data_ptr()
    else:
        po = _like(out, "out", here, shape, _torch.bfloat16)
    if lse is None:
        lse = _new((heads, total), _torch.float32, q, stream)
        return out, lse, po, lse.data_ptr()
    return out, lse, po, _like(lse, "lse", here, (heads, total), _torch.float32)


def _workspace(given, size, sizes, like, here: int, stream):
    """The workspace (kept by the caller of this), its address and size: the one given, or one of size(*sizes) bytes."""
    if given is None:
        need = size(*sizes)
        if not need:
            return None, 0, 0
        given = _new(need, _torch.uint8, like, stream, result=False)
        return given, given.data_ptr(), need
    if given.get_device() != here or not given.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor of the current device")
    return given, given.data_ptr(), given.numel() * given.element_size()


def _causal_cu(cu_seqlens_q, cu_seqlens_kv):
    cq, ck = _host_i32(cu_seqlens_q), _host_i32(cu_seqlens_kv)
    if cq.size != ck.size or cq.size < 1:
        raise ValueError("cu_seqlens_q and cu_seqlens_kv must have the same length")
    return cq, ck


def _causal_sizes(q, k, cu_seqlens_q, cu_seqlens_kv):
    cq, ck = _causal_cu(cu_seqlens_q, cu_seqlens_kv)
    sq, sk = q.shape, k.shape
    if len(sq) != 3 or len(sk) != 3 or sk[2] != sq[2]:
        raise ValueError("q [total_q, heads, head_dim], k and v [total_kv, kv_heads, head_dim] expected")
    pq = _i32_ptr(cq)
    return cq, ck, sq, sk, (pq, pq if ck is cq else _i32_ptr(ck), cq.size - 1, sq[0], sk[0], sq[1], sk[1], sq[2])


def vfm_cattn_fwd_workspace_size(cu_seqlens_q, cu_seqlens_kv, n_heads: int, n_kv_heads: int, head_dim: int) -> int:
    lib = _calls or load_library().by_address
    cq, ck = _causal_cu(cu_seqlens_q, cu_seqlens_kv)
    return int(lib.vfm_cattn_fwd_workspace_size(_i32_ptr(cq), _i32_ptr(ck), cq.size - 1, int(cq[-1]), int(ck[-1]), int(n_heads),
                                                int(n_kv_heads), int(head_dim)))


def vfm_cattn_fwd(q, k, v, cu_seqlens_q, cu_seqlens_kv, scale: float, out=None, lse=None, workspace=None, stream=None) -> Tuple:
    """Causal attention with grouped heads: out[total_q, heads, head_dim] (bf16), lse[heads, total_q] (fp32).  k, v:
    [total_kv, kv_heads, head_dim]; the last query of a sequence sees its last key.  q, k, v may be parts of one
    tensor (tokens apart, a token's heads contiguous)."""
    lib = _calls or load_library().by_address
    cq, ck, sq, sk, sizes = _causal_sizes(q, k, cu_seqlens_q, cu_seqlens_kv)
    here = _current_device()
    rows = (*_rows(q, "q", here, sq), *_rows(k, "k", here, sk), *_rows(v, "v", here, sk))
    out, lse, po, pl = _out_lse(q, sq, out, lse, here, stream)
    workspace, pw, nw = _workspace(workspace, lib.vfm_cattn_fwd_workspace_size, sizes, q, here, stream)
    _check(lib.vfm_cattn_fwd(*rows, *sizes, scale, po, pl, pw, nw, VFM_BF16, _stream_ptr(stream)))
    return out, lse


def vfm_cattn_bwd_workspace_size(cu_seqlens_q, cu_seqlens_kv, n_heads: int, n_kv_heads: int, head_dim: int) -> int:
    lib = _calls or load_library().by_address
    cq, ck = _causal_cu(cu_seqlens_q, cu_seqlens_kv)
    return int(lib.vfm_cattn_bwd_workspace_size(_i32_ptr(cq), _i32_ptr(ck), cq.size - 1, int(cq[-1]), int(ck[-1]), int(n_heads),
                                                int(n_kv_heads), int(head_dim)))


def vfm_cattn_bwd(q, k, v, out, lse, dout, cu_seqlens_q, cu_seqlens_kv, scale: float, dq=None, dk=None, dv=None,
                  workspace=None, stream=None) -> Tuple:
    """Gradients of vfm_cattn_fwd: dq (shape of q), dk, dv (shape of k), bf16; given ones may be parts of one tensor."""
    lib = _calls or load_library().by_address
    cq, ck, sq, sk, sizes = _causal_sizes(q, k, cu_seqlens_q, cu_seqlens_kv)
    here, bf16 = _current_device(), _torch.bfloat16
    rows = (*_rows(q, "q", here, sq), *_rows(k, "k", here, sk), *_rows(v, "v", here, sk))
    given = (_like(out, "out", here, sq, bf16), _like(lse, "lse", here, (sq[1], sq[0]), _torch.float32), _like(dout, "dout", here, sq, bf16))
    if dq is None:
        dq = _new(sq, bf16, q, stream)
    if dk is None:
        dk = _new(sk, bf16, k, stream)
    if dv is None:
        dv = _new(sk, bf16, v, stream)
    grads = (*_rows(dq, "dq", here, sq), *_rows(dk, "dk", here, sk), *_rows(dv, "dv", here, sk))
    workspace, pw, nw = _workspace(workspace, lib.vfm_cattn_bwd_workspace_size, sizes, q, here, stream)
    _check(lib.vfm_cattn_bwd(*rows, *given, *sizes, scale, *grads, pw, nw, VFM_BF16, _stream_ptr(stream)))
    return dq, dk, dv


def _kv4_cache(k4, v4, k_scales, v_scales, here: int):
    """Addresses and sizes of a cache: (k4, v4, k_scales, v_scales, n_pages, page_size), kv_heads, head_dim."""
    shape, u8 = k4.shape, _torch.uint8
    if len(shape) != 4:
        raise ValueError("k4 must be [n_pages, kv_heads, page_size, head_dim / 2]")
    n_pages, kvh, page, half = shape
    blocks = (n_pages, kvh, page, half // 16)
    return (_like(k4, "k4", here, shape, u8), _like(v4, "v4", here, shape, u8), _like(k_scales, "k_scales", here, blocks, u8),
            _like(v_scales, "v_scales", here, blocks, u8), n_pages, page), kvh, 2 * half


def _kv4_pages(pages, here: int, n_seqs: int):
    shape = pages.shape
    if len(shape) != 2:
        raise ValueError("pages must be [n_seqs, max_pages]")
    return _like(pages, "pages", here, (n_seqs, shape[1]), _torch.int32), shape[1]


def vfm_kv4_append(k, v, k4, v4, k_scales, v_scales, pages, lens, cu_seqlens, stream=None) -> None:
    """Quantises k, v [total, kv_heads, head_dim] (bf16, tokens may lie apart) into the paged 4-bit cache at the places
    lens[s], lens[s] + 1, ... of their sequences.  pages [n_seqs, max_pages] and lens [n_seqs]: int32 on the device."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    n, here = cu.size - 1, _current_device()
    cache, kvh, hd = _kv4_cache(k4, v4, k_scales, v_scales, here)
    table, max_pages = _kv4_pages(pages, here, n)
    total = k.shape[0]
    rows = (total, kvh, hd)
    _check(lib.vfm_kv4_append(*_rows(k, "k", here, rows), *_rows(v, "v", here, rows), _i32_ptr(cu), n, total,
                              _like(lens, "lens", here, (n,), _torch.int32), table, max_pages, *cache, kvh, hd, VFM_BF16, _stream_ptr(stream)))


def vfm_kv4_gather(k4, v4, k_scales, v_scales, pages, cu_seqlens, k=None, v=None, stream=None) -> Tuple:
    """The first cu_seqlens[s+1] - cu_seqlens[s] places of every sequence as bf16 k, v [total, kv_heads, head_dim]."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    n, here, bf16 = cu.size - 1, _current_device(), _torch.bfloat16
    cache, kvh, hd = _kv4_cache(k4, v4, k_scales, v_scales, here)
    table, max_pages = _kv4_pages(pages, here, n)
    total = int(cu[n])
    rows = (total, kvh, hd)
    if k is None:
        k = _new(rows, bf16, k4, stream)
    if v is None:
        v = _new(rows, bf16, k4, stream)
    _check(lib.vfm_kv4_gather(*cache, table, max_pages, _i32_ptr(cu), n, total, kvh, hd, _like(k, "k", here, rows, bf16),
                              _like(v, "v", here, rows, bf16), VFM_BF16, _stream_ptr(stream)))
    return k, v


def vfm_kv4_attn_workspace_size(cu_seqlens, n_heads: int, n_kv_heads: int, head_dim: int) -> int:
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    return int(lib.vfm_kv4_attn_workspace_size(_i32_ptr(cu), cu.size - 1, int(cu[-1]), int(n_heads), int(n_kv_heads), int(head_dim)))


def vfm_kv4_attn(q, k4, v4, k_scales, v_scales, pages, lens, cu_seqlens, scale: float, out=None, lse=None, workspace=None,
                 stream=None) -> Tuple:
    """Attention of the new tokens q [total, heads, head_dim] (bf16, tokens may lie apart) over the 4-bit cache, which holds
    their own keys and values already: token t of sequence s sees the places 0 .. lens[s] + t.  Returns out (bf16) and
    lse [heads, total] (fp32)."""
    lib = _calls or load_library().by_address
    cu = _host_i32(cu_seqlens)
    n, here = cu.size - 1, _current_device()
    cache, kvh, hd = _kv4_cache(k4, v4, k_scales, v_scales, here)
    table, max_pages = _kv4_pages(pages, here, n)
    shape = q.shape
    if len(shape) != 3 or shape[2] != hd:
        raise ValueError(f"q must be [total, heads, {hd}]")
    total, heads, _ = shape
    pq = _rows(q, "q", here, shape)
    pn = _like(lens, "lens", here, (n,), _torch.int32)
    cu_p = _i32_ptr(cu)
    out, lse, po, pl = _out_lse(q, shape, out, lse, here, stream)
    workspace, pw, nw = _workspace(workspace, lib.vfm_kv4_attn_workspace_size, (cu_p, n, total, heads, kvh, hd), q, here, stream)
    _check(lib.vfm_kv4_attn(*pq, *cache, table, max_pages, pn, cu_p, n, total, heads, kvh, hd, scale, po, pl, pw, nw, VFM_BF16,
                            _stream_ptr(stream)))
    return out, lse
