"""ctypes bindings with the same names as the C ABI in ``include/startrail.h``.

Argument marshalling only: tensors are torch tensors on the GPU ([B, S, heads, D] with D
contiguous, fp32 or bf16), outputs are allocated with torch when not supplied, and every
call is enqueued on torch's current stream.  A non-zero status raises StarTrailError.

The calls that a training step makes many times try the native half first (``csrc/st_binding.cpp``),
which reads plain tensors, lists and numbers in a tenth of the time; what it does not take (it then
answers None, and has called nothing) goes through ctypes below, which also raises the errors.
Without it, or with another torch or Python than it was built for, everything goes through ctypes.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
import sys
import warnings
from typing import List, NamedTuple, Optional, Sequence, Tuple

import torch

ST_F32, ST_BF16, ST_E4M3 = 0, 1, 2
ST_RING_STEPWISE, ST_RING_FUSED = 0, 1
ST_KV_ASSIGN = 1
ST_GRAD_ASSIGN = 1
ST_ROPE_HALVES, ST_ROPE_NEIGHBOURS, ST_ROPE_MAX_AXES = 0, 1, 4
ST_MAX_CHUNKS = 256

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libstartrail.so")


class StarTrailError(RuntimeError):
    def __init__(self, status: int, where: str, text: str):
        super().__init__(f"{where}: status {status} ({text})")
        self.status = status


class st_tensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("stride_b", C.c_int64), ("stride_s", C.c_int64), ("stride_h", C.c_int64)]


class st_block_desc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("Sq", C.c_int32), ("Sk", C.c_int32), ("q_offset", C.c_int64), ("k_offset", C.c_int64),
                ("causal", C.c_int32), ("scale", C.c_float), ("q_seg", C.c_int32), ("q_offset2", C.c_int64)]


class st_ring_desc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("Sq", C.c_int32), ("Sk", C.c_int32), ("q_offset", C.c_int64), ("causal", C.c_int32),
                ("scale", C.c_float), ("n_chunks", C.c_int32),
                ("k_ptr", C.POINTER(C.c_void_p)), ("v_ptr", C.POINTER(C.c_void_p)),
                ("k_stride_b", C.c_int64), ("k_stride_s", C.c_int64), ("k_stride_h", C.c_int64),
                ("v_stride_b", C.c_int64), ("v_stride_s", C.c_int64), ("v_stride_h", C.c_int64),
                ("k_offset", C.POINTER(C.c_int64)), ("q_seg", C.c_int32), ("q_offset2", C.c_int64)]


class st_score(C.Structure):
    _fields_ = [("softcap", C.c_float), ("slopes", C.c_void_p), ("spans", C.c_void_p)]


class st_rope_desc(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("B", C.c_int32), ("S", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("rot", C.c_int32), ("pairing", C.c_int32), ("norm", C.c_int32), ("eps", C.c_float), ("n_axes", C.c_int32),
                ("axis_pairs", C.c_int32 * 4), ("offset", C.c_int64), ("seg", C.c_int32), ("offset2", C.c_int64)]


class st_cache(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_pages", C.c_int32), ("page", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("B", C.c_int32),
                ("width", C.c_int32), ("k", st_tensor), ("v", st_tensor), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("table", C.c_void_p), ("lens", C.c_void_p)]


class st_cache_rows(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("T", C.c_int32), ("Hq", C.c_int32), ("max_rows", C.c_int32), ("causal", C.c_int32),
                ("window", C.c_int32), ("scale", C.c_float), ("softcap", C.c_float), ("slopes", C.c_void_p)]


class st_comm_report(C.Structure):
    _fields_ = [("ring_iterations", C.c_int32), ("startrail_iterations", C.c_int32),
                ("ring_p2p_bytes_per_iter", C.c_int64), ("startrail_p2p_bytes_per_iter", C.c_int64),
                ("ring_p2p_bytes", C.c_int64), ("startrail_p2p_bytes", C.c_int64),
                ("startrail_collective_bytes", C.c_int64), ("ring_p2p_seconds", C.c_double),
                ("startrail_p2p_seconds", C.c_double), ("startrail_collective_seconds", C.c_double)]


class st_device_report(C.Structure):
    _fields_ = [("name", C.c_char * 64), ("arch", C.c_char * 32), ("compute_units", C.c_int32), ("xcds", C.c_int32),
                ("max_clock_mhz", C.c_int32), ("memory_clock_mhz", C.c_int32), ("memory_bus_bits", C.c_int32),
                ("hbm_bytes", C.c_int64)]


class st_profile_entry(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("launches", C.c_int32), ("total_ms", C.c_float)]


def library_path() -> str:
    return _LIB_PATH


def _load() -> C.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python paper_2407_00611_amd/build.py` "
                          "(there is no CPU fallback)")
    lib = C.CDLL(_LIB_PATH)
    T, D, R = C.POINTER(st_tensor), C.POINTER(st_block_desc), C.POINTER(st_ring_desc)
    M, P = C.POINTER(st_score), C.POINTER(st_rope_desc)
    K, W = C.POINTER(st_cache), C.POINTER(st_cache_rows)
    vp, f32p, i32p = C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)
    sigs = {
        "st_attn_block_fwd": (C.c_int, [D, T, T, T, f32p, f32p, vp]),
        "st_attn_merge": (C.c_int, [f32p, f32p, f32p, f32p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp, vp]),
        "st_attn_combine": (C.c_int, [C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_int32, C.c_int32, C.c_int32,
                                      C.c_int32, C.c_int32, C.c_int32, C.c_int32, f32p, f32p, C.c_int32, vp, vp]),
        "st_attn_delta": (C.c_int, [D, T, T, C.c_int32, f32p, vp]),
        "st_attn_block_bwd": (C.c_int, [D, T, T, T, T, f32p, f32p, f32p, f32p, f32p, vp, C.c_size_t, vp]),
        "st_attn_block_bwd_workspace_bytes": (C.c_size_t, [D]),
        "st_cast_from_f32": (C.c_int, [f32p, vp, C.c_int64, C.c_int32, vp]),
        "st_visit_order": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, i32p, i32p]),
        "st_team_visit_order": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, i32p]),
        "st_schedule_report": (C.c_int, [C.c_int32, C.c_int32, C.c_int64, C.c_int64, C.c_int64, C.c_int32,
                                         C.c_double, C.c_double, C.POINTER(st_comm_report)]),
        "st_ring_workspace_bytes": (C.c_size_t, [R, C.c_int32, C.c_int32]),
        "st_ring_fwd": (C.c_int, [R, T, i32p, i32p, C.c_int32, C.c_int32, f32p, f32p, vp, vp, C.c_size_t, vp]),
        "st_ring_bwd": (C.c_int, [R, T, T, T, C.c_int32, f32p, i32p, C.c_int32, C.c_int32, f32p,
                                  C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), vp, C.c_size_t, vp]),
        "st_ring_bwd_noalloc": (C.c_int, [R, T, T, T, C.c_int32, f32p, i32p, C.c_int32, C.c_int32, f32p,
                                          C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), vp]),
        "st_ring_bwd_noalloc_max_bytes": (C.c_size_t, []),
        "st_ring_bwd_last": (C.c_int, [R, T, T, T, C.c_int32, f32p, i32p, C.c_int32, C.c_int32, f32p,
                                       C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_int32,
                                       C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), vp, C.c_size_t, vp]),
        "st_mask_spans": (C.c_int, [C.c_int32, C.c_int32, C.c_int64, C.c_int32, C.c_int64, C.c_int32, vp, C.c_int32, vp, vp, vp]),
        "st_attn_score_workspace_bytes": (C.c_size_t, [D, M, C.c_int32]),
        "st_attn_score_fwd": (C.c_int, [D, M, T, T, T, f32p, f32p, vp, vp, C.c_size_t, vp]),
        "st_attn_score_bwd": (C.c_int, [D, M, T, T, T, T, f32p, f32p, C.c_int32, f32p, f32p, f32p, vp, vp, vp, vp, C.c_size_t, vp]),
        "st_qk_rope_fwd": (C.c_int, [P, T, T, f32p, f32p, vp, vp, T, T, vp]),
        "st_qk_rope_bwd_workspace_bytes": (C.c_size_t, [P]),
        "st_qk_rope_bwd": (C.c_int, [P, T, T, T, T, C.c_int32, f32p, f32p, vp, vp, C.c_int32, T, T, f32p, f32p, vp, C.c_size_t, vp]),
        "st_cache_append": (C.c_int, [P, K, vp, T, T, T, f32p, f32p, vp, vp, T, vp]),
        "st_cache_read": (C.c_int, [K, vp, C.c_int32, C.c_int32, T, T, vp]),
        "st_attn_cache_workspace_bytes": (C.c_size_t, [W, K]),
        "st_attn_cache": (C.c_int, [W, K, vp, vp, T, f32p, f32p, vp, vp, C.c_size_t, vp]),
        "st_device_facts": (C.c_int, [C.POINTER(st_device_report)]),
        "st_mfma_probe": (C.c_int, [vp, C.c_int64, C.c_int32, C.c_int32, f32p, C.c_int64, C.POINTER(C.c_double), vp]),
        "st_mfma_probe_mixes": (C.c_int32, []),
        "st_mfma_probe_mix_name": (C.c_char_p, [C.c_int32]),
        "st_profile_begin": (C.c_int, []),
        "st_profile_end": (C.c_int, [C.POINTER(st_profile_entry), C.c_int32, C.POINTER(C.c_int32)]),
        "st_status_str": (C.c_char_p, [C.c_int]),
        "st_last_error": (C.c_char_p, []),
        "st_version": (C.c_int32, []),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


_lib = _load()


class _Declines:
    """In the place of a native half that is not there or not for this process: leaves every call to ctypes."""
    built_for = None

    def __getattr__(self, name):
        return lambda *args: None


def _native_half():
    """csrc/st_binding.cpp, linked against the library that has just been loaded.  It reads torch's and Python's objects as their
    headers laid them out, so it is taken only where it was built for this torch and this Python."""
    try:
        from . import _binding
    except ImportError as e:
        warnings.warn(f"calls are marshalled by ctypes, at several times the host time: {e}", RuntimeWarning)
        return _Declines()
    here = f"torch {torch.__version__}, Python {sys.version_info.major}.{sys.version_info.minor}"
    if _binding.built_for != here:
        warnings.warn(f"calls are marshalled by ctypes, at several times the host time: the native half was built for {_binding.built_for}, "
                      f"this is {here}", RuntimeWarning)
        return _Declines()
    return _binding


_binding = _native_half()

EXPORTS = ["st_attn_block_fwd", "st_attn_merge", "st_attn_combine", "st_attn_delta", "st_attn_block_bwd", "st_attn_block_bwd_workspace_bytes", "st_cast_from_f32",
           "st_visit_order", "st_team_visit_order", "st_schedule_report", "st_ring_workspace_bytes", "st_ring_fwd", "st_ring_bwd", "st_ring_bwd_noalloc", "st_ring_bwd_noalloc_max_bytes", "st_ring_bwd_last", "st_mask_spans", "st_attn_score_workspace_bytes", "st_attn_score_fwd", "st_attn_score_bwd", "st_qk_rope_fwd",
           "st_qk_rope_bwd_workspace_bytes", "st_qk_rope_bwd", "st_cache_append", "st_cache_read", "st_attn_cache_workspace_bytes", "st_attn_cache", "st_device_facts", "st_mfma_probe", "st_mfma_probe_mixes", "st_mfma_probe_mix_name", "st_profile_begin",
           "st_profile_end", "st_status_str",
           "st_last_error", "st_version"]


def _check(status: int, where: str) -> None:
    if status != 0:
        raise StarTrailError(status, where, f"{_lib.st_status_str(status).decode()}: {_lib.st_last_error().decode()}")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return ST_F32
    if t.dtype == torch.bfloat16:
        return ST_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _torch_dtype(code: int):
    return torch.float32 if code == ST_F32 else torch.bfloat16


def _view(t: torch.Tensor) -> st_tensor:
    stride = t.stride()
    if len(stride) != 4:
        raise ValueError("expected a [B, S, heads, D] tensor")
    if stride[3] != 1 and t.shape[3] > 1:
        raise ValueError("the D dimension must be contiguous")
    return st_tensor(t.data_ptr() if t.numel() else None, stride[0], stride[1], stride[2])


def _stream(stream) -> C.c_void_p:
    if stream is None:
        if torch.cuda.is_initialized():          # the handle alone, without a Stream object around it
            return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()))
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _raw_stream(stream):
    """The stream's handle as a number, or None where only _stream knows how to get it."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if torch.cuda.is_initialized() else None
    return getattr(stream, "cuda_stream", None)


def _done(status: Optional[int], where: str) -> bool:
    """Whether the native half has made the call (its status is checked)."""
    if status:
        _check(status, where)
    return status is not None


def _ptr(t: Optional[torch.Tensor]) -> C.c_void_p:
    return C.c_void_p(t.data_ptr() if t is not None and t.numel() else None)


def _aligned(buf: torch.Tensor, a: int) -> Tuple[int, int]:
    """First a-byte aligned address inside a byte buffer and the bytes from there to its end."""
    ptr = (buf.data_ptr() + a - 1) // a * a
    return ptr, max(buf.numel() * buf.element_size() - (ptr - buf.data_ptr()), 0)      # (the buffer may end before the boundary)


def _f32_dense(t: torch.Tensor, shape, name: str) -> torch.Tensor:
    if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 tensor of shape {tuple(shape)}")
    return t


_INT32, _INT64 = 1 << 31, 1 << 63


def _fit(end: int, *xs: int) -> None:
    """ctypes cuts off what does not fit a field of the structs or an argument."""
    for x in xs:
        if not -end <= x < end:
            raise ValueError(f"{x} does not fit {end.bit_length()} bits")


def _q_runs(q_offset) -> Tuple[int, int, int]:
    """q_offset is the position of query row 0, or (position of row 0, rows in the first run, position of the
    first row of the second run) for a shard made of two runs of the sequence."""
    if isinstance(q_offset, (tuple, list)):
        off, seg, off2 = q_offset
        off, seg, off2 = int(off), int(seg), int(off2)
        _fit(_INT64, off, off2)
        _fit(_INT32, seg)
        return off, seg, off2
    off = int(q_offset)
    _fit(_INT64, off)
    return off, 0, 0


def _block_desc(q, k, q_offset, k_offset, causal, scale) -> st_block_desc:
    B, Sq, Hq, D = q.shape
    _, Sk, Hkv, _ = k.shape
    off, seg, off2 = _q_runs(q_offset)
    k_off = int(k_offset)
    _fit(_INT32, max(B, Sq, Hq, D, Sk, Hkv))
    _fit(_INT64, k_off)
    return st_block_desc(_dtype_code(q), B, Hq, Hkv, D, Sq, Sk, off, k_off,
                         1 if causal else 0, float(scale), seg, off2)


def st_version() -> int:
    return int(_lib.st_version())


def st_status_str(status: int) -> str:
    return _lib.st_status_str(int(status)).decode()


def st_last_error() -> str:
    return _lib.st_last_error().decode()


def st_device_facts() -> dict:
    r = st_device_report()
    _check(_lib.st_device_facts(C.byref(r)), "st_device_facts")
    return {"name": r.name.decode(), "arch": r.arch.decode(), "compute_units": int(r.compute_units), "xcds": int(r.xcds),
            "max_clock_mhz": int(r.max_clock_mhz), "memory_clock_mhz": int(r.memory_clock_mhz),
            "memory_bus_bits": int(r.memory_bus_bits), "hbm_bytes": int(r.hbm_bytes)}


def st_mfma_probe(operands: torch.Tensor, iters: int, sink: torch.Tensor, mix: int = 0, stream=None) -> float:
    """Enqueues the MFMA loop `mix` (0: MFMAs only) on `operands` (any contiguous tensor, read as bf16 bits);
    returns the flop its MFMAs execute."""
    if not operands.is_contiguous() or sink.dtype != torch.float32 or not sink.is_contiguous():
        raise ValueError("operands must be contiguous, sink contiguous fp32")
    flop = C.c_double(0.0)
    _check(_lib.st_mfma_probe(_ptr(operands), operands.numel() * operands.element_size(), int(mix), int(iters), _ptr(sink),
                              sink.numel(), C.byref(flop), _stream(stream)), "st_mfma_probe")
    return float(flop.value)


def st_mfma_probe_mixes() -> int:
    return int(_lib.st_mfma_probe_mixes())


def st_mfma_probe_mix_name(mix: int) -> str:
    return _lib.st_mfma_probe_mix_name(int(mix)).decode()


def st_profile_begin() -> None:
    _check(_lib.st_profile_begin(), "st_profile_begin")


def st_profile_end() -> dict:
    """{kernel name: (launches, total_ms)} of everything launched since st_profile_begin()."""
    buf = (st_profile_entry * 32)()
    n = C.c_int32(0)
    _check(_lib.st_profile_end(buf, 32, C.byref(n)), "st_profile_end")
    return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms)) for i in range(n.value)}


def st_attn_block_fwd(q, k, v, q_offset: int, k_offset: int, causal: bool, scale: float,
                      o_part=None, lse_part=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    if o_part is not None and lse_part is not None and \
            _done(_binding.block_fwd(q, k, v, q_offset, k_offset, causal, scale, o_part, lse_part, _raw_stream(stream)), "st_attn_block_fwd"):
        return o_part, lse_part
    B, Sq, Hq, D = q.shape
    o_part = torch.empty((B, Sq, Hq, D), dtype=torch.float32, device=q.device) if o_part is None else \
        _f32_dense(o_part, (B, Sq, Hq, D), "o_part")
    lse_part = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device) if lse_part is None else \
        _f32_dense(lse_part, (B, Hq, Sq), "lse_part")
    d = _block_desc(q, k, q_offset, k_offset, causal, scale)
    tq, tk, tv = _view(q), _view(k), _view(v)
    _check(_lib.st_attn_block_fwd(C.byref(d), C.byref(tq), C.byref(tk), C.byref(tv), _ptr(o_part), _ptr(lse_part),
                                  _stream(stream)), "st_attn_block_fwd")
    return o_part, lse_part


def st_attn_merge(o_acc, lse_acc, o_part, lse_part, out_dtype: int = ST_F32, o_out_lowp=None, stream=None) -> None:
    if _done(_binding.merge(o_acc, lse_acc, o_part, lse_part, out_dtype, o_out_lowp, _raw_stream(stream)), "st_attn_merge"):
        return
    B, Sq, Hq, D = o_acc.shape
    _f32_dense(o_acc, (B, Sq, Hq, D), "o_acc"); _f32_dense(o_part, (B, Sq, Hq, D), "o_part")
    _f32_dense(lse_acc, (B, Hq, Sq), "lse_acc"); _f32_dense(lse_part, (B, Hq, Sq), "lse_part")
    if o_out_lowp is not None and (tuple(o_out_lowp.shape) != (B, Sq, Hq, D) or not o_out_lowp.is_contiguous()
                                   or o_out_lowp.dtype != _torch_dtype(out_dtype)):
        raise ValueError("o_out_lowp must be dense [B,Sq,Hq,D] in out_dtype")
    _check(_lib.st_attn_merge(_ptr(o_acc), _ptr(lse_acc), _ptr(o_part), _ptr(lse_part), B, Sq, Hq, D, out_dtype,
                              _ptr(o_out_lowp), _stream(stream)), "st_attn_merge")


def st_attn_combine(o_parts, lse_parts, row0: int = 0, Sq_out: int = None, out_dtype: int = ST_F32, o_out=None,
                    lse_out=None, o_out_lowp=None, stream=None):
    """n partial states of the same rows -> (o_out, lse_out) of rows [row0, row0 + Sq_out)."""
    if o_out is not None and lse_out is not None and \
            _done(_binding.combine(o_parts, lse_parts, row0, Sq_out, out_dtype, o_out, lse_out, o_out_lowp, _raw_stream(stream)), "st_attn_combine"):
        return o_out, lse_out
    n = len(o_parts)
    if n == 0 or len(lse_parts) != n:
        raise ValueError("need as many lse_parts as o_parts, at least one")
    B, Sq_in, Hq, D = o_parts[0].shape
    Sq_out = Sq_in - row0 if Sq_out is None else Sq_out
    for x in range(n):
        _f32_dense(o_parts[x], (B, Sq_in, Hq, D), "o_parts[x]")
        _f32_dense(lse_parts[x], (B, Hq, Sq_in), "lse_parts[x]")
    dev = o_parts[0].device
    o_out = torch.empty((B, Sq_out, Hq, D), dtype=torch.float32, device=dev) if o_out is None else \
        _f32_dense(o_out, (B, Sq_out, Hq, D), "o_out")
    lse_out = torch.empty((B, Hq, Sq_out), dtype=torch.float32, device=dev) if lse_out is None else \
        _f32_dense(lse_out, (B, Hq, Sq_out), "lse_out")
    if o_out_lowp is not None and (tuple(o_out_lowp.shape) != (B, Sq_out, Hq, D) or not o_out_lowp.is_contiguous()
                                   or o_out_lowp.dtype != _torch_dtype(out_dtype)):
        raise ValueError("o_out_lowp must be dense [B,Sq_out,Hq,D] in out_dtype")
    op = (C.c_void_p * n)(*[_ptr(t) for t in o_parts])
    lp = (C.c_void_p * n)(*[_ptr(t) for t in lse_parts])
    _check(_lib.st_attn_combine(op, lp, n, B, Sq_in, Hq, D, int(row0), int(Sq_out), _ptr(o_out), _ptr(lse_out), out_dtype,
                                _ptr(o_out_lowp), _stream(stream)), "st_attn_combine")
    return o_out, lse_out


def st_attn_delta(d_o, o, delta=None, stream=None) -> torch.Tensor:
    B, Sq, Hq, D = d_o.shape
    if delta is None and stream is None and d_o.is_cuda:
        delta = torch.empty((B, Hq, Sq), dtype=torch.float32, device=d_o.device)
    if delta is not None and _done(_binding.delta(d_o, o, delta, _raw_stream(stream)), "st_attn_delta"):
        return delta
    delta = torch.empty((B, Hq, Sq), dtype=torch.float32, device=d_o.device) if delta is None else \
        _f32_dense(delta, (B, Hq, Sq), "delta")
    d = st_block_desc(_dtype_code(d_o), B, Hq, Hq, D, Sq, 0, 0, 0, 0, 1.0)
    td, to = _view(d_o), _view(o)
    _check(_lib.st_attn_delta(C.byref(d), C.byref(td), C.byref(to), _dtype_code(o), _ptr(delta), _stream(stream)),
           "st_attn_delta")
    return delta


def st_attn_block_bwd_workspace_bytes(q, k, q_offset: int, k_offset: int, causal: bool, scale: float) -> int:
    d = _block_desc(q, k, q_offset, k_offset, causal, scale)
    return int(_lib.st_attn_block_bwd_workspace_bytes(C.byref(d)))


def st_attn_block_bwd(q, k, v, d_o, lse_final, delta, q_offset: int, k_offset: int, causal: bool, scale: float,
                      dq_acc, dk_acc, dv_acc, stream=None, workspace=None) -> None:
    """workspace: a uint8 tensor of st_attn_block_bwd_workspace_bytes(...) bytes, None to have one allocated, or
    False to pass none (the C call then keeps the dK/dV work in its general kernel)."""
    if workspace is not None and workspace is not False and \
            _done(_binding.block_bwd(q, k, v, d_o, lse_final, delta, q_offset, k_offset, causal, scale, dq_acc, dk_acc, dv_acc, workspace,
                                     _raw_stream(stream)), "st_attn_block_bwd"):
        return
    B, Sq, Hq, D = q.shape
    Sk, Hkv = k.shape[1], k.shape[2]
    _f32_dense(lse_final, (B, Hq, Sq), "lse_final"); _f32_dense(delta, (B, Hq, Sq), "delta")
    _f32_dense(dq_acc, (B, Sq, Hq, D), "dq_acc")
    _f32_dense(dk_acc, (B, Sk, Hkv, D), "dk_acc"); _f32_dense(dv_acc, (B, Sk, Hkv, D), "dv_acc")
    d = _block_desc(q, k, q_offset, k_offset, causal, scale)
    tq, tk, tv, td = _view(q), _view(k), _view(v), _view(d_o)
    if workspace is None:
        need = int(_lib.st_attn_block_bwd_workspace_bytes(C.byref(d)))
        if need > 0:
            workspace = torch.empty(need + 256, dtype=torch.uint8, device=q.device)
    ws_ptr, ws_bytes = (None, 0) if workspace is None or workspace is False else _aligned(workspace, 256)
    _check(_lib.st_attn_block_bwd(C.byref(d), C.byref(tq), C.byref(tk), C.byref(tv), C.byref(td), _ptr(lse_final),
                                  _ptr(delta), _ptr(dq_acc), _ptr(dk_acc), _ptr(dv_acc), C.c_void_p(ws_ptr), ws_bytes,
                                  _stream(stream)),
           "st_attn_block_bwd")


def st_cast_from_f32(src, dst_dtype: int, dst=None, stream=None) -> torch.Tensor:
    if dst is not None and _done(_binding.cast(src, dst, dst_dtype, _raw_stream(stream)), "st_cast_from_f32"):
        return dst
    if src.dtype != torch.float32 or not src.is_contiguous():
        raise ValueError("src must be contiguous fp32")
    dst = torch.empty(src.shape, dtype=_torch_dtype(dst_dtype), device=src.device) if dst is None else dst
    if not dst.is_contiguous() or dst.numel() != src.numel() or dst.dtype != _torch_dtype(dst_dtype):
        raise ValueError("dst must be contiguous, of dst_dtype and as large as src")
    _check(_lib.st_cast_from_f32(_ptr(src), _ptr(dst), src.numel(), dst_dtype, _stream(stream)), "st_cast_from_f32")
    return dst


def st_team_visit_order(P: int, Cteam: int, rank: int) -> List[int]:
    out = (C.c_int32 * max(int(P), 1))()              # the library validates the layout; P entries always suffice
    _check(_lib.st_team_visit_order(int(P), int(Cteam), int(rank), out), "st_team_visit_order")
    return list(out)[:int(P) // (int(Cteam) * int(Cteam))]


def st_schedule_report(P: int, Cteam: int, B: int, N: int, H: int, bytes_per_element: int = 2,
                       W: float = 1.0, L: float = 0.0) -> dict:
    out = st_comm_report()
    _check(_lib.st_schedule_report(int(P), int(Cteam), int(B), int(N), int(H), int(bytes_per_element), float(W), float(L),
                                   C.byref(out)), "st_schedule_report")
    return {name: getattr(out, name) for name, _ in st_comm_report._fields_}


def st_visit_order(P: int, Cteam: int, rank: int) -> Tuple[List[int], List[int]]:
    n = max(int(P), 1)
    shard = (C.c_int32 * n)()
    member = (C.c_int32 * n)()
    _check(_lib.st_visit_order(int(P), int(Cteam), int(rank), shard, member), "st_visit_order")
    return list(shard), list(member)


class _Ring:
    """Keeps the host-side tables of an st_ring_desc alive for the duration of a call."""

    def __init__(self, q, k_chunks: Sequence[torch.Tensor], v_chunks: Sequence[torch.Tensor], q_offset: int,
                 k_offsets: Sequence[int], causal: bool, scale: float):
        n = len(k_chunks)
        if n < 1 or len(v_chunks) != n or len(k_offsets) != n:
            raise ValueError("need one K, one V and one offset per chunk")
        B, Sq, Hq, D = q.shape
        k0, v0 = k_chunks[0], v_chunks[0]
        shape, k_stride, v_stride, dtype = k0.shape, k0.stride(), v0.stride(), q.dtype
        for k, v in zip(k_chunks, v_chunks):
            if k.shape != shape or v.shape != shape or k.stride() != k_stride or v.stride() != v_stride \
                    or k.dtype != dtype or v.dtype != dtype:
                raise ValueError("all chunks must share shape, strides and dtype")
            if k is k0:
                _view(k), _view(v)                # the others have the shape and the strides of these
        self.k_ptr = (C.c_void_p * n)(*[k.data_ptr() for k in k_chunks])
        self.v_ptr = (C.c_void_p * n)(*[v.data_ptr() for v in v_chunks])
        self.k_off = (C.c_int64 * n)(*[int(x) for x in k_offsets])
        off, seg, off2 = _q_runs(q_offset)
        self.desc = st_ring_desc(_dtype_code(q), B, Hq, shape[2], D, Sq, shape[1], off, 1 if causal else 0, float(scale), n,
                                 self.k_ptr, self.v_ptr, k_stride[0], k_stride[1], k_stride[2], v_stride[0], v_stride[1],
                                 v_stride[2], self.k_off, seg, off2)


def st_ring_workspace_bytes(q, k_chunks, v_chunks, q_offset, k_offsets, causal, scale, mode: int,
                            backward: bool) -> int:
    r = _Ring(q, k_chunks, v_chunks, q_offset, k_offsets, causal, scale)
    return int(_lib.st_ring_workspace_bytes(C.byref(r.desc), mode, 1 if backward else 0))


def _i32_array(xs: Optional[Sequence[int]]):
    if xs is None:
        return None
    return (C.c_int32 * max(len(xs), 1))(*[int(x) for x in xs])


def st_ring_fwd(q, k_chunks, v_chunks, q_offset: int, k_offsets: Sequence[int], causal: bool, scale: float,
                order: Sequence[int], member_of: Optional[Sequence[int]] = None, mode: int = ST_RING_FUSED,
                o_acc=None, lse=None, o_lowp=None, want_lowp: bool = True, workspace=None, stream=None):
    """Returns (o_acc fp32, lse fp32, o_lowp or None)."""
    if o_acc is not None and lse is not None and workspace is not None and (o_lowp is not None or not want_lowp) and \
            _done(_binding.ring_fwd(q, k_chunks, v_chunks, q_offset, k_offsets, causal, scale, order, member_of, mode, o_acc, lse, o_lowp,
                                    workspace, _raw_stream(stream)), "st_ring_fwd"):
        return o_acc, lse, o_lowp
    B, Sq, Hq, D = q.shape
    r = _Ring(q, k_chunks, v_chunks, q_offset, k_offsets, causal, scale)
    o_acc = torch.empty((B, Sq, Hq, D), dtype=torch.float32, device=q.device) if o_acc is None else \
        _f32_dense(o_acc, (B, Sq, Hq, D), "o_acc")
    lse = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device) if lse is None else \
        _f32_dense(lse, (B, Hq, Sq), "lse")
    if o_lowp is None and want_lowp:
        o_lowp = torch.empty((B, Sq, Hq, D), dtype=q.dtype, device=q.device)
    if workspace is None:
        need = int(_lib.st_ring_workspace_bytes(C.byref(r.desc), mode, 0))
        workspace = torch.empty(need + 256, dtype=torch.uint8, device=q.device)
    ws_ptr = (workspace.data_ptr() + 255) // 256 * 256
    ws_bytes = workspace.numel() * workspace.element_size() - (ws_ptr - workspace.data_ptr())
    tq = _view(q)
    _check(_lib.st_ring_fwd(C.byref(r.desc), C.byref(tq), _i32_array(order), _i32_array(member_of), len(order), mode,
                            _ptr(o_acc), _ptr(lse), _ptr(o_lowp), C.c_void_p(ws_ptr), ws_bytes, _stream(stream)),
           "st_ring_fwd")
    return o_acc, lse, o_lowp


def st_ring_bwd(q, k_chunks, v_chunks, d_o, o, lse_final, q_offset: int, k_offsets: Sequence[int], causal: bool,
                scale: float, order: Sequence[int], dq_acc, dk_acc: Sequence[Optional[torch.Tensor]],
                dv_acc: Sequence[Optional[torch.Tensor]], mode: int = ST_RING_FUSED, workspace=None,
                stream=None) -> None:
    if workspace is not None and \
            _done(_binding.ring_bwd(q, k_chunks, v_chunks, d_o, o, lse_final, q_offset, k_offsets, causal, scale, order, dq_acc, dk_acc,
                                    dv_acc, False, None, None, mode, workspace, _raw_stream(stream)), "st_ring_bwd"):
        return
    B, Sq, Hq, D = q.shape
    r = _Ring(q, k_chunks, v_chunks, q_offset, k_offsets, causal, scale)
    n = len(k_chunks)
    _f32_dense(dq_acc, (B, Sq, Hq, D), "dq_acc"); _f32_dense(lse_final, (B, Hq, Sq), "lse_final")
    kv_shape = tuple(k_chunks[0].shape)
    for t in list(dk_acc) + list(dv_acc):
        if t is not None:
            _f32_dense(t, kv_shape, "dk_acc/dv_acc entry")
    dk_ptr = (C.c_void_p * n)(*[(t.data_ptr() if t is not None else None) for t in dk_acc])
    dv_ptr = (C.c_void_p * n)(*[(t.data_ptr() if t is not None else None) for t in dv_acc])
    if workspace is None:
        need = int(_lib.st_ring_workspace_bytes(C.byref(r.desc), mode, 1))
        workspace = torch.empty(need + 256, dtype=torch.uint8, device=q.device)
    ws_ptr = (workspace.data_ptr() + 255) // 256 * 256
    ws_bytes = workspace.numel() * workspace.element_size() - (ws_ptr - workspace.data_ptr())
    tq, td, to = _view(q), _view(d_o), _view(o)
    _check(_lib.st_ring_bwd(C.byref(r.desc), C.byref(tq), C.byref(td), C.byref(to), _dtype_code(o), _ptr(lse_final),
                            _i32_array(order), len(order), mode, _ptr(dq_acc),
                            dk_ptr, dv_ptr,
                            C.c_void_p(ws_ptr), ws_bytes, _stream(stream)), "st_ring_bwd")


def st_ring_bwd_noalloc_max_bytes() -> int:
    return int(_lib.st_ring_bwd_noalloc_max_bytes())


def st_ring_bwd_noalloc(q, k_chunks, v_chunks, d_o, o, lse_final, q_offset: int, k_offsets: Sequence[int], causal: bool,
                        scale: float, order: Sequence[int], dq_acc, dk_acc: Sequence[Optional[torch.Tensor]],
                        dv_acc: Sequence[Optional[torch.Tensor]], mode: int = ST_RING_FUSED, stream=None) -> None:
    """st_ring_bwd on the library's static scratch: this wrapper allocates no device memory either."""
    if _done(_binding.ring_bwd(q, k_chunks, v_chunks, d_o, o, lse_final, q_offset, k_offsets, causal, scale, order, dq_acc, dk_acc, dv_acc,
                               False, None, None, mode, None, _raw_stream(stream)), "st_ring_bwd_noalloc"):
        return
    B, Sq, Hq, D = q.shape
    r = _Ring(q, k_chunks, v_chunks, q_offset, k_offsets, causal, scale)
    n = len(k_chunks)
    _f32_dense(dq_acc, (B, Sq, Hq, D), "dq_acc"); _f32_dense(lse_final, (B, Hq, Sq), "lse_final")
    kv_shape = tuple(k_chunks[0].shape)
    for t in list(dk_acc) + list(dv_acc):
        if t is not None:
            _f32_dense(t, kv_shape, "dk_acc/dv_acc entry")
    dk_ptr = (C.c_void_p * n)(*[(t.data_ptr() if t is not None else None) for t in dk_acc])
    dv_ptr = (C.c_void_p * n)(*[(t.data_ptr() if t is not None else None) for t in dv_acc])
    tq, td, to = _view(q), _view(d_o), _view(o)
    _check(_lib.st_ring_bwd_noalloc(C.byref(r.desc), C.byref(tq), C.byref(td), C.byref(to), _dtype_code(o),
                                    _ptr(lse_final), _i32_array(order), len(order), mode, _ptr(dq_acc),
                                    dk_ptr, dv_ptr,
                                    _stream(stream)), "st_ring_bwd_noalloc")


def st_ring_bwd_last(q, k_chunks, v_chunks, d_o, o, lse_final, q_offset: int, k_offsets: Sequence[int], causal: bool,
                     scale: float, order: Sequence[int], dq_acc, dk_acc: Sequence[Optional[torch.Tensor]],
                     dv_acc: Sequence[Optional[torch.Tensor]], assign: bool = False,
                     dk_lowp: Optional[Sequence[Optional[torch.Tensor]]] = None,
                     dv_lowp: Optional[Sequence[Optional[torch.Tensor]]] = None, mode: int = ST_RING_FUSED,
                     workspace=None, stream=None) -> None:
    if workspace is not None and \
            _done(_binding.ring_bwd(q, k_chunks, v_chunks, d_o, o, lse_final, q_offset, k_offsets, causal, scale, order, dq_acc, dk_acc,
                                    dv_acc, assign, dk_lowp, dv_lowp, mode, workspace, _raw_stream(stream)), "st_ring_bwd_last"):
        return
    B, Sq, Hq, D = q.shape
    r = _Ring(q, k_chunks, v_chunks, q_offset, k_offsets, causal, scale)
    n = len(k_chunks)
    _f32_dense(dq_acc, (B, Sq, Hq, D), "dq_acc"); _f32_dense(lse_final, (B, Hq, Sq), "lse_final")
    kv_shape = tuple(k_chunks[0].shape)
    for t in list(dk_acc) + list(dv_acc):
        if t is not None:
            _f32_dense(t, kv_shape, "dk_acc/dv_acc entry")

    def table(ts):
        if ts is None:
            return None
        for t in ts:
            if t is not None and not (t.is_cuda and t.is_contiguous() and t.dtype == q.dtype and t.shape == kv_shape):
                raise ValueError("dk_lowp/dv_lowp entry: expected a dense device tensor shaped like a chunk, in the dtype of q")
        return (C.c_void_p * n)(*[(t.data_ptr() if t is not None else None) for t in ts])

    dk_ptr, dv_ptr = _ptr_table(dk_acc, n), _ptr_table(dv_acc, n)
    lk, lv = table(dk_lowp), table(dv_lowp)
    if workspace is None:
        need = int(_lib.st_ring_workspace_bytes(C.byref(r.desc), mode, 1))
        workspace = torch.empty(need + 256, dtype=torch.uint8, device=q.device)
    ws_ptr = (workspace.data_ptr() + 255) // 256 * 256
    ws_bytes = workspace.numel() * workspace.element_size() - (ws_ptr - workspace.data_ptr())
    tq, td, to = _view(q), _view(d_o), _view(o)
    _check(_lib.st_ring_bwd_last(C.byref(r.desc), C.byref(tq), C.byref(td), C.byref(to), _dtype_code(o), _ptr(lse_final),
                                 _i32_array(order), len(order), mode, _ptr(dq_acc), dk_ptr, dv_ptr,
                                 ST_KV_ASSIGN if assign else 0, lk, lv, C.c_void_p(ws_ptr), ws_bytes, _stream(stream)),
           "st_ring_bwd_last")


def _ptr_table(ts, n):
    return (C.c_void_p * n)(*[(t.data_ptr() if t is not None else None) for t in ts])


# ---- attention with modified scores, norms and rotations of queries and keys

@contextlib.contextmanager
def _switched(device, stream):
    """The tensors' device as the current one, and `stream` as torch's, so that what is allocated meanwhile belongs to it."""
    with torch.cuda.device(device):
        if stream is None:
            yield
        else:
            with torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=device)):
                yield


_AS_IT_IS = contextlib.nullcontext()


def _on_device(stream, *tensors):
    """All tensors (None: left out) on one GPU; a context in which outputs and workspaces are allocated and the call is made."""
    device = tensors[0].device
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"tensors on {device} and {t.device}")
    if device.type != "cuda":
        raise ValueError(f"expected tensors on a GPU, not on {device}")
    return _AS_IT_IS if stream is None and device.index == torch._C._cuda_getDevice() else _switched(device, stream)


def _short(call, stream, *args):
    """The outputs of a native call that makes its own, on the current stream; None where it leaves the call to ctypes (which raises
    the error of a call that failed, too)."""
    if stream is not None or not torch.cuda.is_initialized():
        return None
    device = torch._C._cuda_getDevice()
    done = call(*args, device, torch._C._cuda_getCurrentRawStream(device))
    return done[1:] if done is not None and done[0] == 0 else None


def _dense(t, shape, dtype, name):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    return t


def _score_desc(q, k, v, q_offset, k_offset, causal, scale, softcap, slopes, spans):
    if q.dim() != 4 or k.dim() != 4 or v.shape != k.shape or k.shape[0] != q.shape[0] or k.shape[3] != q.shape[3]:
        raise ValueError("expected q [B,Sq,Hq,D] and k, v [B,Sk,Hkv,D]")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k and v must have one dtype")
    if slopes is not None:
        _dense(slopes, (q.shape[2],), torch.float32, "slopes")
    if spans is not None:
        _dense(spans, (q.shape[0], q.shape[1], 2), torch.int64, "spans")
    return _block_desc(q, k, q_offset, k_offset, causal, scale), \
        st_score(float(softcap), slopes.data_ptr() if slopes is not None else None, spans.data_ptr() if spans is not None else None)


def _score_workspace(d, m, backward: bool, workspace, device):
    """(pointer, bytes, tensor that has to live until the call is made)"""
    if workspace is None:
        need = int(_lib.st_attn_score_workspace_bytes(C.byref(d), C.byref(m), 1 if backward else 0))
        if need == 0:
            return None, 0, None
        workspace = torch.empty(need + 256, dtype=torch.uint8, device=device)
    ptr, size = _aligned(workspace, 256)
    return ptr, size, workspace


def st_mask_spans(bounds, Sq: int, q_offset, causal: bool, prefix=None, spans=None, stream=None) -> torch.Tensor:
    """Spans [B, Sq, 2] of the rows of packed documents: bounds int64 [B, n_docs + 1] (rising positions at which the documents
    start, and the end of the last one), prefix int64 [B, n_docs] or None (first tokens that a whole document sees)."""
    done = _short(_binding.mask_spans, stream, bounds, Sq, q_offset, causal, prefix, spans)
    if done is not None:
        return done[0]
    with _on_device(stream, bounds, prefix, spans):
        if bounds.dim() != 2 or bounds.shape[1] < 1:
            raise ValueError("bounds must be [B, n_docs + 1]")
        B, n = bounds.shape[0], bounds.shape[1] - 1
        _fit(_INT32, B, int(Sq), n)
        _dense(bounds, (B, n + 1), torch.int64, "bounds")
        if prefix is not None:
            _dense(prefix, (B, n), torch.int64, "prefix")
        spans = torch.empty((B, int(Sq), 2), dtype=torch.int64, device=bounds.device) if spans is None else \
            _dense(spans, (B, int(Sq), 2), torch.int64, "spans")
        off, seg, off2 = _q_runs(q_offset)
        _check(_lib.st_mask_spans(B, int(Sq), off, seg, off2, 1 if causal else 0, _ptr(bounds), n, _ptr(prefix), _ptr(spans),
                                  _stream(None)), "st_mask_spans")
    return spans


def st_attn_score_workspace_bytes(q, k, v, q_offset, k_offset: int, causal: bool, scale: float, softcap: float = 0.0, slopes=None,
                                  spans=None, backward: bool = False) -> int:
    d, m = _score_desc(q, k, v, q_offset, k_offset, causal, scale, softcap, slopes, spans)
    return int(_lib.st_attn_score_workspace_bytes(C.byref(d), C.byref(m), 1 if backward else 0))


def st_attn_score_fwd(q, k, v, q_offset, k_offset: int, causal: bool, scale: float, softcap: float = 0.0, slopes=None, spans=None,
                      o_part=None, lse_part=None, o_lowp=None, lowp: bool = False, workspace=None, stream=None):
    """(O, lse) of a query shard against one chunk.  O is the fp32 partial state, or with lowp=True alone O in the dtype of q; both
    are written where both o_part and o_lowp are given (the fp32 one is returned)."""
    done = _short(_binding.score_fwd, stream, q, k, v, q_offset, k_offset, causal, scale, softcap, slopes, spans, o_part, lse_part, o_lowp,
                  lowp, workspace)
    if done is not None:
        return done
    with _on_device(stream, q, k, v, slopes, spans, o_part, lse_part, o_lowp, workspace):
        d, m = _score_desc(q, k, v, q_offset, k_offset, causal, scale, softcap, slopes, spans)
        B, Sq, Hq, D = q.shape
        if o_lowp is None and lowp:
            o_lowp = torch.empty((B, Sq, Hq, D), dtype=q.dtype, device=q.device)
        elif o_lowp is not None:
            _dense(o_lowp, (B, Sq, Hq, D), q.dtype, "o_lowp")
        if o_part is None and o_lowp is None:
            o_part = torch.empty((B, Sq, Hq, D), dtype=torch.float32, device=q.device)
        elif o_part is not None:
            _f32_dense(o_part, (B, Sq, Hq, D), "o_part")
        lse_part = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device) if lse_part is None else \
            _f32_dense(lse_part, (B, Hq, Sq), "lse_part")
        tq, tk, tv = _view(q), _view(k), _view(v)
        ws, size, held = _score_workspace(d, m, False, workspace, q.device)
        _check(_lib.st_attn_score_fwd(C.byref(d), C.byref(m), C.byref(tq), C.byref(tk), C.byref(tv), _ptr(o_part), _ptr(lse_part),
                                      _ptr(o_lowp), C.c_void_p(ws), size, _stream(None)), "st_attn_score_fwd")
    return (o_part if o_part is not None else o_lowp), lse_part


def st_attn_score_bwd(q, k, v, d_o, lse_final, delta, q_offset, k_offset: int, causal: bool, scale: float, softcap: float = 0.0,
                      slopes=None, spans=None, dq_acc=None, dk_acc=None, dv_acc=None, assign: bool = False, dq_lowp=None, dk_lowp=None,
                      dv_lowp=None, workspace=None, stream=None):
    """Gradients of the pair.  With accumulators (all three, fp32) they are added to, or overwritten with assign=True, and the
    *_lowp given are their values in the dtype of q; without accumulators the gradients are written in the dtype of q, into the
    *_lowp given or new tensors.  Returns (dq, dk, dv): the accumulators, or those."""
    if dq_lowp is None and dk_lowp is None and dv_lowp is None:
        done = _short(_binding.score_bwd, stream, q, k, v, q_offset, k_offset, causal, scale, softcap, slopes, spans, d_o, lse_final, delta,
                      dq_acc, dk_acc, dv_acc, assign, workspace)
        if done is not None:
            return done
    with _on_device(stream, q, k, v, d_o, lse_final, delta, slopes, spans, dq_acc, dk_acc, dv_acc, dq_lowp, dk_lowp, dv_lowp, workspace):
        d, m = _score_desc(q, k, v, q_offset, k_offset, causal, scale, softcap, slopes, spans)
        B, Sq, Hq, D = q.shape
        if d_o.shape != q.shape or d_o.dtype != q.dtype:
            raise ValueError("d_o must have the shape and dtype of q")
        _f32_dense(lse_final, (B, Hq, Sq), "lse_final"); _f32_dense(delta, (B, Hq, Sq), "delta")
        acc, low, shapes = [dq_acc, dk_acc, dv_acc], [dq_lowp, dk_lowp, dv_lowp], [tuple(q.shape), tuple(k.shape), tuple(k.shape)]
        if any(a is not None for a in acc) and any(a is None for a in acc):
            raise ValueError("dq_acc, dk_acc and dv_acc: all or none")
        alone = acc[0] is None
        for x, name in enumerate(("dq", "dk", "dv")):
            if not alone:
                _f32_dense(acc[x], shapes[x], name + "_acc")
            if low[x] is not None:
                _dense(low[x], shapes[x], q.dtype, name + "_lowp")
            elif alone:
                low[x] = torch.empty(shapes[x], dtype=q.dtype, device=q.device)
        tq, tk, tv, td = _view(q), _view(k), _view(v), _view(d_o)
        ws, size, held = _score_workspace(d, m, True, workspace, q.device)
        _check(_lib.st_attn_score_bwd(C.byref(d), C.byref(m), C.byref(tq), C.byref(tk), C.byref(tv), C.byref(td), _ptr(lse_final),
                                      _ptr(delta), ST_GRAD_ASSIGN if assign or alone else 0, *[_ptr(a) for a in acc],
                                      *[_ptr(x) for x in low], C.c_void_p(ws), size, _stream(None)), "st_attn_score_bwd")
    return tuple(low) if alone else tuple(acc)


_PAIRS = {"halves": ST_ROPE_HALVES, "neighbours": ST_ROPE_NEIGHBOURS}


def _rope_desc(q, k, freq, offset, positions, axes, pairs, norm, eps, q_weight, k_weight):
    B, S, Hq, D = q.shape
    if k is not None and (k.dim() != 4 or k.shape[:2] != q.shape[:2] or k.shape[3] != D or k.dtype != q.dtype):
        raise ValueError("expected q [B,S,Hq,D] and k [B,S,Hkv,D] of one dtype")
    if pairs not in _PAIRS:
        raise ValueError(f"pairs must be 'halves' or 'neighbours', not {pairs!r}")
    n = freq.numel()
    _dense(freq, (n,), torch.float64, "freq")
    axes = [n] if axes is None else [int(x) for x in axes]
    if not 1 <= len(axes) <= ST_ROPE_MAX_AXES or sum(axes) != n:
        raise ValueError(f"axes: up to {ST_ROPE_MAX_AXES} numbers of pairs that add up to the {n} frequencies")
    if positions is not None:
        _dense(positions, (len(axes), B, S), torch.int32, "positions")
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None:
            _dense(w, (D,), torch.float32, name)
    off, seg, off2 = _q_runs(offset)
    _fit(_INT32, *q.shape, *(k.shape if k is not None else ()), *axes, 2 * n)
    return st_rope_desc(_dtype_code(q), B, S, Hq, k.shape[2] if k is not None else 0, D, 2 * n,
                        _PAIRS[pairs], 1 if norm else 0, float(eps), len(axes),
                        (C.c_int32 * ST_ROPE_MAX_AXES)(*axes), off, seg, off2)


def _like(t, ref, name):
    if t.shape != ref.shape or t.dtype != ref.dtype:
        raise ValueError(f"{name} must have the shape and dtype of its input")
    return t


def _maybe_view(t):
    return _view(t) if t is not None else st_tensor(None, 0, 0, 0)


def st_qk_rope_fwd(q, k, freq, offset=0, positions=None, axes=None, pairs: str = "halves", norm: bool = True, eps: float = 1e-6,
                   q_weight=None, k_weight=None, q_out=None, k_out=None, stream=None):
    """RMS norm of every head of q [B,S,Hq,D] and k [B,S,Hkv,D] (or None) over its D values, with fp32 weights [D] where given, and
    the rotation of its first 2 len(freq) values: freq fp64 radians per position.  Positions are those of a shard's rows (offset: the
    first one's, or (offset, rows of the first run, offset of the second)), or `positions` int32 [axes,B,S] with `axes` the numbers
    of pairs that each axis turns.  Returns (q_out, k_out), new tensors unless given; they may be q and k."""
    done = _short(_binding.rope_fwd, stream, q, k, freq, offset, positions, axes, _PAIRS.get(pairs), norm, eps, q_weight, k_weight, q_out, k_out)
    if done is not None:
        return done
    with _on_device(stream, q, k, freq, positions, q_weight, k_weight, q_out, k_out):
        d = _rope_desc(q, k, freq, offset, positions, axes, pairs, norm, eps, q_weight, k_weight)
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else _like(q_out, q, "q_out")
        if k is not None:
            k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None else _like(k_out, k, "k_out")
        tq, tk, oq, ok = _view(q), _maybe_view(k), _view(q_out), _maybe_view(k_out if k is not None else None)
        _check(_lib.st_qk_rope_fwd(C.byref(d), C.byref(tq), C.byref(tk), _ptr(q_weight), _ptr(k_weight), _ptr(freq), _ptr(positions),
                                   C.byref(oq), C.byref(ok), _stream(None)), "st_qk_rope_fwd")
    return q_out, k_out if k is not None else None


def st_qk_rope_bwd(q, k, d_q, d_k, freq, offset=0, positions=None, axes=None, pairs: str = "halves", norm: bool = True,
                   eps: float = 1e-6, q_weight=None, k_weight=None, dx_q=None, dx_k=None, dw_q=None, dw_k=None, assign: bool = False,
                   workspace=None, stream=None):
    """Gradients of st_qk_rope_fwd: d_q, d_k those of its outputs, fp32 or in the dtype of q.  Returns (dx_q, dx_k, dw_q, dw_k); the
    weights' (None without weights) are added to the dw_q, dw_k given, or overwrite them with assign=True."""
    if dw_q is None and dw_k is None:
        done = _short(_binding.rope_bwd, stream, q, k, freq, offset, positions, axes, _PAIRS.get(pairs), norm, eps, q_weight, k_weight, d_q, d_k,
                      dx_q, dx_k, workspace)
        if done is not None:
            return done
    with _on_device(stream, q, k, d_q, d_k, freq, positions, q_weight, k_weight, dx_q, dx_k, dw_q, dw_k, workspace):
        d = _rope_desc(q, k, freq, offset, positions, axes, pairs, norm, eps, q_weight, k_weight)
        if d_q.shape != q.shape or (k is not None and (d_k.shape != k.shape or d_k.dtype != d_q.dtype)):
            raise ValueError("d_q and d_k must have the shapes of q and k, and one dtype")
        D = q.shape[3]
        dx_q = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dx_q is None else _like(dx_q, q, "dx_q")
        if k is not None:
            dx_k = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dx_k is None else _like(dx_k, k, "dx_k")
        fresh = [(q_weight is not None and dw_q is None), (k is not None and k_weight is not None and dw_k is None)]
        if (dw_q is not None or dw_k is not None) and any(fresh):
            raise ValueError("dw_q and dw_k: both or neither, where both have weights")
        if any(fresh):
            assign = True
            dw_q = torch.empty((D,), dtype=torch.float32, device=q.device) if fresh[0] else None
            dw_k = torch.empty((D,), dtype=torch.float32, device=q.device) if fresh[1] else None
        for w, name in ((dw_q, "dw_q"), (dw_k, "dw_k")):
            if w is not None:
                _f32_dense(w, (D,), name)
        ptr, size = None, 0
        if dw_q is not None or dw_k is not None:
            if workspace is None:
                workspace = torch.empty(int(_lib.st_qk_rope_bwd_workspace_bytes(C.byref(d))) + 256, dtype=torch.uint8, device=q.device)
            ptr, size = _aligned(workspace, 256)
        tq, tk, gq, gk, oq, ok = (_maybe_view(t) for t in (q, k, d_q, d_k if k is not None else None, dx_q, dx_k if k is not None else None))
        _check(_lib.st_qk_rope_bwd(C.byref(d), C.byref(tq), C.byref(tk), C.byref(gq), C.byref(gk), _dtype_code(d_q), _ptr(q_weight),
                                   _ptr(k_weight), _ptr(freq), _ptr(positions), ST_GRAD_ASSIGN if assign else 0, C.byref(oq),
                                   C.byref(ok), _ptr(dw_q), _ptr(dw_k), C.c_void_p(ptr), size, _stream(None)), "st_qk_rope_bwd")
    return dx_q, (dx_k if k is not None else None), dw_q, dw_k


def st_qk_rope_bwd_workspace_bytes(q, k, freq, norm: bool = True) -> int:
    return int(_lib.st_qk_rope_bwd_workspace_bytes(C.byref(_rope_desc(q, k, freq, 0, None, None, "halves", norm, 1e-6, None, None))))


# ---- a cache of keys and values in pages

class KVCache(NamedTuple):
    """A cache as the calls below take it.  k, v [n_pages, page, Hkv, D] (any strides with D contiguous) in fp32, bf16 or
    float8_e4m3fn; table int32 [B, width]: the pages of every sequence; lens int32 [B]: its tokens, those of the rows at hand among
    them; k_scale, v_scale uint8 [n_pages, Hkv], with pages in 8 bits only: a stored value stands for itself times 2^(scale - 127)."""
    k: torch.Tensor
    v: torch.Tensor
    table: torch.Tensor
    lens: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


_CHUNK_TYPES = {torch.float32: ST_F32, torch.bfloat16: ST_BF16}
_PAGE_TYPES = {torch.float32: ST_F32, torch.bfloat16: ST_BF16, torch.float8_e4m3fn: ST_E4M3}


def _cache_desc(c: KVCache) -> st_cache:
    if c.k.dim() != 4 or c.v.shape != c.k.shape or c.v.dtype != c.k.dtype:
        raise ValueError("expected k, v [n_pages,page,Hkv,D] of one shape and dtype")
    if c.k.dtype not in _PAGE_TYPES:
        raise TypeError(f"unsupported dtype {c.k.dtype}")
    n_pages, page, Hkv, D = c.k.shape
    if c.table.dim() != 2:
        raise ValueError("table must be [B, width]")
    B, width = c.table.shape
    _dense(c.table, (B, width), torch.int32, "table")
    _dense(c.lens, (B,), torch.int32, "lens")
    for x, name in ((c.k_scale, "k_scale"), (c.v_scale, "v_scale")):
        if (x is not None) != (c.k.dtype == torch.float8_e4m3fn):
            raise ValueError(f"{name}: with pages in 8 bits, and only there")
        if x is not None:
            _dense(x, (n_pages, Hkv), torch.uint8, name)
    _fit(_INT32, n_pages, page, Hkv, D, B, width)
    return st_cache(_PAGE_TYPES[c.k.dtype], n_pages, page, Hkv, D, B, width, _view(c.k), _view(c.v),
                    c.k_scale.data_ptr() if c.k_scale is not None else None, c.v_scale.data_ptr() if c.v_scale is not None else None,
                    c.table.data_ptr(), c.lens.data_ptr())


def _starts(starts, c: KVCache):
    return _dense(starts, (c.lens.shape[0] + 1,), torch.int32, "starts")


def st_cache_append(q, k, v, starts, cache: KVCache, freq, offset: int = 0, positions=None, axes=None, pairs: str = "halves",
                    norm: bool = True, eps: float = 1e-6, q_weight=None, k_weight=None, q_out=None, stream=None):
    """New rows, packed: q [1,T,Hq,D] (or None), k and v [1,T,Hkv,D], of which sequence b has starts[b] .. starts[b + 1] - 1 (int32
    [B + 1]), its last tokens.  Norms and rotations as in st_qk_rope_fwd at the tokens' places in their sequences + offset (or at
    `positions` int32 [axes,1,T]); keys and values go into the cache.  Returns the queries (a new tensor unless q_out is given, which
    may be q), None without."""
    done = _short(_binding.cache_append, stream, *cache, q, k, v, starts, freq, offset, positions, axes, _PAIRS.get(pairs), norm, eps, q_weight, k_weight, q_out)
    if done is not None:
        return done[0]
    with _on_device(stream, k, q, v, starts, *cache, freq, positions, q_weight, k_weight, q_out):
        c = _cache_desc(cache)
        if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype:
            raise ValueError("expected k and v [1,T,Hkv,D] of one shape and dtype")
        if q is not None and (q.dim() != 4 or q.shape[:2] != k.shape[:2] or q.shape[3] != k.shape[3] or q.dtype != k.dtype):
            raise ValueError("expected q [1,T,Hq,D] with the rows and the dtype of k")
        if q is None and q_out is not None:
            raise ValueError("q_out without q")
        _starts(starts, cache)
        d = _rope_desc(k, k, freq, offset, positions, axes, pairs, norm, eps, q_weight, k_weight)
        d.Hq = q.shape[2] if q is not None else 0
        _fit(_INT32, d.Hq)
        if q is not None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else _like(q_out, q, "q_out")
        tq, tk, tv, to = _maybe_view(q), _view(k), _view(v), _maybe_view(q_out)
        _check(_lib.st_cache_append(C.byref(d), C.byref(c), _ptr(starts), C.byref(tq), C.byref(tk), C.byref(tv), _ptr(q_weight), _ptr(k_weight),
                                    _ptr(freq), _ptr(positions), C.byref(to), _stream(None)), "st_cache_append")
    return q_out


def st_cache_read(cache: KVCache, first, count: int, dtype=None, k_out=None, v_out=None, stream=None):
    """(k, v) chunks [B,count,Hkv,D]: tokens first[b] .. first[b] + count - 1 of every sequence (int32 [B], None: from 0), zeros past
    its end.  dtype: that of the pages; of pages in 8 bits torch.bfloat16 (unless given) or torch.float32."""
    if k_out is None and v_out is None:
        done = _short(_binding.cache_read, stream, *cache, first, count, None if dtype is None else _CHUNK_TYPES.get(dtype, -1))
        if done is not None:
            return done
    with _on_device(stream, cache.k, *cache[1:], first, k_out, v_out):
        c = _cache_desc(cache)
        if dtype is None:
            dtype = k_out.dtype if k_out is not None else torch.bfloat16 if c.dtype == ST_E4M3 else cache.k.dtype
        code = _CHUNK_TYPES.get(dtype)
        if code is None:
            raise TypeError(f"unsupported dtype {dtype}")
        if first is not None:
            _dense(first, (c.B,), torch.int32, "first")
        _fit(_INT32, int(count))
        if int(count) < 0:
            raise ValueError("count must not be negative")
        shape, out = (c.B, int(count), c.Hkv, c.D), []
        for x, name in ((k_out, "k_out"), (v_out, "v_out")):
            if x is None:
                x = torch.empty(shape, dtype=dtype, device=cache.k.device)
            elif tuple(x.shape) != shape or x.dtype != dtype:
                raise ValueError(f"{name} must be a {dtype} tensor of shape {shape}")
            out.append(x)
        tk, tv = _view(out[0]), _view(out[1])
        _check(_lib.st_cache_read(C.byref(c), _ptr(first), int(count), code, C.byref(tk), C.byref(tv), _stream(None)), "st_cache_read")
    return tuple(out)


def _cache_rows(q, cache, causal, scale, max_rows, window, softcap, slopes) -> st_cache_rows:
    if q.dim() != 4 or q.shape[0] != 1 or q.shape[3] != cache.k.shape[3]:
        raise ValueError("expected q [1,T,Hq,D] with the head size of the cache")
    T, Hq = q.shape[1], q.shape[2]
    if slopes is not None:
        _dense(slopes, (Hq,), torch.float32, "slopes")
    max_rows = T if max_rows is None else int(max_rows)
    _fit(_INT32, T, Hq, max_rows, int(window))
    return st_cache_rows(_dtype_code(q), T, Hq, max_rows, 1 if causal else 0, int(window), float(scale), float(softcap),
                         slopes.data_ptr() if slopes is not None else None)


def st_attn_cache_workspace_bytes(q, cache: KVCache, max_rows: Optional[int] = None) -> int:
    r, c = _cache_rows(q, cache, True, 1.0, max_rows, 0, 0.0, None), _cache_desc(cache)
    return int(_lib.st_attn_cache_workspace_bytes(C.byref(r), C.byref(c)))


def st_attn_cache(q, starts, cache: KVCache, causal: bool, scale: float, max_rows: Optional[int] = None, window: int = 0,
                  softcap: float = 0.0, slopes=None, q_first=None, o_part=None, lse_part=None, o_lowp=None, lowp: bool = False,
                  workspace=None, stream=None):
    """(O, lse) of packed rows q [1,T,Hq,D] against the cache: sequence b has rows starts[b] .. starts[b + 1] - 1 (int32 [B + 1]), at
    positions from q_first[b] on (int64 [B], counted from the cache's first token; None: its last tokens).  A row sees the tokens up
    to its position (causal), the last `window` of them (0: all).  No sequence has more than max_rows rows (None: T), and the call is planned
    for as many, as for tokens up to the table's width: give it where it is known (1 for single tokens).  O [1,T,Hq,D] is
    the fp32 state, or with lowp=True alone in the dtype of q; both are written where o_part and o_lowp are given (the fp32 one is
    returned); lse fp32 [1,Hq,T].  Rows of no sequence are left as they were."""
    done = _short(_binding.cache_attn, stream, *cache, q, starts, causal, scale, max_rows, window, softcap, slopes, q_first, o_part, lse_part, o_lowp, lowp,
                  workspace)
    if done is not None:
        return done
    with _on_device(stream, q, starts, *cache, slopes, q_first, o_part, lse_part, o_lowp, workspace):
        r, c = _cache_rows(q, cache, causal, scale, max_rows, window, softcap, slopes), _cache_desc(cache)
        T, Hq = r.T, r.Hq
        _starts(starts, cache)
        if q_first is not None:
            _dense(q_first, (c.B,), torch.int64, "q_first")
        if o_lowp is None and lowp:
            o_lowp = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        elif o_lowp is not None:
            _dense(o_lowp, q.shape, q.dtype, "o_lowp")
        if o_part is None and o_lowp is None:
            o_part = torch.empty(q.shape, dtype=torch.float32, device=q.device)
        elif o_part is not None:
            _f32_dense(o_part, q.shape, "o_part")
        lse_part = torch.empty((1, Hq, T), dtype=torch.float32, device=q.device) if lse_part is None else _f32_dense(lse_part, (1, Hq, T), "lse_part")
        if workspace is None:
            need = int(_lib.st_attn_cache_workspace_bytes(C.byref(r), C.byref(c)))
            workspace = torch.empty(need + 256, dtype=torch.uint8, device=q.device) if need else None
        ws, size = _aligned(workspace, 256) if workspace is not None else (None, 0)
        tq = _view(q)
        _check(_lib.st_attn_cache(C.byref(r), C.byref(c), _ptr(starts), _ptr(q_first), C.byref(tq), _ptr(o_part), _ptr(lse_part), _ptr(o_lowp),
                                  C.c_void_p(ws), size, _stream(None)), "st_attn_cache")
    return (o_part if o_part is not None else o_lowp), lse_part
