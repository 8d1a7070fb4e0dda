"""ctypes binding of liblookat.so: torch tensors in, C-ABI calls out.

Marshalling only — shapes, pointers, strides, the current HIP stream.  Every step of
the method runs in the library's kernels.  If the library is missing the calls raise
(the product has no CPU path).

The calls of a decode step and of a prompt block are marshalled by csrc/marshal.cpp where their
arguments need no work (no copy, no allocation, nothing to refuse); it answers None where they do,
and the Python code below takes the call, as it takes all of them where that module cannot be loaded.  One user's step (12 heads x 1024 keys, 12 layers, one call each): 107 us in
Python, host-bound at 8.7 us a call; 80 us now, the time of the kernels.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import NamedTuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "liblookat.so")

LOOKAT_F16 = 1
LOOKAT_F32 = 2

_lib = None
_marshal = None     # the native marshalling module, bound to the library that is loaded


class LookatError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"lookat status {status}: {message}")
        self.status = status


class _PythonOnly:
    """In the place of the native marshalling where it cannot be loaded: leaves every call to the Python code below."""
    @staticmethod
    def _leave(*args):
        return None
    encode_keys = build_lut = attend_decode = decode_step = decode_step_split = decode_step_gqa = score_prefill = _leave
    pages_write = attend_pages = pages_copy = pages_fork = pages_free = pages_reserve = pages_compact = _leave
    attend_pages_chunk = pages_weigh = pages_evict = beam_select = _leave


class _Shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d_k", ctypes.c_int32),
                ("m", ctypes.c_int32), ("K", ctypes.c_int32)]


class _Pool(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int32), ("H", ctypes.c_int32), ("d_k", ctypes.c_int32), ("m", ctypes.c_int32),
                ("page", ctypes.c_int32), ("value_type", ctypes.c_int), ("codes", ctypes.c_void_p),
                ("values", ctypes.c_void_p), ("exponents", ctypes.c_void_p)]


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads the built library; raises if it has not been built (python -m paper_2601_10155_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise LookatError(-100, f"{_LIB_PATH} is not built; run `python -m paper_2601_10155_amd.build`")
        lib = ctypes.CDLL(_LIB_PATH)
        i32, i64, vp, sz, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
        sp = ctypes.POINTER(_Shape)
        lib.lookat_encode_keys.argtypes = [sp, i64, vp, ctypes.c_int, vp, vp, i64, vp]
        lib.lookat_encode_keys.restype = ctypes.c_int
        lib.lookat_build_lut.argtypes = [sp, i32, vp, ctypes.c_int, vp, vp, vp]
        lib.lookat_build_lut.restype = ctypes.c_int
        lib.lookat_attend_decode_workspace_bytes.argtypes = [sp, i64, i32]
        lib.lookat_attend_decode_workspace_bytes.restype = sz
        lib.lookat_attend_decode_auto_splits.argtypes = [sp, i64]
        lib.lookat_attend_decode_auto_splits.restype = i32
        lib.lookat_attend_decode_launch_shape.argtypes = [sp, i64, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        lib.lookat_attend_decode_launch_shape.restype = ctypes.c_int
        lib.lookat_attend_decode.argtypes = [sp, i64, vp, vp, i64, vp, i64, f32, i32, vp, sz, vp, vp, vp]
        lib.lookat_attend_decode.restype = ctypes.c_int
        lib.lookat_attend_decode_noalloc.argtypes = [sp, i64, vp, vp, i64, vp, i64, f32, i32, vp, vp, vp]
        lib.lookat_attend_decode_noalloc.restype = ctypes.c_int
        lib.lookat_attend_decode_gqa_workspace_bytes.argtypes = [sp, i32, i64, i32]
        lib.lookat_attend_decode_gqa_workspace_bytes.restype = sz
        lib.lookat_attend_decode_gqa.argtypes = [sp, i32, i64, vp, vp, i64, vp, i64, f32, i32, vp, sz, vp, vp, vp]
        lib.lookat_attend_decode_gqa.restype = ctypes.c_int
        lib.lookat_decode_step.argtypes = [sp, i64, vp, vp, ctypes.c_int, vp, vp, i64, vp, i64, f32, vp, vp]
        lib.lookat_decode_step.restype = ctypes.c_int
        lib.lookat_decode_step_entries_per_workgroup.argtypes = [sp, i64]
        lib.lookat_decode_step_entries_per_workgroup.restype = i32
        lib.lookat_probe_decode_step_entries.argtypes = [sp, i32, i64, vp, vp, ctypes.c_int, vp, vp, i64, vp, i64, f32, vp, vp]
        lib.lookat_probe_decode_step_entries.restype = ctypes.c_int
        lib.lookat_decode_step_split_workspace_bytes.argtypes = [sp, i64, i32]
        lib.lookat_decode_step_split_workspace_bytes.restype = sz
        lib.lookat_decode_step_split.argtypes = [sp, i64, vp, vp, ctypes.c_int, vp, vp, i64, vp, i64, f32, i32, vp, sz, vp, vp]
        lib.lookat_decode_step_split.restype = ctypes.c_int
        lib.lookat_decode_step_gqa_workspace_bytes.argtypes = [sp, i32, i64, i32]
        lib.lookat_decode_step_gqa_workspace_bytes.restype = sz
        lib.lookat_decode_step_gqa.argtypes = [sp, i32, i64, vp, vp, ctypes.c_int, vp, vp, i64, vp, i64, f32, i32, vp, sz, vp, vp]
        lib.lookat_decode_step_gqa.restype = ctypes.c_int
        lib.lookat_score_prefill.argtypes = [sp, i32, i64, vp, ctypes.c_int, vp, vp, i64, vp, vp]
        lib.lookat_score_prefill.restype = ctypes.c_int
        lib.lookat_probe_score_prefill_lookup.argtypes = lib.lookat_score_prefill.argtypes
        lib.lookat_probe_score_prefill_lookup.restype = ctypes.c_int
        lib.lookat_probe_score_prefill_short.argtypes = lib.lookat_score_prefill.argtypes
        lib.lookat_probe_score_prefill_short.restype = ctypes.c_int
        lib.lookat_probe_score_prefill_form.argtypes = [sp, i32, i64, ctypes.c_int]
        lib.lookat_probe_score_prefill_form.restype = i32
        lib.lookat_kmeans_step.argtypes = [sp, i64, vp, vp, vp, vp, vp]
        lib.lookat_kmeans_step.restype = ctypes.c_int
        pp = ctypes.POINTER(_Pool)
        lib.lookat_pages_write.argtypes = [pp, i32, i64, vp, i64, vp, ctypes.c_int, i64, vp, i32, i64, vp, vp, vp]
        lib.lookat_pages_write.restype = ctypes.c_int
        lib.lookat_attend_pages_workspace_bytes.argtypes = [pp, i32, i32, i32, i64, i32]
        lib.lookat_attend_pages_workspace_bytes.restype = sz
        lib.lookat_attend_pages.argtypes = [pp, i32, i32, vp, vp, i32, i64, vp, i64, f32, i32, vp, sz, vp, vp]
        lib.lookat_attend_pages.restype = ctypes.c_int
        lib.lookat_attend_pages_chunk_workspace_bytes.argtypes = [pp, i32, i32, i32, i32, i64, i32]
        lib.lookat_attend_pages_chunk_workspace_bytes.restype = sz
        lib.lookat_attend_pages_chunk.argtypes = [pp, i32, i32, i32, vp, ctypes.c_int, i64, i64, i64, vp, vp, i32, i64, vp, vp, i64, f32, i32, vp, sz,
                                                  vp, vp]
        lib.lookat_attend_pages_chunk.restype = ctypes.c_int
        lib.lookat_pages_weigh_workspace_bytes.argtypes = [pp, i32, i32, i32, i64]
        lib.lookat_pages_weigh_workspace_bytes.restype = sz
        lib.lookat_pages_weigh.argtypes = [pp, i32, i32, vp, vp, i32, i64, vp, i64, f32, f32, vp, i32, i64, vp, sz, vp]
        lib.lookat_pages_weigh.restype = ctypes.c_int
        lib.lookat_pages_evict_workspace_bytes.argtypes = [pp, i32, i32]
        lib.lookat_pages_evict_workspace_bytes.restype = sz
        lib.lookat_pages_evict.argtypes = [pp, i32, vp, i32, i64, vp, vp, i32, i64, vp, i32, i32, vp, i32, i64, vp, i32, i64, vp, sz, vp]
        lib.lookat_pages_evict.restype = ctypes.c_int
        lib.lookat_beam_select_workspace_bytes.argtypes = [i32, i32, i32, i32]
        lib.lookat_beam_select_workspace_bytes.restype = sz
        lib.lookat_beam_select.argtypes = [i32, i32, i32, i32, vp, ctypes.c_int, i64, vp, i32, vp, vp, vp, vp, sz, vp]
        lib.lookat_beam_select.restype = ctypes.c_int
        lib.lookat_pages_copy.argtypes = [pp, i32, vp, vp, vp]
        lib.lookat_pages_copy.restype = ctypes.c_int
        lib.lookat_pages_fork.argtypes = [pp, i32, vp, i32, i64, vp, vp, i32, vp, vp, vp]
        lib.lookat_pages_fork.restype = ctypes.c_int
        lib.lookat_pages_free.argtypes = [pp, i32, vp, i32, i64, vp, vp, i32, vp, vp]
        lib.lookat_pages_free.restype = ctypes.c_int
        lib.lookat_pages_reserve_workspace_bytes.argtypes = [pp, i32]
        lib.lookat_pages_reserve_workspace_bytes.restype = sz
        lib.lookat_pages_reserve.argtypes = [pp, i32, vp, i32, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.lookat_pages_reserve.restype = ctypes.c_int
        lib.lookat_pages_compact_workspace_bytes.argtypes = [pp]
        lib.lookat_pages_compact_workspace_bytes.restype = sz
        lib.lookat_pages_compact.argtypes = [pp, i32, vp, i32, i64, vp, vp, vp, i64, vp, vp, vp, sz, vp]
        lib.lookat_pages_compact.restype = ctypes.c_int
        lib.lookat_probe_stream_read.argtypes = [vp, sz, vp, vp]
        lib.lookat_probe_stream_read.restype = ctypes.c_int
        lib.lookat_probe_stream_write.argtypes = [vp, sz, ctypes.c_uint32, vp]
        lib.lookat_probe_stream_write.restype = ctypes.c_int
        lib.lookat_probe_stream_read_shaped.argtypes = [vp, sz, vp, i32, i32, i32, i32, i32, vp]
        lib.lookat_probe_stream_read_shaped.restype = ctypes.c_int
        lib.lookat_probe_empty_launch.argtypes = [i32, i32, vp]
        lib.lookat_probe_empty_launch.restype = ctypes.c_int
        lib.lookat_probe_attend_decode_ticket_workspace_bytes.argtypes = [sp, i64, i32]
        lib.lookat_probe_attend_decode_ticket_workspace_bytes.restype = sz
        lib.lookat_probe_attend_decode_ticket.argtypes = [sp, i64, vp, vp, i64, vp, i64, f32, i32, vp, sz, vp, vp,
                                                          ctypes.POINTER(i32), vp]
        lib.lookat_probe_attend_decode_ticket.restype = ctypes.c_int
        lib.lookat_last_error.restype = ctypes.c_char_p
        lib.lookat_version.restype = ctypes.c_int
        try:
            from . import _marshal as native
            native.bind(torch._C._cuda_getCurrentRawStream, *(
                ctypes.cast(getattr(lib, "lookat_" + name), vp).value for name in (
                    "encode_keys", "build_lut", "attend_decode", "attend_decode_workspace_bytes", "decode_step", "decode_step_split",
                    "decode_step_split_workspace_bytes", "decode_step_gqa", "decode_step_gqa_workspace_bytes", "score_prefill")))
            native.bind_pages(*(ctypes.cast(getattr(lib, "lookat_" + name), vp).value for name in (
                "pages_write", "attend_pages", "attend_pages_workspace_bytes", "pages_copy", "pages_fork", "pages_free", "pages_reserve",
                "pages_reserve_workspace_bytes", "pages_compact", "pages_compact_workspace_bytes")))
            native.bind_serving(*(ctypes.cast(getattr(lib, "lookat_" + name), vp).value for name in (
                "attend_pages_chunk", "attend_pages_chunk_workspace_bytes", "pages_weigh", "pages_weigh_workspace_bytes", "pages_evict",
                "pages_evict_workspace_bytes", "beam_select", "beam_select_workspace_bytes")))
        except (ImportError, AttributeError, TypeError) as e:
            # (not built, or for another torch: the same library calls are made, 2 to 6 us later each)
            warnings.warn(f"the native marshalling is not available ({e}); run `python -m paper_2601_10155_amd.build`", RuntimeWarning)
            native = _PythonOnly()
        globals()["_marshal"] = native
        _lib = lib
    return _lib


def _native():
    if _lib is None:
        load_library()
    return _marshal


def last_error() -> str:
    return load_library().lookat_last_error().decode()


def version() -> int:
    return int(load_library().lookat_version())


def _check(status: int):
    if status != 0:
        raise LookatError(status, last_error())


def _dtype_tag(t: torch.Tensor) -> int:
    if t.dtype == torch.float16:
        return LOOKAT_F16
    if t.dtype == torch.float32:
        return LOOKAT_F32
    raise TypeError(f"expected float16 or float32 tensor, got {t.dtype}")


def _dev(t: torch.Tensor, name: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    return t


def _stream(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


def _bh_stride(t: torch.Tensor, name: str) -> int:
    """Element stride between consecutive (b,h) slabs of a [B,H,L,x] tensor whose slabs are dense."""
    B, H, L, X = t.shape
    if t.stride(3) != 1 or (L > 1 and t.stride(2) != X):
        raise ValueError(f"{name}: each (b,h) slab must be dense [L,{X}]")
    sh = t.stride(1) if H > 1 else max(t.stride(0), L * X)
    if B > 1 and t.stride(0) != H * sh:
        raise ValueError(f"{name}: batch stride must be H times the head stride")
    return sh


def lookat_encode_keys(keys: torch.Tensor, codebooks: torch.Tensor, codes_out: torch.Tensor | None = None,
                       cache: torch.Tensor | None = None, position: int = 0) -> torch.Tensor:
    """keys [B,H,N,d_k] fp16|fp32, codebooks [H,m,256,d_sub] fp32 -> codes [B,H,N,m] uint8.

    With `cache` ([B,H,Lmax,m] uint8) the codes are written in place at rows
    position .. position+N-1 and the cache is returned."""
    rc = _native().encode_keys(keys, codebooks, codes_out, cache, position)
    if rc is not None:
        if rc:
            _check(rc)
        return codes_out if cache is None else cache
    lib = load_library()
    keys = _dev(keys, "keys").contiguous()
    cb = _dev(codebooks, "codebooks").contiguous()
    B, H, N, d_k = keys.shape
    Hc, m, K, d_sub = cb.shape
    if Hc != H or m * d_sub != d_k or cb.dtype != torch.float32:
        raise ValueError("codebooks must be fp32 [H,m,K,d_k/m]")
    shape = _Shape(B, H, d_k, m, K)
    if cache is not None:
        if cache.dtype != torch.uint8 or cache.shape[:2] != (B, H) or cache.shape[3] != m:
            raise ValueError("cache must be uint8 [B,H,Lmax,m]")
        if position < 0 or position + N > cache.shape[2]:
            raise ValueError("position + N exceeds the cache length")
        stride = _bh_stride(cache, "cache")
        ptr = cache.data_ptr() + position * m
        ret = cache
    else:
        if codes_out is None:
            codes_out = torch.empty((B, H, N, m), dtype=torch.uint8, device=keys.device)
        if codes_out.dtype != torch.uint8 or tuple(codes_out.shape) != (B, H, N, m) or not codes_out.is_contiguous():
            raise ValueError("codes_out must be a contiguous uint8 [B,H,N,m] tensor")
        stride = N * m
        ptr = codes_out.data_ptr()
        ret = codes_out
    _check(lib.lookat_encode_keys(ctypes.byref(shape), N, keys.data_ptr(), _dtype_tag(keys), cb.data_ptr(),
                                  ptr, stride, _stream(keys)))
    return ret


def lookat_build_lut(q: torch.Tensor, codebooks: torch.Tensor, lut_out: torch.Tensor | None = None) -> torch.Tensor:
    """q [B,H,T,d_k] fp16|fp32 -> lut [B,H,T,m,256] fp32."""
    rc = _native().build_lut(q, codebooks, lut_out)
    if rc is not None:
        if rc:
            _check(rc)
        return lut_out
    lib = load_library()
    q = _dev(q, "q").contiguous()
    cb = _dev(codebooks, "codebooks").contiguous()
    B, H, T, d_k = q.shape
    Hc, m, K, d_sub = cb.shape
    if Hc != H or m * d_sub != d_k or cb.dtype != torch.float32:
        raise ValueError("codebooks must be fp32 [H,m,K,d_k/m]")
    shape = _Shape(B, H, d_k, m, K)
    if lut_out is None:
        lut_out = torch.empty((B, H, T, m, K), dtype=torch.float32, device=q.device)
    if lut_out.dtype != torch.float32 or lut_out.numel() != B * H * T * m * K or not lut_out.is_contiguous():
        raise ValueError("lut_out must be a contiguous fp32 tensor of B*H*T*m*K elements")
    _check(lib.lookat_build_lut(ctypes.byref(shape), T, q.data_ptr(), _dtype_tag(q), cb.data_ptr(),
                                lut_out.data_ptr(), _stream(q)))
    return lut_out


def _decode_shape(lut, codes, values):
    B, H, L, m = codes.shape
    d_k = values.shape[3]
    if lut.numel() != B * H * m * 256 or lut.dtype != torch.float32 or not lut.is_contiguous():
        raise ValueError("lut must be contiguous fp32 [B,H,m,256]")
    if codes.dtype != torch.uint8 or values.dtype != torch.float16:
        raise ValueError("codes must be uint8 and values fp16")
    if tuple(values.shape[:3]) != (B, H, L):
        raise ValueError("values must be [B,H,L,d_k] matching codes [B,H,L,m]")
    return _Shape(B, H, d_k, m, 256), L


def attend_decode_workspace_bytes(B: int, H: int, d_k: int, m: int, L: int, num_splits: int = 0) -> int:
    shape = _Shape(B, H, d_k, m, 256)
    return int(load_library().lookat_attend_decode_workspace_bytes(ctypes.byref(shape), L, num_splits))


def attend_decode_gqa_workspace_bytes(B: int, H: int, group: int, d_k: int, m: int, L: int, num_splits: int = 0) -> int:
    """Workspace of lookat_attend_decode_gqa (H = key/value heads; num_splits 0 = the library's choice)."""
    shape = _Shape(B, H, d_k, m, 256)
    return int(load_library().lookat_attend_decode_gqa_workspace_bytes(ctypes.byref(shape), group, L, num_splits))


def attend_decode_auto_splits(B: int, H: int, d_k: int, m: int, L: int) -> int:
    shape = _Shape(B, H, d_k, m, 256)
    return int(load_library().lookat_attend_decode_auto_splits(ctypes.byref(shape), L))


def attend_decode_launch_shape(B: int, H: int, d_k: int, m: int, L: int, num_splits: int = 0) -> tuple[int, int]:
    """(ranges per (b,h), wavefronts per workgroup) of the launch lookat_attend_decode makes for this problem."""
    shape = _Shape(B, H, d_k, m, 256)
    ranges, waves = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(load_library().lookat_attend_decode_launch_shape(ctypes.byref(shape), L, num_splits, ctypes.byref(ranges),
                                                            ctypes.byref(waves)))
    return int(ranges.value), int(waves.value)


def lookat_attend_decode(lut: torch.Tensor, codes: torch.Tensor, values: torch.Tensor, scale: float,
                         num_splits: int = 0, workspace: torch.Tensor | None = None,
                         out: torch.Tensor | None = None, scores_out: torch.Tensor | None = None) -> torch.Tensor:
    """lut [B,H,m,256] fp32, codes [B,H,L,m] u8, values [B,H,L,d_k] fp16 -> out [B,H,d_k] fp32.

    codes / values may be views of longer caches ([B,H,Lmax,*] sliced to L rows)."""
    rc = _native().attend_decode(lut, codes, values, scale, num_splits, workspace, out, scores_out)
    if rc is not None:
        if out is None and rc.__class__ is not int:
            return rc                # the output, allocated there
        if rc:
            _check(rc)
        return out
    lib = load_library()
    _dev(lut, "lut"), _dev(codes, "codes"), _dev(values, "values")
    shape, L = _decode_shape(lut, codes, values)
    B, H, d_k = shape.B, shape.H, shape.d_k
    cs = _bh_stride(codes, "codes")
    vs = _bh_stride(values, "values")
    need = int(lib.lookat_attend_decode_workspace_bytes(ctypes.byref(shape), L, num_splits))
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=values.device)
    if out is None:
        out = torch.empty((B, H, d_k), dtype=torch.float32, device=values.device)
    if out.dtype != torch.float32 or out.numel() != B * H * d_k or not out.is_contiguous():
        raise ValueError("out must be contiguous fp32 [B,H,d_k]")
    if scores_out is not None and (scores_out.dtype != torch.float32 or scores_out.numel() != B * H * L
                                   or not scores_out.is_contiguous()):
        raise ValueError("scores_out must be contiguous fp32 [B,H,L]")
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib.lookat_attend_decode(ctypes.byref(shape), L, lut.data_ptr(), codes.data_ptr(), cs,
                                    values.data_ptr(), vs, float(scale), int(num_splits), ws_ptr, ws_bytes,
                                    out.data_ptr(), scores_out.data_ptr() if scores_out is not None else None,
                                    _stream(values)))
    return out


def lookat_attend_decode_noalloc(lut: torch.Tensor, codes: torch.Tensor, values: torch.Tensor, scale: float,
                                 out: torch.Tensor, num_splits: int = 0,
                                 scores_out: torch.Tensor | None = None) -> torch.Tensor:
    """lookat_attend_decode without a workspace (the library's own scratch memory): for callers that
    cannot allocate.  `out` [B,H,d_k] fp32 must be given; nothing is allocated here or in the library."""
    lib = load_library()
    _dev(lut, "lut"), _dev(codes, "codes"), _dev(values, "values"), _dev(out, "out")
    shape, L = _decode_shape(lut, codes, values)
    if out.dtype != torch.float32 or out.numel() != shape.B * shape.H * shape.d_k or not out.is_contiguous():
        raise ValueError("out must be contiguous fp32 [B,H,d_k]")
    if scores_out is not None and (scores_out.dtype != torch.float32 or scores_out.numel() != shape.B * shape.H * L
                                   or not scores_out.is_contiguous()):
        raise ValueError("scores_out must be contiguous fp32 [B,H,L]")
    _check(lib.lookat_attend_decode_noalloc(ctypes.byref(shape), L, lut.data_ptr(), codes.data_ptr(),
                                            _bh_stride(codes, "codes"), values.data_ptr(), _bh_stride(values, "values"),
                                            float(scale), int(num_splits), out.data_ptr(),
                                            scores_out.data_ptr() if scores_out is not None else None, _stream(values)))
    return out


def lookat_attend_decode_gqa(lut: torch.Tensor, codes: torch.Tensor, values: torch.Tensor, scale: float,
                             num_splits: int = 0, workspace: torch.Tensor | None = None,
                             out: torch.Tensor | None = None, scores_out: torch.Tensor | None = None) -> torch.Tensor:
    """Grouped queries: lut [B,H*g,m,256] fp32, codes [B,H,L,m] u8, values [B,H,L,d_k] fp16
    -> out [B,H*g,d_k] fp32; H counts key/value heads, g = lut.shape[1] // H query heads share each."""
    lib = load_library()
    _dev(lut, "lut"), _dev(codes, "codes"), _dev(values, "values")
    B, H, L, m = codes.shape
    d_k = values.shape[3]
    if lut.dim() != 4 or lut.shape[0] != B or lut.shape[1] % H or tuple(lut.shape[2:]) != (m, 256) \
            or lut.dtype != torch.float32 or not lut.is_contiguous():
        raise ValueError("lut must be contiguous fp32 [B,H*g,m,256]")
    g = lut.shape[1] // H
    if codes.dtype != torch.uint8 or values.dtype != torch.float16 or tuple(values.shape[:3]) != (B, H, L):
        raise ValueError("codes must be uint8 [B,H,L,m] and values fp16 [B,H,L,d_k]")
    shape = _Shape(B, H, d_k, m, 256)
    cs = _bh_stride(codes, "codes")
    vs = _bh_stride(values, "values")
    need = int(lib.lookat_attend_decode_gqa_workspace_bytes(ctypes.byref(shape), g, L, num_splits))
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=values.device)
    if out is None:
        out = torch.empty((B, H * g, d_k), dtype=torch.float32, device=values.device)
    if out.dtype != torch.float32 or out.numel() != B * H * g * d_k or not out.is_contiguous():
        raise ValueError("out must be contiguous fp32 [B,H*g,d_k]")
    if scores_out is not None and (scores_out.dtype != torch.float32 or scores_out.numel() != B * H * g * L
                                   or not scores_out.is_contiguous()):
        raise ValueError("scores_out must be contiguous fp32 [B,H*g,L]")
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib.lookat_attend_decode_gqa(ctypes.byref(shape), g, L, lut.data_ptr(), codes.data_ptr(), cs,
                                        values.data_ptr(), vs, float(scale), int(num_splits), ws_ptr, ws_bytes,
                                        out.data_ptr(), scores_out.data_ptr() if scores_out is not None else None,
                                        _stream(values)))
    return out


def lookat_decode_step(q: torch.Tensor, k_new: torch.Tensor, codebooks: torch.Tensor, codes: torch.Tensor,
                       values: torch.Tensor, scale: float, out: torch.Tensor | None = None) -> torch.Tensor:
    """Fused decode step.  q, k_new [B,H,d_k] (same dtype), codes [B,H,L,m] u8 (row L-1 is written),
    values [B,H,L,d_k] fp16 (row L-1 already holds the new value) -> out [B,H,d_k] fp32.
    codes / values may be views of longer caches sliced to L rows."""
    rc = _native().decode_step(q, k_new, codebooks, codes, values, scale, out)
    if rc is not None:
        if rc:
            _check(rc)
        return out
    return _decode_step(q, k_new, codebooks, codes, values, scale, out, None, None)


def decode_step_entries_per_workgroup(B: int, H: int, d_k: int, m: int, L: int) -> int:
    """Batch entries one workgroup of lookat_decode_step serves for this problem (1 or 2; 0: no kernel)."""
    shape = _Shape(B, H, d_k, m, 256)
    return int(load_library().lookat_decode_step_entries_per_workgroup(ctypes.byref(shape), L))


def lookat_probe_decode_step_entries(entries_per_workgroup: int, q: torch.Tensor, k_new: torch.Tensor,
                                     codebooks: torch.Tensor, codes: torch.Tensor, values: torch.Tensor, scale: float,
                                     out: torch.Tensor | None = None) -> torch.Tensor:
    """lookat_decode_step on the kernel instance that serves `entries_per_workgroup` (1 or 2) batch entries of
    a head per workgroup (2: even B, d_k = 64; measurement aid)."""
    return _decode_step(q, k_new, codebooks, codes, values, scale, out, None, None,
                        _entries=int(entries_per_workgroup))


def lookat_decode_step_split(q: torch.Tensor, k_new: torch.Tensor, codebooks: torch.Tensor, codes: torch.Tensor,
                             values: torch.Tensor, scale: float, num_splits: int = 0,
                             workspace: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """The fused decode step with every (b,h)'s sequence cut into num_splits ranges (0 = the library's
    choice): for few (b,h) pairs and long contexts.  Arguments as lookat_decode_step."""
    rc = _native().decode_step_split(q, k_new, codebooks, codes, values, scale, num_splits, workspace, out)
    if rc is not None:
        if out is None and rc.__class__ is not int:
            return rc                # the output, allocated there
        if rc:
            _check(rc)
        return out
    return _decode_step(q, k_new, codebooks, codes, values, scale, out, int(num_splits), workspace)


def lookat_decode_step_gqa(q: torch.Tensor, k_new: torch.Tensor, codebooks: torch.Tensor, codes: torch.Tensor,
                           values: torch.Tensor, scale: float, num_splits: int = 0,
                           workspace: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Fused decode step with grouped queries: q [B,H*g,d_k], k_new [B,H,d_k] (same dtype), codebooks
    [H,m,256,d_k/m], codes [B,H,L,m] u8 (row L-1 is written), values [B,H,L,d_k] fp16 -> out [B,H*g,d_k] fp32;
    H counts key/value heads, g = q.shape[1] // H."""
    rc = _native().decode_step_gqa(q, k_new, codebooks, codes, values, scale, num_splits, workspace, out)
    if rc is not None:
        if out is None and rc.__class__ is not int:
            return rc                # the output, allocated there
        if rc:
            _check(rc)
        return out
    lib = load_library()
    q = _dev(q, "q").contiguous()
    k_new = _dev(k_new, "k_new").contiguous()
    cb = _dev(codebooks, "codebooks").contiguous()
    _dev(codes, "codes"), _dev(values, "values")
    B, H, L, m = codes.shape
    d_k = values.shape[3]
    if q.dim() != 3 or q.shape[0] != B or q.shape[1] % H or q.shape[2] != d_k or q.dtype != k_new.dtype \
            or k_new.numel() != B * H * d_k:
        raise ValueError("q must be [B,H*g,d_k] and k_new [B,H,d_k], of one dtype")
    g = q.shape[1] // H
    if cb.dtype != torch.float32 or tuple(cb.shape) != (H, m, 256, d_k // m):
        raise ValueError("codebooks must be fp32 [H,m,256,d_k/m]")
    if codes.dtype != torch.uint8 or values.dtype != torch.float16 or tuple(values.shape[:3]) != (B, H, L):
        raise ValueError("codes must be uint8 [B,H,L,m] and values fp16 [B,H,L,d_k]")
    cs = _bh_stride(codes, "codes")
    vs = _bh_stride(values, "values")
    if out is None:
        out = torch.empty((B, H * g, d_k), dtype=torch.float32, device=values.device)
    if out.dtype != torch.float32 or out.numel() != B * H * g * d_k or not out.is_contiguous():
        raise ValueError("out must be contiguous fp32 [B,H*g,d_k]")
    shape = _Shape(B, H, d_k, m, 256)
    need = int(lib.lookat_decode_step_gqa_workspace_bytes(ctypes.byref(shape), g, L, num_splits))
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=values.device)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib.lookat_decode_step_gqa(ctypes.byref(shape), g, L, q.data_ptr(), k_new.data_ptr(), _dtype_tag(q),
                                      cb.data_ptr(), codes.data_ptr(), cs, values.data_ptr(), vs, float(scale),
                                      int(num_splits), ws_ptr, ws_bytes, out.data_ptr(), _stream(values)))
    return out


def decode_step_split_workspace_bytes(B: int, H: int, d_k: int, m: int, L: int, num_splits: int = 0) -> int:
    shape = _Shape(B, H, d_k, m, 256)
    return int(load_library().lookat_decode_step_split_workspace_bytes(ctypes.byref(shape), L, num_splits))


def _decode_step(q, k_new, codebooks, codes, values, scale, out, num_splits, workspace, _entries=None):
    lib = load_library()
    q = _dev(q, "q").contiguous()
    k_new = _dev(k_new, "k_new").contiguous()
    cb = _dev(codebooks, "codebooks").contiguous()
    _dev(codes, "codes"), _dev(values, "values")
    B, H, L, m = codes.shape
    d_k = values.shape[3]
    if q.dtype != k_new.dtype or q.numel() != B * H * d_k or k_new.numel() != B * H * d_k:
        raise ValueError("q and k_new must both be [B,H,d_k] of one dtype")
    if cb.dtype != torch.float32 or tuple(cb.shape) != (H, m, 256, d_k // m):
        raise ValueError("codebooks must be fp32 [H,m,256,d_k/m]")
    if codes.dtype != torch.uint8 or values.dtype != torch.float16 or tuple(values.shape[:3]) != (B, H, L):
        raise ValueError("codes must be uint8 [B,H,L,m] and values fp16 [B,H,L,d_k]")
    cs = _bh_stride(codes, "codes")
    vs = _bh_stride(values, "values")
    if out is None:
        out = torch.empty((B, H, d_k), dtype=torch.float32, device=values.device)
    if out.dtype != torch.float32 or out.numel() != B * H * d_k or not out.is_contiguous():
        raise ValueError("out must be contiguous fp32 [B,H,d_k]")
    shape = _Shape(B, H, d_k, m, 256)
    if num_splits is None:
        if _entries is not None:
            _check(lib.lookat_probe_decode_step_entries(ctypes.byref(shape), _entries, L, q.data_ptr(), k_new.data_ptr(),
                                                        _dtype_tag(q), cb.data_ptr(), codes.data_ptr(), cs,
                                                        values.data_ptr(), vs, float(scale), out.data_ptr(),
                                                        _stream(values)))
            return out
        _check(lib.lookat_decode_step(ctypes.byref(shape), L, q.data_ptr(), k_new.data_ptr(), _dtype_tag(q),
                                      cb.data_ptr(), codes.data_ptr(), cs, values.data_ptr(), vs, float(scale),
                                      out.data_ptr(), _stream(values)))
        return out
    need = int(lib.lookat_decode_step_split_workspace_bytes(ctypes.byref(shape), L, num_splits))
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=values.device)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib.lookat_decode_step_split(ctypes.byref(shape), L, q.data_ptr(), k_new.data_ptr(), _dtype_tag(q),
                                        cb.data_ptr(), codes.data_ptr(), cs, values.data_ptr(), vs, float(scale),
                                        num_splits, ws_ptr, ws_bytes, out.data_ptr(), _stream(values)))
    return out


def lookat_score_prefill(q: torch.Tensor, codebooks: torch.Tensor, codes: torch.Tensor,
                         scores_out: torch.Tensor | None = None, _entry: str = "lookat_score_prefill") -> torch.Tensor:
    """q [B,H,T,d_k] fp16|fp32, codes [B,H,L,m] u8 (L >= T) -> causal scores [B,H,T,L] fp32
    (-inf where key l is later than query t's position t + L - T)."""
    if _entry == "lookat_score_prefill":
        rc = _native().score_prefill(q, codebooks, codes, scores_out)
        if rc is not None:
            if rc:
                _check(rc)
            return scores_out
    lib = load_library()
    q = _dev(q, "q").contiguous()
    cb = _dev(codebooks, "codebooks").contiguous()
    _dev(codes, "codes")
    B, H, T, d_k = q.shape
    Hc, m, K, d_sub = cb.shape
    L = codes.shape[2]
    if Hc != H or m * d_sub != d_k or cb.dtype != torch.float32:
        raise ValueError("codebooks must be fp32 [H,m,K,d_k/m]")
    if codes.dtype != torch.uint8 or codes.shape[:2] != (B, H) or codes.shape[3] != m:
        raise ValueError("codes must be uint8 [B,H,L,m]")
    cs = _bh_stride(codes, "codes")
    if scores_out is None:
        scores_out = torch.empty((B, H, T, L), dtype=torch.float32, device=q.device)
    if scores_out.dtype != torch.float32 or scores_out.numel() != B * H * T * L or not scores_out.is_contiguous():
        raise ValueError("scores_out must be contiguous fp32 [B,H,T,L]")
    shape = _Shape(B, H, d_k, m, K)
    _check(getattr(lib, _entry)(ctypes.byref(shape), T, L, q.data_ptr(), _dtype_tag(q), cb.data_ptr(),
                                codes.data_ptr(), cs, scores_out.data_ptr(), _stream(q)))
    return scores_out


def lookat_probe_score_prefill_lookup(q: torch.Tensor, codebooks: torch.Tensor, codes: torch.Tensor,
                                      scores_out: torch.Tensor | None = None) -> torch.Tensor:
    """lookat_score_prefill forced onto its lookup-and-sum kernel (measurement aid)."""
    return lookat_score_prefill(q, codebooks, codes, scores_out, _entry="lookat_probe_score_prefill_lookup")


def lookat_probe_score_prefill_short(q: torch.Tensor, codebooks: torch.Tensor, codes: torch.Tensor,
                                     scores_out: torch.Tensor | None = None) -> torch.Tensor:
    """lookat_score_prefill forced onto its kernel for short blocks (measurement aid)."""
    return lookat_score_prefill(q, codebooks, codes, scores_out, _entry="lookat_probe_score_prefill_short")


def probe_score_prefill_form(B: int, H: int, T: int, L: int, d_k: int, m: int, dtype: torch.dtype) -> int:
    """Which kernel lookat_score_prefill takes: 1 lookup-and-sum, 2 dense, 3 dense with the codebook in LDS (0: none)."""
    shape = _Shape(B, H, d_k, m, 256)
    return int(load_library().lookat_probe_score_prefill_form(ctypes.byref(shape), T, L,
                                                              {torch.float16: LOOKAT_F16, torch.float32: LOOKAT_F32}[dtype]))


def lookat_kmeans_step(calib: torch.Tensor, codebooks: torch.Tensor, codebooks_out: torch.Tensor | None = None,
                       assign_out: torch.Tensor | None = None):
    """One Lloyd iteration. calib [H,Nc,d_k] fp32, codebooks [H,m,256,d_sub] fp32 ->
    (new codebooks, assignment [H,Nc,m] uint8 against the input codebooks)."""
    lib = load_library()
    calib = _dev(calib, "calib").contiguous()
    cb = _dev(codebooks, "codebooks").contiguous()
    H, Nc, d_k = calib.shape
    Hc, m, K, d_sub = cb.shape
    if Hc != H or m * d_sub != d_k or cb.dtype != torch.float32 or calib.dtype != torch.float32:
        raise ValueError("calib must be fp32 [H,Nc,d_k] and codebooks fp32 [H,m,K,d_k/m]")
    if codebooks_out is None:
        codebooks_out = torch.empty_like(cb)
    if assign_out is None:
        assign_out = torch.empty((H, Nc, m), dtype=torch.uint8, device=calib.device)
    shape = _Shape(1, H, d_k, m, K)
    _check(lib.lookat_kmeans_step(ctypes.byref(shape), Nc, calib.data_ptr(), cb.data_ptr(), codebooks_out.data_ptr(),
                                  assign_out.data_ptr(), _stream(calib)))
    return codebooks_out, assign_out


def lookat_kmeans(calib: torch.Tensor, codebooks: torch.Tensor, iters: int) -> torch.Tensor:
    """`iters` Lloyd iterations from the given initial codebooks (ping-pong between two buffers)."""
    cur = codebooks.contiguous().clone()
    nxt = torch.empty_like(cur)
    assign = torch.empty((calib.shape[0], calib.shape[1], cur.shape[1]), dtype=torch.uint8, device=calib.device)
    for _ in range(int(iters)):
        lookat_kmeans_step(calib, cur, nxt, assign)
        cur, nxt = nxt, cur
    return cur


# ---- the paged cache with 8-bit values (include/lookat_pages.h) ------------------------------------------------
LOOKAT_VALUES_I8 = 1
LOOKAT_VALUES_E4M3 = 2


class PagePool(NamedTuple):
    """The pages of one layer's cache: codes [P,H,page,m] uint8, values [P,H,page/8,d_k,8] int8 or float8_e4m3fn (token t of a
    page at [t // 8, :, t % 8]), exponents [P,H] int8; a stored q stands for q * 2^exponent."""
    codes: torch.Tensor
    values: torch.Tensor
    exponents: torch.Tensor


def page_pool(pages: int, H: int, d_k: int, m: int, page: int = 64, value_dtype: torch.dtype = torch.int8, device="cuda") -> PagePool:
    """A pool of `pages` free pages for `page` tokens of H heads each (value_dtype int8 or float8_e4m3fn)."""
    if value_dtype not in (torch.int8, torch.float8_e4m3fn):
        raise TypeError(f"expected int8 or float8_e4m3fn values, got {value_dtype}")
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device=device)  # noqa: E731
    return PagePool(zeros(pages, H, page, m), zeros(pages, H, page // 8, d_k, 8).view(value_dtype), zeros(pages, H).view(torch.int8))


def _pool(pool: PagePool) -> _Pool:
    codes, values, exponents = pool
    if codes.dim() != 4 or values.dim() != 5 or codes.dtype != torch.uint8 or exponents.dtype != torch.int8:
        raise ValueError("a pool is codes uint8 [P,H,page,m], values [P,H,page/8,d_k,8] and exponents int8 [P,H]")
    P, H, page, m = codes.shape
    if tuple(values.shape[:2]) != (P, H) or values.shape[2] * 8 != page or values.shape[4] != 8 or tuple(exponents.shape) != (P, H):
        raise ValueError("the pool's values must be [P,H,page/8,d_k,8] and its exponents [P,H] for codes [P,H,page,m]")
    if values.dtype == torch.int8:
        tag = LOOKAT_VALUES_I8
    elif values.dtype == torch.float8_e4m3fn:
        tag = LOOKAT_VALUES_E4M3
    else:
        raise TypeError(f"expected int8 or float8_e4m3fn values, got {values.dtype}")
    if not (codes.is_contiguous() and values.is_contiguous() and exponents.is_contiguous()):
        raise ValueError("the pool's tensors must be contiguous")
    _dev(codes, "codes")
    if values.device != codes.device or exponents.device != codes.device:
        raise ValueError("the pool's tensors must live on one device")
    return _Pool(P, H, values.shape[3], m, page, tag, codes.data_ptr(), values.data_ptr(), exponents.data_ptr())


def _int_array(t: torch.Tensor, name: str, pool: PagePool, n: int | None = None) -> int:
    """A dense int32 array on the pool's device; its address."""
    if t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous() or (n is not None and t.shape[0] != n):
        raise ValueError(f"{name} must be a contiguous int32 [{'n' if n is None else n}] tensor")
    if t.device != pool.codes.device:
        raise ValueError(f"{name} must live on the pool's device")
    return t.data_ptr()


def _table(t: torch.Tensor, name: str, pool: PagePool) -> tuple[int, int, int, int]:
    """Rows, entries per row, row stride and address of a table whose rows are dense."""
    if t.dtype != torch.int32 or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be int32 [S,W] with dense rows")
    if t.device != pool.codes.device:
        raise ValueError(f"{name} must live on the pool's device")
    S, W = t.shape
    return S, W, t.stride(0) if S > 1 else max(W, 1), t.data_ptr()


class _OnDevice:
    """The pool's device as the current one during a call, and the stream that is current there."""

    def __init__(self, pool: PagePool):
        self.index = pool.codes.device.index
        self.guard = None if torch.cuda.current_device() == self.index else torch.cuda.device(self.index)

    def __enter__(self) -> int:
        if self.guard is not None:
            self.guard.__enter__()
        return torch._C._cuda_getCurrentRawStream(self.index)

    def __exit__(self, *args):
        if self.guard is not None:
            self.guard.__exit__(*args)


def _scratch(workspace, need: int, pool: PagePool) -> torch.Tensor | None:
    if not need:
        return workspace
    if workspace is not None and workspace.device != pool.codes.device:
        raise ValueError("workspace must live on the pool's device")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=pool.codes.device)
    return workspace


def _bytes(t: torch.Tensor | None) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


def lookat_pages_write(pool: PagePool, codes: torch.Tensor, values: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                       counts: torch.Tensor | None = None) -> None:
    """The last counts[b] tokens (default N) of every sequence enter its pages: codes [B,H,N,m] uint8 (of lookat_encode_keys), values
    [B,H,N,d_k] fp16|fp32 in rows 0..counts[b]-1, table [B,W] int32, lengths [B] int32 INCLUDING them.  In place."""
    rc = _native().pages_write(pool, codes, values, table, lengths, counts)
    if rc is not None:
        if rc:
            _check(rc)
        return
    lib = load_library()
    c_pool = _pool(pool)
    if codes.dim() != 4 or values.dim() != 4 or codes.dtype != torch.uint8 or tuple(codes.shape[:3]) != tuple(values.shape[:3]) \
            or codes.shape[1] != c_pool.H or codes.shape[3] != c_pool.m or values.shape[3] != c_pool.d_k:
        raise ValueError("codes must be uint8 [B,H,N,m] and values [B,H,N,d_k] of the pool's heads")
    B, H, N, _ = codes.shape
    tag = _dtype_tag(values)
    if codes.device != pool.codes.device or values.device != pool.codes.device:
        raise ValueError("codes and values must live on the pool's device")
    rows, W, stride, t_ptr = _table(table, "table", pool)
    if rows != B:
        raise ValueError("table must have a row for every sequence")
    l_ptr = _int_array(lengths, "lengths", pool, B)
    n_ptr = None if counts is None else _int_array(counts, "counts", pool, B)
    if N == 0 or B == 0:
        return
    with _OnDevice(pool) as stream:
        _check(lib.lookat_pages_write(ctypes.byref(c_pool), B, N, codes.data_ptr(), _bh_stride(codes, "codes"), values.data_ptr(), tag,
                                      _bh_stride(values, "values"), t_ptr, W, stride, l_ptr, n_ptr, stream))


def attend_pages_workspace_bytes(pool: PagePool, B: int, group: int, W: int, max_length: int = 0, num_splits: int = 0) -> int:
    return int(load_library().lookat_attend_pages_workspace_bytes(ctypes.byref(_pool(pool)), B, group, W, max_length, num_splits))


def lookat_attend_pages(lut: torch.Tensor, pool: PagePool, table: torch.Tensor, lengths: torch.Tensor, scale: float, max_length: int = 0,
                        num_splits: int = 0, workspace: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """lut [B,H*g,m,256] fp32 (of lookat_build_lut; g query heads share a key/value head), table [B,W] int32, lengths [B] int32
    -> out [B,H*g,d_k] fp32; zeros for a sequence without tokens.  max_length: the longest length the caller knows of (0: W * page);
    it sizes the launch only."""
    rc = _native().attend_pages(lut, pool, table, lengths, scale, max_length, num_splits, workspace, out)
    if rc is not None:
        if out is None and rc.__class__ is not int:
            return rc                # the output, allocated there
        if rc:
            _check(rc)
        return out
    lib = load_library()
    c_pool = _pool(pool)
    B, W, stride, t_ptr = _table(table, "table", pool)
    H, d_k, m = c_pool.H, c_pool.d_k, c_pool.m
    if not H:
        raise ValueError("the pool has no heads")
    if lut.dim() != 4 or lut.shape[0] != B or lut.shape[1] % H or tuple(lut.shape[2:]) != (m, 256) or lut.dtype != torch.float32 \
            or not lut.is_contiguous():
        raise ValueError("lut must be contiguous fp32 [B,H*g,m,256]")
    g = lut.shape[1] // H
    l_ptr = _int_array(lengths, "lengths", pool, B)
    if out is None:
        out = torch.empty((B, H * g, d_k), dtype=torch.float32, device=pool.codes.device)
    if out.dtype != torch.float32 or out.numel() != B * H * g * d_k or not out.is_contiguous():
        raise ValueError("out must be contiguous fp32 [B,H*g,d_k]")
    if lut.device != pool.codes.device or out.device != pool.codes.device:
        raise ValueError("lut and out must live on the pool's device")
    with _OnDevice(pool) as stream:
        need = lib.lookat_attend_pages_workspace_bytes(ctypes.byref(c_pool), B, g, W, max_length, num_splits)
        workspace = _scratch(workspace, need, pool)
        _check(lib.lookat_attend_pages(ctypes.byref(c_pool), B, g, lut.data_ptr(), t_ptr, W, stride, l_ptr, int(max_length), float(scale),
                                       int(num_splits), _ptr(workspace), _bytes(workspace), out.data_ptr(), stream))
    return out


def attend_pages_chunk_workspace_bytes(pool: PagePool, B: int, N: int, group: int, W: int, max_length: int = 0, num_splits: int = 0) -> int:
    return int(load_library().lookat_attend_pages_chunk_workspace_bytes(ctypes.byref(_pool(pool)), B, N, group, W, max_length, num_splits))


def lookat_attend_pages_chunk(q: torch.Tensor, codebooks: torch.Tensor, pool: PagePool, table: torch.Tensor, lengths: torch.Tensor, scale: float,
                              counts: torch.Tensor | None = None, max_length: int = 0, num_splits: int = 0,
                              workspace: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """q [B,H*g,N,d_k] fp16|fp32 (rows dense, other strides as they are: a transposed [B,N,H*g,d_k] is taken without a copy), codebooks
    [H,m,256,d_k/m] fp32, table [B,W] int32, lengths [B] int32 INCLUDING the chunk's tokens, which the pages hold already, counts [B] int32 (None: N)
    -> out [B,H*g,N,d_k] fp32: row n of sequence b, at position lengths[b] - counts[b] + n, attends over the tokens up to its own.  Rows from
    counts[b] on are left as they were (zeros if out is not given).  max_length: as in lookat_attend_pages."""
    rc = _native().attend_pages_chunk(q, codebooks, pool, table, lengths, scale, counts, max_length, num_splits, workspace, out)
    if rc is not None:
        if out is None and rc.__class__ is not int:
            return rc                # the output, allocated there
        if rc:
            _check(rc)
        return out
    lib = load_library()
    c_pool = _pool(pool)
    B, W, stride, t_ptr = _table(table, "table", pool)
    H, d_k, m = c_pool.H, c_pool.d_k, c_pool.m
    if not H:
        raise ValueError("the pool has no heads")
    if q.dim() != 4 or q.shape[0] != B or not q.shape[1] or q.shape[1] % H or q.shape[3] != d_k:
        raise ValueError("q must be [B,H*g,N,d_k] with a row of table for every sequence")
    tag = _dtype_tag(q)
    Hq, N = q.shape[1], q.shape[2]
    if codebooks.dtype != torch.float32 or tuple(codebooks.shape) != (H, m, 256, d_k // m) or not codebooks.is_contiguous():
        raise ValueError("codebooks must be contiguous fp32 [H,m,256,d_k/m] of the pool's heads")
    if q.device != pool.codes.device or codebooks.device != pool.codes.device:
        raise ValueError("q and codebooks must live on the pool's device")
    l_ptr = _int_array(lengths, "lengths", pool, B)
    n_ptr = None if counts is None else _int_array(counts, "counts", pool, B)
    unit = 16 // q.element_size()
    if q.stride(3) != 1 or q.data_ptr() % 16 or any(q.shape[i] > 1 and q.stride(i) % unit for i in range(3)):
        q = q.contiguous()
    if q.data_ptr() % 16:
        q = q.clone()
    # (a stride that no index uses may be anything)
    sb, sh, sn = (q.stride(i) if q.shape[i] > 1 else 0 for i in range(3))
    if out is None:
        out = (torch.empty if counts is None else torch.zeros)((B, Hq, N, d_k), dtype=torch.float32, device=pool.codes.device)
    if out.dtype != torch.float32 or tuple(out.shape) != (B, Hq, N, d_k) or not out.is_contiguous():
        raise ValueError("out must be contiguous fp32 [B,H*g,N,d_k]")
    if out.device != pool.codes.device:
        raise ValueError("out must live on the pool's device")
    if not N or not B:
        return out
    num_splits = _int32(num_splits, "num_splits")
    with _OnDevice(pool) as stream:
        need = lib.lookat_attend_pages_chunk_workspace_bytes(ctypes.byref(c_pool), B, N, Hq // H, W, max_length, num_splits)
        workspace = _scratch(workspace, need, pool)
        _check(lib.lookat_attend_pages_chunk(ctypes.byref(c_pool), B, N, Hq // H, q.data_ptr(), tag, sb, sh, sn, codebooks.data_ptr(), t_ptr, W, stride,
                                             l_ptr, n_ptr, int(max_length), float(scale), num_splits, _ptr(workspace), _bytes(workspace),
                                             out.data_ptr(), stream))
    return out


def _int32(x: int, name: str) -> int:
    """(ctypes would cut a larger number to its low bits.)"""
    if not -2 ** 31 <= int(x) < 2 ** 31:
        raise ValueError(f"{name} = {x} is out of range")
    return int(x)


def _weight_rows(t: torch.Tensor, name: str, pool: PagePool, B: int, H: int) -> tuple[int, int, int]:
    """Columns, stride between heads and address of fp32 weights [B,H,N] whose rows are dense."""
    if t.dtype != torch.float32 or t.dim() != 3 or tuple(t.shape[:2]) != (B, H) or not t.shape[2]:
        raise ValueError(f"{name} must be fp32 [B,H,N] of the pool's heads")
    if t.device != pool.codes.device:
        raise ValueError(f"{name} must live on the pool's device")
    return t.shape[2], _bh_stride(t.unsqueeze(2), name), t.data_ptr()


def pages_weigh_workspace_bytes(pool: PagePool, B: int, group: int, W: int, max_length: int = 0) -> int:
    return int(load_library().lookat_pages_weigh_workspace_bytes(ctypes.byref(_pool(pool)), B, group, W, max_length))


def lookat_pages_weigh(lut: torch.Tensor, pool: PagePool, table: torch.Tensor, lengths: torch.Tensor, scale: float, weights: torch.Tensor,
                       decay: float = 1.0, max_length: int = 0, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Adds the attention that the queries of lut [B,H*g,m,256] (as lookat_attend_pages takes it) pay to every token, summed over a key/value
    head's g query heads, to decay * weights [B,H,N] fp32 (N >= the longest length, or only the first N tokens have one).  In place; returns weights."""
    rc = _native().pages_weigh(lut, pool, table, lengths, scale, weights, decay, max_length, workspace)
    if rc is not None:
        if rc:
            _check(rc)
        return weights
    lib = load_library()
    c_pool = _pool(pool)
    B, W, stride, t_ptr = _table(table, "table", pool)
    H, m = c_pool.H, c_pool.m
    if not H:
        raise ValueError("the pool has no heads")
    if lut.dim() != 4 or lut.shape[0] != B or not lut.shape[1] or lut.shape[1] % H or tuple(lut.shape[2:]) != (m, 256) or lut.dtype != torch.float32 \
            or not lut.is_contiguous():
        raise ValueError("lut must be contiguous fp32 [B,H*g,m,256]")
    if lut.device != pool.codes.device:
        raise ValueError("lut must live on the pool's device")
    l_ptr = _int_array(lengths, "lengths", pool, B)
    if not B:
        return weights
    columns, w_stride, w_ptr = _weight_rows(weights, "weights", pool, B, H)
    g = lut.shape[1] // H
    with _OnDevice(pool) as stream:
        workspace = _scratch(workspace, lib.lookat_pages_weigh_workspace_bytes(ctypes.byref(c_pool), B, g, W, max_length), pool)
        _check(lib.lookat_pages_weigh(ctypes.byref(c_pool), B, g, lut.data_ptr(), t_ptr, W, stride, l_ptr, int(max_length), float(scale), float(decay),
                                      w_ptr, columns, w_stride, _ptr(workspace), _bytes(workspace), stream))
    return weights


def pages_evict_workspace_bytes(pool: PagePool, B: int, W_out: int) -> int:
    return int(load_library().lookat_pages_evict_workspace_bytes(ctypes.byref(_pool(pool)), B, W_out))


def lookat_pages_evict(pool: PagePool, table: torch.Tensor, lengths: torch.Tensor, weights: torch.Tensor, keep: torch.Tensor,
                       table_out: torch.Tensor, first: int = 0, recent: int = 0, weights_out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None) -> None:
    """min(lengths[b], keep[b]) tokens of every sequence, each head its own - the last `recent`, the first `first`, then the heaviest of weights
    [B,H,N] fp32 - enter the pages of table_out [B,W_out] int32 at positions 0.., in their order (keep [B] int32; reserve that many for empty slots
    first, free the old ones afterwards).  weights_out [B,H,M] fp32, if given, gets the kept tokens' weights in their new places."""
    rc = _native().pages_evict(pool, table, lengths, weights, keep, table_out, first, recent, weights_out, workspace)
    if rc is not None:
        if rc:
            _check(rc)
        return
    lib = load_library()
    c_pool = _pool(pool)
    B, W, stride, t_ptr = _table(table, "table", pool)
    rows, W_out, out_stride, o_ptr = _table(table_out, "table_out", pool)
    if rows != B:
        raise ValueError("table_out must have a row for every sequence")
    l_ptr, k_ptr = _int_array(lengths, "lengths", pool, B), _int_array(keep, "keep", pool, B)
    if not B:
        return
    columns, w_stride, w_ptr = _weight_rows(weights, "weights", pool, B, c_pool.H)
    out = (0, 0, None) if weights_out is None else _weight_rows(weights_out, "weights_out", pool, B, c_pool.H)
    with _OnDevice(pool) as stream:
        workspace = _scratch(workspace, lib.lookat_pages_evict_workspace_bytes(ctypes.byref(c_pool), B, W_out), pool)
        _check(lib.lookat_pages_evict(ctypes.byref(c_pool), B, t_ptr, W, stride, l_ptr, w_ptr, columns, w_stride, k_ptr, _int32(first, "first"),
                                      _int32(recent, "recent"),
                                      o_ptr, W_out, out_stride, out[2], out[0], out[1], _ptr(workspace), _bytes(workspace), stream))


def lookat_pages_copy(pool: PagePool, src: torch.Tensor, dst: torch.Tensor) -> None:
    """Pages src[i] onto pages dst[i] (int32 [n]; the destinations distinct and none of them a source)."""
    rc = _native().pages_copy(pool, src, dst)
    if rc is not None:
        if rc:
            _check(rc)
        return
    lib = load_library()
    c_pool = _pool(pool)
    n = src.shape[0] if src.dim() else 0
    s_ptr, d_ptr = _int_array(src, "src", pool), _int_array(dst, "dst", pool, n)
    with _OnDevice(pool) as stream:
        _check(lib.lookat_pages_copy(ctypes.byref(c_pool), n, s_ptr, d_ptr, stream))


def _books(pool: PagePool, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor) -> tuple:
    S, W, stride, t_ptr = _table(table, "table", pool)
    return S, t_ptr, W, stride, _int_array(lengths, "lengths", pool, S), _int_array(refs, "refs", pool, pool.codes.shape[0])


def lookat_pages_fork(pool: PagePool, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor, src: torch.Tensor,
                      dst: torch.Tensor) -> None:
    """The empty sequences dst[i] begin as src[i]: rows and lengths copied, pages shared and counted once more.
    table [S,W], lengths [S], refs [P], src, dst [n], all int32.  In place."""
    rc = _native().pages_fork(pool, table, lengths, refs, src, dst)
    if rc is not None:
        if rc:
            _check(rc)
        return
    lib = load_library()
    c_pool = _pool(pool)
    books = _books(pool, table, lengths, refs)
    n = src.shape[0] if src.dim() else 0
    s_ptr, d_ptr = _int_array(src, "src", pool), _int_array(dst, "dst", pool, n)
    with _OnDevice(pool) as stream:
        _check(lib.lookat_pages_fork(ctypes.byref(c_pool), *books, n, s_ptr, d_ptr, stream))


def lookat_pages_free(pool: PagePool, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor, slots: torch.Tensor) -> None:
    """Gives up the sequences `slots` (int32 [n]): their pages are counted once less, their rows become -1, their lengths 0.  In place."""
    rc = _native().pages_free(pool, table, lengths, refs, slots)
    if rc is not None:
        if rc:
            _check(rc)
        return
    lib = load_library()
    c_pool = _pool(pool)
    books = _books(pool, table, lengths, refs)
    ptr = _int_array(slots, "slots", pool)
    with _OnDevice(pool) as stream:
        _check(lib.lookat_pages_free(ctypes.byref(c_pool), *books, slots.shape[0], ptr, stream))


def lookat_pages_reserve(pool: PagePool, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor, new_lengths: torch.Tensor,
                         missing: torch.Tensor | None = None, copies: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Room for the sequences to grow to new_lengths [S] int32 (not above lengths: as it is): free pages in ascending order, shared last
    pages copied, lengths set.  Returns `missing` [1] int32: 0, or how many pages are lacking and nothing was changed.
    `copies` [2,S] int32, if given, gets the pages that were copied and their copies (-1: none), for lookat_pages_copy(pool, *copies) on the
    pools of other layers that share these books."""
    rc = _native().pages_reserve(pool, table, lengths, refs, new_lengths, missing, copies, workspace)
    if rc is not None:
        if missing is None and rc.__class__ is not int:
            return rc                # allocated there
        if rc:
            _check(rc)
        return missing
    lib = load_library()
    c_pool = _pool(pool)
    books = _books(pool, table, lengths, refs)
    ptr = _int_array(new_lengths, "new_lengths", pool, books[0])
    if missing is None:
        missing = torch.empty(1, dtype=torch.int32, device=pool.codes.device)
    m_ptr = _int_array(missing, "missing", pool, 1)
    if copies is not None and (copies.dtype != torch.int32 or tuple(copies.shape) != (2, books[0]) or not copies.is_contiguous()
                               or copies.device != pool.codes.device):
        raise ValueError("copies must be a contiguous int32 [2,S] tensor on the pool's device")
    with _OnDevice(pool) as stream:
        workspace = _scratch(workspace, lib.lookat_pages_reserve_workspace_bytes(ctypes.byref(c_pool), books[0]), pool)
        _check(lib.lookat_pages_reserve(ctypes.byref(c_pool), *books, ptr, m_ptr, _ptr(copies), _ptr(workspace), _bytes(workspace), stream))
    return missing


def lookat_pages_compact(pool: PagePool, table: torch.Tensor, lengths: torch.Tensor, refs: torch.Tensor, table_out: torch.Tensor | None = None,
                         refs_out: torch.Tensor | None = None, live: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """The pages in use move to the lowest ids.  Returns the new table [S,W], the new refs [P] and live [1], the number of pages in use
    (int32); the old table and refs are not changed."""
    if table_out is None and refs_out is None and live is None:
        rc = _native().pages_compact(pool, table, lengths, refs, workspace)
        if rc.__class__ is tuple:
            return rc
        if rc:
            _check(rc)
    lib = load_library()
    c_pool = _pool(pool)
    books = _books(pool, table, lengths, refs)
    if table_out is None:
        table_out = torch.empty(table.shape, dtype=torch.int32, device=pool.codes.device)
    if refs_out is None:
        refs_out = torch.empty_like(refs)
    if live is None:
        live = torch.empty(1, dtype=torch.int32, device=pool.codes.device)
    S, W, stride, t_ptr = _table(table_out, "table_out", pool)
    if (S, W) != (books[0], books[2]):
        raise ValueError("table_out must have the table's shape")
    r_ptr, l_ptr = _int_array(refs_out, "refs_out", pool, pool.codes.shape[0]), _int_array(live, "live", pool, 1)
    with _OnDevice(pool) as device_stream:
        workspace = _scratch(workspace, lib.lookat_pages_compact_workspace_bytes(ctypes.byref(c_pool)), pool)
        _check(lib.lookat_pages_compact(ctypes.byref(c_pool), *books, t_ptr, stride, r_ptr, l_ptr, _ptr(workspace), _bytes(workspace),
                                        device_stream))
    return table_out, refs_out, live


# ---- beam search (include/lookat_search.h) ---------------------------------------------------------------------
def beam_select_workspace_bytes(Q: int, beams: int, V: int, n: int) -> int:
    return int(load_library().lookat_beam_select_workspace_bytes(Q, beams, V, n))


def lookat_beam_select(logits: torch.Tensor, scores: torch.Tensor, beams: int, n: int, first_parent: int = 0, scores_out: torch.Tensor | None = None,
                       parents: torch.Tensor | None = None, tokens: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """The n best continuations of each request: logits [Q*beams,V] fp16|fp32 (rows dense), scores [Q*beams] fp32 -> scores [Q,n] fp32 =
    scores + log_softmax(logits), falling, parents [Q,n] int32 (first_parent + row: the slots that lookat_pages_fork copies) and tokens [Q,n] int32;
    -inf, -1, -1 where there are fewer.  Beams of score -inf and tokens of logit -inf are not chosen."""
    if scores_out is None and parents is None and tokens is None:
        rc = _native().beam_select(logits, scores, beams, n, first_parent, workspace)
        if rc.__class__ is tuple:
            return rc
        if rc:
            _check(rc)
    lib = load_library()
    beams, n, first_parent = _int32(beams, "beams"), _int32(n, "n"), _int32(first_parent, "first_parent")
    device = _dev(logits, "logits").device
    if logits.dim() != 2 or beams < 1 or n < 1 or not logits.shape[0] or logits.shape[0] % beams or not logits.shape[1]:
        raise ValueError("logits must be [Q*beams,V]")
    tag = _dtype_tag(logits)
    (R, V), Q = logits.shape, logits.shape[0] // beams
    if V > 1 and logits.stride(1) != 1 or (R > 1 and logits.stride(0) < V):
        raise ValueError("logits: rows must be dense and apart")
    if scores.dtype != torch.float32 or tuple(scores.shape) != (R,) or not scores.is_contiguous():
        raise ValueError("scores must be contiguous fp32 [Q*beams]")
    new = lambda t, dtype: torch.empty((Q, n), dtype=dtype, device=device) if t is None else t  # noqa: E731
    scores_out, parents, tokens = new(scores_out, torch.float32), new(parents, torch.int32), new(tokens, torch.int32)
    for t, name, dtype in ((scores_out, "scores_out", torch.float32), (parents, "parents", torch.int32), (tokens, "tokens", torch.int32)):
        if t.dtype != dtype or tuple(t.shape) != (Q, n) or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dtype} [Q,n]")
    if any(t.device != device for t in (scores, scores_out, parents, tokens)):
        raise ValueError("all tensors must live on the logits' device")
    if workspace is not None and (workspace.device != device or not workspace.is_contiguous()):
        raise ValueError("workspace must be contiguous and live on the logits' device")
    with torch.cuda.device(device):
        need = lib.lookat_beam_select_workspace_bytes(Q, beams, V, n)
        if need and (workspace is None or _bytes(workspace) < need):
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
        _check(lib.lookat_beam_select(Q, beams, V, n, logits.data_ptr(), tag, logits.stride(0) if R > 1 else V, scores.data_ptr(), first_parent,
                                      scores_out.data_ptr(), parents.data_ptr(), tokens.data_ptr(), _ptr(workspace), _bytes(workspace),
                                      torch._C._cuda_getCurrentRawStream(device.index)))
    return scores_out, parents, tokens


def lookat_probe_stream_read(src: torch.Tensor, sink: torch.Tensor) -> None:
    """Measurement aid: streams all bytes of `src` once through a plain read kernel."""
    lib = load_library()
    _dev(src, "src"), _dev(sink, "sink")
    if not src.is_contiguous():
        raise ValueError("src must be contiguous")
    _check(lib.lookat_probe_stream_read(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(),
                                        _stream(src)))


def lookat_probe_stream_write(dst: torch.Tensor, word: int = 0) -> None:
    """Measurement aid: overwrites all bytes of `dst` once with a 32-bit pattern through a plain write kernel."""
    lib = load_library()
    _dev(dst, "dst")
    if not dst.is_contiguous():
        raise ValueError("dst must be contiguous")
    _check(lib.lookat_probe_stream_write(dst.data_ptr(), dst.numel() * dst.element_size(), int(word) & 0xffffffff,
                                         _stream(dst)))


def lookat_probe_stream_read_shaped(src: torch.Tensor, sink: torch.Tensor, threads: int, loads_per_thread: int,
                                    workgroups: int = 0, contiguous: bool = False, nontemporal: bool = True) -> None:
    """Measurement aid: the read stream in a chosen launch shape (see include/lookat_probe.h)."""
    lib = load_library()
    _dev(src, "src"), _dev(sink, "sink")
    if not src.is_contiguous():
        raise ValueError("src must be contiguous")
    _check(lib.lookat_probe_stream_read_shaped(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(),
                                               int(threads), int(loads_per_thread), int(workgroups), int(bool(contiguous)),
                                               int(bool(nontemporal)), _stream(src)))


def lookat_probe_empty_launch(workgroups: int, threads: int) -> None:
    """Measurement aid: launches a kernel that does nothing on the current stream."""
    _check(load_library().lookat_probe_empty_launch(int(workgroups), int(threads),
                                                    torch.cuda.current_stream().cuda_stream))


def probe_attend_decode_ticket_workspace_bytes(B: int, H: int, d_k: int, m: int, L: int, num_splits: int = 0) -> int:
    shape = _Shape(B, H, d_k, m, 256)
    return int(load_library().lookat_probe_attend_decode_ticket_workspace_bytes(ctypes.byref(shape), L, num_splits))


def lookat_probe_attend_decode_ticket(lut: torch.Tensor, codes: torch.Tensor, values: torch.Tensor, scale: float,
                                      num_splits: int = 0, workspace: torch.Tensor | None = None,
                                      out: torch.Tensor | None = None, scores_out: torch.Tensor | None = None):
    """Measurement aid: lookat_attend_decode on the flat geometry with the in-kernel ticket merge.
    Returns (out, pieces per (b,h)).  A workspace allocated here is zeroed (its ticket counters must be)."""
    lib = load_library()
    _dev(lut, "lut"), _dev(codes, "codes"), _dev(values, "values")
    shape, L = _decode_shape(lut, codes, values)
    B, H, d_k = shape.B, shape.H, shape.d_k
    need = int(lib.lookat_probe_attend_decode_ticket_workspace_bytes(ctypes.byref(shape), L, num_splits))
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.zeros(need, dtype=torch.uint8, device=values.device)
    if out is None:
        out = torch.empty((B, H, d_k), dtype=torch.float32, device=values.device)
    pieces = ctypes.c_int32(0)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib.lookat_probe_attend_decode_ticket(ctypes.byref(shape), L, lut.data_ptr(), codes.data_ptr(),
                                                 _bh_stride(codes, "codes"), values.data_ptr(), _bh_stride(values, "values"),
                                                 float(scale), int(num_splits), ws_ptr, ws_bytes, out.data_ptr(),
                                                 scores_out.data_ptr() if scores_out is not None else None,
                                                 ctypes.byref(pieces), _stream(values)))
    return out, int(pieces.value)


# short aliases
encode_keys = lookat_encode_keys
build_lut = lookat_build_lut
attend_decode = lookat_attend_decode
