"""Thin ctypes binding of libperq.so: argument marshalling only.

Every function has the name of the C entry point it calls (see include/perq.h for what
each computes).  torch is used for device memory and streams; all arithmetic of the path
happens inside the CUDA library.  There is no CPU fallback: if the library cannot be
loaded, importing this module's functions raises.

Calls take a `stream` (None: the current one; a torch stream or a handle).  It has to have waited for whatever makes the arguments; tensors
that a call makes are that stream's memory, and the caller's own streams wait for it before they read them.
"""
from __future__ import annotations

import ctypes as C
import functools
import importlib.util
import os
from typing import Optional

import numpy as np
import torch

from . import build as _build

PERQ_FMT_INT4 = 0
PERQ_FMT_MXFP4 = 1
PERQ_FMT_F32_DEBUG = 2
PERQ_FMT_FP4 = 3
PERQ_FMT_INT4_ASYM = 4
PERQ_FMT_INT8 = 5
FMT_BY_NAME = {"int4": PERQ_FMT_INT4, "mxfp4": PERQ_FMT_MXFP4, "f32": PERQ_FMT_F32_DEBUG, "fp4": PERQ_FMT_FP4,
               "int4_asym": PERQ_FMT_INT4_ASYM, "int8": PERQ_FMT_INT8}
OUT_BY_DTYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}        # perq_out_t

PERQ_OK = 0
PERQ_ERR_SHAPE = 2
PERQ_ERR_BLOCK = 3
PERQ_ERR_WORKSPACE = 9

_lib = None
_rotate_quantize = _swiglu_rotate_quantize = None       # the calls of these: perq_call.c, or ctypes where that is not built or cannot be loaded
_rotate_quantize_i8 = _matmul_i8 = _grouped_matmul_i8 = None
_cache_write_i8 = _cache_read_i8 = _attention_i8 = None


class PerqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, status_string(status), status))


def load() -> C.CDLL:
    """Load libperq.so from the package directory (never builds implicitly)."""
    global _lib, _rotate_quantize, _swiglu_rotate_quantize, _rotate_quantize_i8, _matmul_i8, _grouped_matmul_i8, _cache_write_i8, _cache_read_i8, _attention_i8
    if _lib is None:
        path = _build.LIB_PATH
        if not os.path.exists(path):
            raise RuntimeError("%s not found: run `python -m paper_2601_22347_b200.build` "
                               "(or __graft_entry__.build()) first" % path)
        lib = C.CDLL(path)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        lib.perq_rotate_quantize.argtypes = [vp, vp, i64, i32, i32, i32, i32, vp, vp, vp]
        lib.perq_swiglu_rotate_quantize.argtypes = [vp, vp, vp, i64, i32, i32, i32, i32, vp, vp, vp]
        lib.perq_swiglu_rotate_quantize.restype = C.c_int
        lib.perq_rotate_quantize_host.argtypes = [vp, vp, i64, i32, i32, i32, i32, vp, vp, vp, sz, vp]
        lib.perq_host_workspace_bytes.argtypes = [i64, i32, i32, i32, C.POINTER(sz)]
        lib.perq_out_sizes.argtypes = [i64, i32, i32, i32, C.POINTER(sz), C.POINTER(sz)]
        lib.perq_block_l1_stats.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp, vp, sz, vp]
        lib.perq_block_l1_stats_static.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp, vp]
        lib.perq_block_l1_stats_workspace_bytes.argtypes = [i64, i32, i32, C.POINTER(sz)]
        lib.perq_token_diagnostics.argtypes = [vp, vp, i64, i32, i32, vp, vp]
        lib.perq_validate_perm.argtypes = [vp, i32, vp, vp]
        lib.perq_massdiff_perm.argtypes = [vp, i32, i32, vp]
        lib.perq_massdiff_perm_device.argtypes = [vp, i32, i32, vp, vp, sz, vp]
        lib.perq_chan_abs_max.argtypes = [vp, i64, i32, vp, vp]
        lib.perq_absmax_perm.argtypes = [vp, i32, vp]
        lib.perq_zigzag_perm.argtypes = [vp, i32, i32, vp]
        for name in ("perq_chan_abs_max", "perq_absmax_perm", "perq_zigzag_perm"):
            getattr(lib, name).restype = C.c_int
        lib.perq_matmul_i8.argtypes = [vp, vp, i32, vp, vp, i32, vp, i64, i32, i32, vp, i32, vp, sz, vp]
        lib.perq_matmul_i8_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, C.POINTER(sz)]
        lib.perq_grouped_matmul_i8.argtypes = [vp, vp, i32, vp, vp, i32, vp, vp, i64, i32, i32, i32, vp, i32, vp, sz, vp]
        lib.perq_grouped_matmul_i8_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i32, C.POINTER(sz)]
        lib.perq_rotate_quantize_i8.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp]
        lib.perq_code_sums.argtypes = [vp, i32, i64, i32, vp, vp]
        for name in ("perq_rotate_quantize_i8", "perq_code_sums", "perq_matmul_i8", "perq_matmul_i8_workspace_bytes", "perq_grouped_matmul_i8", "perq_grouped_matmul_i8_workspace_bytes"):
            getattr(lib, name).restype = C.c_int
        cache = [vp, vp, vp, i64, i32, i32, i32, i32, i32, i64, i32]             # offsets, lengths, pages; T, S, heads, D, b, page, n_pages, width
        lib.perq_cache_write_i8.argtypes = [vp, vp, i32, i64, i64] + cache + [vp, vp, vp, vp, vp]
        lib.perq_cache_read_i8.argtypes = [vp, vp, vp, vp] + cache + [vp, vp, i32, vp]
        lib.perq_attention_i8.argtypes = ([vp, i32, i64, vp, vp, vp, vp] + cache[:6] + [i32] + cache[6:] +
                                          [i32, C.c_float, i32, i32, vp, i32, vp, sz, vp])
        lib.perq_attention_i8_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i32, C.POINTER(sz)]
        for name in ("perq_cache_write_i8", "perq_cache_read_i8", "perq_attention_i8", "perq_attention_i8_workspace_bytes"):
            getattr(lib, name).restype = C.c_int
        lib.perq_device_error.argtypes = [C.POINTER(C.c_uint32)]
        lib.perq_device_error.restype = C.c_int
        lib.perq_device_error_clear.argtypes = []
        lib.perq_device_error_clear.restype = C.c_int
        lib.perq_status_string.argtypes = [C.c_int]
        lib.perq_status_string.restype = C.c_char_p
        lib.perq_version.restype = C.c_int
        for name in ("perq_rotate_quantize", "perq_rotate_quantize_host", "perq_host_workspace_bytes",
                     "perq_out_sizes", "perq_block_l1_stats", "perq_block_l1_stats_static",
                     "perq_block_l1_stats_workspace_bytes",
                     "perq_token_diagnostics", "perq_validate_perm", "perq_massdiff_perm", "perq_massdiff_perm_device"):
            getattr(lib, name).restype = C.c_int
        _rotate_quantize, _swiglu_rotate_quantize = lib.perq_rotate_quantize, lib.perq_swiglu_rotate_quantize
        _rotate_quantize_i8, _matmul_i8, _grouped_matmul_i8 = lib.perq_rotate_quantize_i8, lib.perq_matmul_i8, lib.perq_grouped_matmul_i8
        _cache_write_i8, _cache_read_i8, _attention_i8 = lib.perq_cache_write_i8, lib.perq_cache_read_i8, lib.perq_attention_i8
        try:
            spec = importlib.util.spec_from_file_location(__package__ + "._perq_call", _build.CALL_PATH)
            call = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(call)
            call.bind(C.cast(lib.perq_rotate_quantize, vp).value, C.cast(lib.perq_swiglu_rotate_quantize, vp).value)
            call.bind_i8(C.cast(lib.perq_rotate_quantize_i8, vp).value, C.cast(lib.perq_matmul_i8, vp).value, C.cast(lib.perq_grouped_matmul_i8, vp).value)
            call.bind_cache(C.cast(lib.perq_cache_write_i8, vp).value, C.cast(lib.perq_cache_read_i8, vp).value, C.cast(lib.perq_attention_i8, vp).value)
            _rotate_quantize, _swiglu_rotate_quantize = call.rotate_quantize, call.swiglu_rotate_quantize
            _rotate_quantize_i8, _matmul_i8, _grouped_matmul_i8 = call.rotate_quantize_i8, call.matmul_i8, call.grouped_matmul_i8
            _cache_write_i8, _cache_read_i8, _attention_i8 = call.cache_write_i8, call.cache_read_i8, call.attention_i8
        except (ImportError, AttributeError):         # (no such file, none that this interpreter can load, or one without these calls)
            pass
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().perq_status_string(int(status)).decode()


def perq_version() -> int:
    return int(load().perq_version())


def _check(rc: int, where: str):
    if rc != PERQ_OK:
        raise PerqError(rc, where)


# Addresses and stream handles go to ctypes as plain integers (the functions' argtypes convert them): small calls
# are bound by the host, and wrapper objects, the torch.cuda.Stream object among them, were a third of its time.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(getattr(stream, "cuda_stream", stream))


def _empty(shape, dtype: torch.dtype, device, stream=None, result: bool = True) -> torch.Tensor:
    """Memory for a call on `stream` (None: the current one).

    It is that stream's: a block that was let go on the current one may be in use by kernels that are still queued there, and the call does not
    wait for them.  Results are noted as in use on the current stream too, where the caller reads them and may let them go."""
    handle = None if stream is None else _stream(stream)
    if handle is None or handle == _stream(None):
        return torch.empty(shape, dtype=dtype, device=device)
    # (0 and 1 are the default stream's, and no handles to make a stream object of)
    with torch.cuda.stream(torch.cuda.default_stream(device) if handle in (0, 1) else torch.cuda.ExternalStream(handle, device)):
        t = torch.empty(shape, dtype=dtype, device=device)
    if result:
        t.record_stream(torch.cuda.current_stream(device))
    return t


def perq_out_sizes(T: int, d: int, fmt: int, group: int):
    cb, sb = C.c_size_t(0), C.c_size_t(0)
    _check(load().perq_out_sizes(T, d, fmt, group, C.byref(cb), C.byref(sb)), "perq_out_sizes")
    return int(cb.value), int(sb.value)


def alloc_outputs(T: int, d: int, fmt: int, group: int, device, stream=None):
    """Device buffers of the right shape for one call on `stream` (torch owns the memory)."""
    if fmt == PERQ_FMT_F32_DEBUG:
        return _empty((T, d), torch.float32, device, stream), None
    codes = _empty((T, d // 2), torch.uint8, device, stream)
    if fmt == PERQ_FMT_FP4:
        scales = _empty((T, 1), torch.float32, device, stream)
    elif fmt == PERQ_FMT_INT4_ASYM:
        scales = _empty((T, 2), torch.float32, device, stream)
    elif fmt == PERQ_FMT_INT4:
        scales = _empty((T, 1 if group == 0 else d // group), torch.float32, device, stream)
    else:
        scales = _empty((T, d // 32), torch.uint8, device, stream)
    return codes, scales


def perq_rotate_quantize(x: torch.Tensor, perm: Optional[torch.Tensor], b: int, fmt: int, group: int = 0,
                         out_codes: Optional[torch.Tensor] = None, out_scales: Optional[torch.Tensor] = None,
                         stream=None):
    """x: bf16 CUDA tensor [T, d] (contiguous); perm: int32 CUDA tensor [d] or None."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_contiguous()
    assert perm is None or (perm.is_cuda and perm.dtype == torch.int32 and perm.is_contiguous())
    T, d = x.shape
    if out_codes is None:
        out_codes, out_scales = alloc_outputs(T, d, fmt, group, x.device, stream)
    if _lib is None:
        load()
    args = (x.data_ptr(), None if perm is None else perm.data_ptr(), T, d, b, fmt, group, _ptr(out_codes), _ptr(out_scales), _stream(stream))
    try:
        rc = _rotate_quantize(*args)
    except TypeError:           # (not plain integers: what ctypes makes of them)
        rc = _lib.perq_rotate_quantize(*args)
    if rc != PERQ_OK:
        _check(rc, "perq_rotate_quantize")
    return out_codes, out_scales


def perq_swiglu_rotate_quantize(gate: torch.Tensor, up: torch.Tensor, perm: Optional[torch.Tensor], b: int, fmt: int,
                                group: int = 0, out_codes: Optional[torch.Tensor] = None,
                                out_scales: Optional[torch.Tensor] = None, stream=None):
    """gate, up: bf16 CUDA tensors [T, d] (contiguous); perm must be None."""
    for t in (gate, up):
        assert t.is_cuda and t.dtype == torch.bfloat16 and t.dim() == 2 and t.is_contiguous()
    assert gate.shape == up.shape
    T, d = gate.shape
    if out_codes is None:
        out_codes, out_scales = alloc_outputs(T, d, fmt, group, gate.device, stream)
    if _lib is None:
        load()
    args = (gate.data_ptr(), up.data_ptr(), _ptr(perm), T, d, b, fmt, group, _ptr(out_codes), _ptr(out_scales), _stream(stream))
    try:
        rc = _swiglu_rotate_quantize(*args)
    except TypeError:           # (as above)
        rc = _lib.perq_swiglu_rotate_quantize(*args)
    _check(rc, "perq_swiglu_rotate_quantize")
    return out_codes, out_scales


def perq_host_workspace_bytes(T: int, d: int, fmt: int, group: int) -> int:
    n = C.c_size_t(0)
    _check(load().perq_host_workspace_bytes(T, d, fmt, group, C.byref(n)), "perq_host_workspace_bytes")
    return int(n.value)


def perq_rotate_quantize_host(x_host: torch.Tensor, perm: Optional[torch.Tensor], b: int, fmt: int, group: int,
                              out_codes_host: torch.Tensor, out_scales_host: Optional[torch.Tensor],
                              workspace: torch.Tensor, stream=None):
    """x_host / outputs: CPU tensors (pinned for asynchronous copies); workspace: CUDA uint8 tensor."""
    assert not x_host.is_cuda and x_host.dtype == torch.bfloat16 and x_host.is_contiguous()
    T, d = x_host.shape
    rc = load().perq_rotate_quantize_host(_ptr(x_host), _ptr(perm), T, d, b, fmt, group, _ptr(out_codes_host),
                                          _ptr(out_scales_host), _ptr(workspace), workspace.numel(),
                                          _stream(stream))
    _check(rc, "perq_rotate_quantize_host")
    return out_codes_host, out_scales_host


def perq_block_l1_stats_workspace_bytes(T: int, d: int, b: int) -> int:
    n = C.c_size_t(0)
    _check(load().perq_block_l1_stats_workspace_bytes(T, d, b, C.byref(n)), "perq_block_l1_stats_workspace_bytes")
    return int(n.value)


def perq_block_l1_stats(x: torch.Tensor, perm: Optional[torch.Tensor], b: int, want=("chan", "block", "token"),
                        workspace: Optional[torch.Tensor] = None, stream=None):
    """Returns (chan_abs_sum[d], block_l1_mean[d/b], token_max_block_l1[T]); entries not in `want` are None."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_contiguous()
    T, d = x.shape
    if workspace is None:
        workspace = _empty(max(16, perq_block_l1_stats_workspace_bytes(T, d, b)), torch.uint8, x.device, stream, result=False)
    chan = _empty(d, torch.float32, x.device, stream) if "chan" in want else None
    block = _empty(d // b, torch.float32, x.device, stream) if "block" in want else None
    token = _empty(T, torch.float32, x.device, stream) if "token" in want else None
    rc = load().perq_block_l1_stats(_ptr(x), _ptr(perm), T, d, b, _ptr(chan), _ptr(block), _ptr(token),
                                    _ptr(workspace), workspace.numel(), _stream(stream))
    _check(rc, "perq_block_l1_stats")
    return chan, block, token


def perq_block_l1_stats_static(x: torch.Tensor, perm: Optional[torch.Tensor], b: int, chan: Optional[torch.Tensor],
                               block: Optional[torch.Tensor], token: Optional[torch.Tensor], stream=None):
    """perq_block_l1_stats with the library's built-in scratch array instead of a workspace.

    The caller passes the output tensors (any may be None); nothing is allocated here or in
    the library.  Shapes whose partial sums do not fit the built-in array raise PerqError
    (status 9).  Calls that may overlap on the GPU must not share a device: they would race
    on the one scratch array."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_contiguous()
    T, d = x.shape
    rc = load().perq_block_l1_stats_static(_ptr(x), _ptr(perm), T, d, b, _ptr(chan), _ptr(block), _ptr(token),
                                           _stream(stream))
    _check(rc, "perq_block_l1_stats_static")
    return chan, block, token


def perq_token_diagnostics(x: torch.Tensor, perm: Optional[torch.Tensor], b: int, out: Optional[torch.Tensor] = None,
                           stream=None) -> torch.Tensor:
    """[T, 5] fp32: ||x||_inf, ||x||_1, largest block l1 under perm, ||y||_inf, ||y - Q(y)||_2 per token."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_contiguous()
    assert perm is None or (perm.is_cuda and perm.dtype == torch.int32 and perm.is_contiguous())
    T, d = x.shape
    if out is None:
        out = _empty((T, 5), torch.float32, x.device, stream)
    _check(load().perq_token_diagnostics(_ptr(x), _ptr(perm), T, d, b, _ptr(out), _stream(stream)),
           "perq_token_diagnostics")
    return out


def perq_validate_perm(perm: torch.Tensor, stream=None) -> torch.Tensor:
    """Returns a 1-element int32 CUDA tensor: 0 valid, bit0 out of range, bit1 duplicate."""
    assert perm.is_cuda and perm.dtype == torch.int32 and perm.is_contiguous()
    status = _empty(1, torch.int32, perm.device, stream)
    _check(load().perq_validate_perm(_ptr(perm), perm.numel(), _ptr(status), _stream(stream)), "perq_validate_perm")
    return status


def perq_device_error() -> int:
    """Device-side error word of the current device (0 = none); synchronises."""
    v = C.c_uint32(0)
    _check(load().perq_device_error(C.byref(v)), "perq_device_error")
    return int(v.value)


def perq_device_error_clear() -> None:
    """Zeroes the device-side error word of the current device; synchronises."""
    _check(load().perq_device_error_clear(), "perq_device_error_clear")


def perq_massdiff_perm_device(chan_abs_sum: torch.Tensor, b: int, perm: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """chan_abs_sum: fp32 CUDA tensor [d]; returns the int32 CUDA permutation [d] (nothing is synchronised)."""
    assert chan_abs_sum.is_cuda and chan_abs_sum.dtype == torch.float32 and chan_abs_sum.is_contiguous()
    d = chan_abs_sum.numel()
    if perm is None:
        perm = _empty(d, torch.int32, chan_abs_sum.device, stream)
    if workspace is None:
        workspace = _empty(d * 4, torch.uint8, chan_abs_sum.device, stream, result=False)
    _check(load().perq_massdiff_perm_device(_ptr(chan_abs_sum), d, b, _ptr(perm), _ptr(workspace),
                                            workspace.numel() * workspace.element_size(), _stream(stream)),
           "perq_massdiff_perm_device")
    return perm


def perq_chan_abs_max(x: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x: bf16 CUDA tensor [T, d]; returns fp32 CUDA tensor [d] (nothing is synchronised)."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.is_contiguous()
    T, d = x.shape
    if out is None:
        out = _empty(d, torch.float32, x.device, stream)
    _check(load().perq_chan_abs_max(_ptr(x), T, d, _ptr(out), _stream(stream)), "perq_chan_abs_max")
    return out


def perq_absmax_perm(chan_abs_max_host: np.ndarray) -> np.ndarray:
    """Host only.  float32 [d] numpy array in, int32 [d] out."""
    a = np.ascontiguousarray(chan_abs_max_host, dtype=np.float32)
    perm = np.empty(a.shape[0], np.int32)
    _check(load().perq_absmax_perm(a.ctypes.data_as(C.c_void_p), a.shape[0], perm.ctypes.data_as(C.c_void_p)), "perq_absmax_perm")
    return perm


def perq_zigzag_perm(chan_abs_max_host: np.ndarray, b: int) -> np.ndarray:
    """Host only.  float32 [d] numpy array in, int32 [d] out."""
    a = np.ascontiguousarray(chan_abs_max_host, dtype=np.float32)
    perm = np.empty(a.shape[0], np.int32)
    _check(load().perq_zigzag_perm(a.ctypes.data_as(C.c_void_p), a.shape[0], b, perm.ctypes.data_as(C.c_void_p)), "perq_zigzag_perm")
    return perm


def perq_massdiff_perm(chan_abs_sum_host: np.ndarray, b: int) -> np.ndarray:
    """Host only.  chan_abs_sum_host: float32 [d] numpy array; returns int32 [d]."""
    a = np.ascontiguousarray(chan_abs_sum_host, dtype=np.float32)
    perm = np.empty(a.shape[0], np.int32)
    rc = load().perq_massdiff_perm(a.ctypes.data_as(C.c_void_p), a.shape[0], b, perm.ctypes.data_as(C.c_void_p))
    _check(rc, "perq_massdiff_perm")
    return perm


# Small calls of these are bound by the host (one row of 4096: 2.6 us in the library, 2.1 for each tensor made here, 0.06 for each
# attribute asked), so the device is asked for once and a tensor's place, type and layout once each.
def _on(t: torch.Tensor, device: int, dtype: torch.dtype) -> bool:
    """A contiguous tensor of that type on that CUDA device."""
    return t.get_device() == device and t.dtype is dtype and t.is_contiguous()


def perq_rotate_quantize_i8(x: torch.Tensor, perm: Optional[torch.Tensor], b: int, out_codes: Optional[torch.Tensor] = None,
                            out_scales: Optional[torch.Tensor] = None, stream=None):
    """x: bf16 CUDA tensor [T, d] (contiguous); perm: int32 CUDA tensor [d] or None.  Returns (int8 [T, d], fp32 [T, 1]).

    All tensors are on the current device."""
    device = torch._C._cuda_getDevice()
    assert x.get_device() == device and x.dtype is torch.bfloat16 and x.is_contiguous()
    T, d = x.shape
    assert perm is None or (_on(perm, device, torch.int32) and perm.numel() == d)
    if out_codes is None:
        out_codes = x.new_empty((T, d), dtype=torch.int8) if stream is None else _empty((T, d), torch.int8, x.device, stream)
    else:
        assert _on(out_codes, device, torch.int8) and out_codes.numel() == T * d
    if out_scales is None:
        out_scales = x.new_empty((T, 1), dtype=torch.float32) if stream is None else _empty((T, 1), torch.float32, x.device, stream)
    else:
        assert _on(out_scales, device, torch.float32) and out_scales.numel() == T
    if _lib is None:
        load()
    args = (x.data_ptr(), None if perm is None else perm.data_ptr(), T, d, b, out_codes.data_ptr(), out_scales.data_ptr(),
            torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream))
    try:
        rc = _rotate_quantize_i8(*args)
    except TypeError:           # (not plain integers: what ctypes makes of them)
        rc = _lib.perq_rotate_quantize_i8(*args)
    if rc != PERQ_OK:
        _check(rc, "perq_rotate_quantize_i8")
    return out_codes, out_scales


def perq_code_sums(codes: torch.Tensor, fmt: int, stream=None) -> torch.Tensor:
    """Sums of the rows of codes (int8 [.., d], or uint8 [.., d / 2] for INT4): int32 CUDA tensor [..]."""
    assert _on(codes, torch._C._cuda_getDevice(), torch.int8 if fmt == PERQ_FMT_INT8 else torch.uint8)
    d = codes.shape[-1] * (1 if fmt == PERQ_FMT_INT8 else 2)
    sums = _empty(codes.shape[:-1], torch.int32, codes.device, stream)
    _check(load().perq_code_sums(_ptr(codes), fmt, sums.numel(), d, _ptr(sums), _stream(stream)), "perq_code_sums")
    return sums


def perq_matmul_i8_workspace_bytes(T: int, N: int, d: int, a_fmt: int, w_fmt: int) -> int:
    n = C.c_size_t(0)
    _check(load().perq_matmul_i8_workspace_bytes(T, N, d, a_fmt, w_fmt, C.byref(n)), "perq_matmul_i8_workspace_bytes")
    return int(n.value)


def perq_grouped_matmul_i8_workspace_bytes(T: int, E: int, N: int, d: int, a_fmt: int, w_fmt: int) -> int:
    n = C.c_size_t(0)
    _check(load().perq_grouped_matmul_i8_workspace_bytes(T, E, N, d, a_fmt, w_fmt, C.byref(n)), "perq_grouped_matmul_i8_workspace_bytes")
    return int(n.value)


# (a workspace is asked for only where the call wants one: few do)
def _product(a_codes, a_scales, a_fmt, w_codes, w_scales, w_fmt, w_sums, offsets, E, N, out, out_dtype, workspace, stream):
    device, f32 = torch._C._cuda_getDevice(), torch.float32
    T, d = a_codes.shape
    assert a_codes.get_device() == device and a_codes.dtype is (torch.int8 if a_fmt == PERQ_FMT_INT8 else torch.uint8) and a_codes.is_contiguous()
    assert w_codes.get_device() == device and w_codes.dtype is (torch.int8 if w_fmt == PERQ_FMT_INT8 else torch.uint8) and w_codes.is_contiguous()
    assert a_scales.get_device() == device and a_scales.dtype is f32 and a_scales.is_contiguous()
    assert w_scales.get_device() == device and w_scales.dtype is f32 and w_scales.is_contiguous()
    assert a_scales.numel() == (2 * T if a_fmt == PERQ_FMT_INT4_ASYM else T) and w_scales.numel() == E * N
    if a_fmt != PERQ_FMT_INT8:
        d *= 2
    assert w_codes.shape[-1] == (d if w_fmt == PERQ_FMT_INT8 else d // 2)
    assert w_sums is None or (_on(w_sums, device, torch.int32) and w_sums.numel() == E * N)
    if out is None:
        out = a_scales.new_empty((T, N), dtype=out_dtype) if stream is None else _empty((T, N), out_dtype, a_scales.device, stream)
    else:
        out_dtype = out.dtype
        assert out.get_device() == device and out.is_contiguous() and out.shape == (T, N)
    assert workspace is None or (workspace.get_device() == device and workspace.is_contiguous())
    if _lib is None:
        load()
    handle = torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)
    while True:
        sums = None if w_sums is None else w_sums.data_ptr()
        space, room = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
        if offsets is None:
            call, plain = _matmul_i8, _lib.perq_matmul_i8
            args = (a_codes.data_ptr(), a_scales.data_ptr(), a_fmt, w_codes.data_ptr(), w_scales.data_ptr(), w_fmt, sums, T, N, d, out.data_ptr(),
                    OUT_BY_DTYPE[out_dtype], space, room, handle)
        else:
            assert _on(offsets, device, torch.int32)
            call, plain = _grouped_matmul_i8, _lib.perq_grouped_matmul_i8
            args = (a_codes.data_ptr(), a_scales.data_ptr(), a_fmt, w_codes.data_ptr(), w_scales.data_ptr(), w_fmt, sums, offsets.data_ptr(), T, E, N, d,
                    out.data_ptr(), OUT_BY_DTYPE[out_dtype], space, room, handle)
        try:
            rc = call(*args)
        except TypeError:       # (as above)
            rc = plain(*args)
        if rc == PERQ_OK:
            return out
        if rc != PERQ_ERR_WORKSPACE or workspace is not None:
            _check(rc, "perq_matmul_i8" if offsets is None else "perq_grouped_matmul_i8")
        n = (perq_matmul_i8_workspace_bytes(T, N, d, a_fmt, w_fmt) if offsets is None else
             perq_grouped_matmul_i8_workspace_bytes(T, E, N, d, a_fmt, w_fmt))
        workspace = _empty(n, torch.uint8, a_codes.device, stream, result=False)       # (let go on return)


def perq_matmul_i8(a_codes: torch.Tensor, a_scales: torch.Tensor, a_fmt: int, w_codes: torch.Tensor, w_scales: torch.Tensor, w_fmt: int,
                   w_sums: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """a: codes [T, d] of tokens, w: codes [N, d] of weight channels (int8, or uint8 [.., d / 2] for INT4); returns out [T, N].

    All tensors are on the current device.  A workspace that the call wants and is not given is made here."""
    N, _ = w_codes.shape
    return _product(a_codes, a_scales, a_fmt, w_codes, w_scales, w_fmt, w_sums, None, 1, N, out, out_dtype, workspace, stream)


def perq_grouped_matmul_i8(a_codes: torch.Tensor, a_scales: torch.Tensor, a_fmt: int, w_codes: torch.Tensor, w_scales: torch.Tensor, w_fmt: int,
                           offsets: torch.Tensor, w_sums: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                           out_dtype: torch.dtype = torch.bfloat16, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """As perq_matmul_i8 with w [E, N, d] and rows offsets[e] .. offsets[e + 1] (int32 CUDA tensor [E + 1]) of the tokens for expert e.

    Rows of no expert are not written: in an `out` made here they are whatever its memory holds."""
    E, N, _ = w_codes.shape
    assert offsets.numel() == E + 1
    return _product(a_codes, a_scales, a_fmt, w_codes, w_scales, w_fmt, w_sums, offsets, E, N, out, out_dtype, workspace, stream)


# ------------------------------------------------------------------------------------------------- the 8-bit cache
# Numbers that the library takes as 32 bits: larger ones would be cut (2 ** 32 + 1 rows to 1), so they are refused here.
def _fit(where: str, rc: int, *numbers) -> None:
    for n in numbers:
        if not -0x80000000 <= n <= 0x7fffffff:
            raise PerqError(rc, where)


def _cache(device, k_codes, k_steps, v_codes, v_steps, offsets, lengths, pages):
    """The cache's sizes: (S, heads, D, page, n_pages, width)."""
    i8, i32, f32 = torch.int8, torch.int32, torch.float32
    assert k_codes.get_device() == device and k_codes.dtype is i8 and k_codes.is_contiguous() and v_codes.get_device() == device and v_codes.dtype is i8 and v_codes.is_contiguous()
    assert k_steps.get_device() == device and k_steps.dtype is f32 and k_steps.is_contiguous() and v_steps.get_device() == device and v_steps.dtype is f32 and v_steps.is_contiguous()
    assert offsets.get_device() == device and offsets.dtype is i32 and offsets.is_contiguous() and lengths.get_device() == device and lengths.dtype is i32 and lengths.is_contiguous()
    assert pages.get_device() == device and pages.dtype is i32 and pages.is_contiguous()
    n_pages, heads, page, D = shape = k_codes.shape
    S, width = pages.shape
    assert v_codes.shape == shape and k_steps.numel() == n_pages * heads == v_steps.numel() and lengths.numel() == S and offsets.numel() == S + 1
    return S, heads, D, page, n_pages, width


# Rows of tokens [T, heads, D] whose heads lie side by side, bf16 or f16; they may be parts of longer rows, so tokens are some elements apart.
def _row_stride(x: torch.Tensor, device: int) -> int:
    assert x.get_device() == device and (x.dtype is torch.bfloat16 or x.dtype is torch.float16)
    T, heads, D = x.shape
    stride = x.stride()
    assert heads == 1 or stride[1] == D and stride[2] == 1 or x.is_contiguous()
    assert stride[2] == 1 or x.is_contiguous()
    return stride[0] if T > 1 and not x.is_contiguous() else heads * D             # (a single row's may be anything)


def perq_cache_write_i8(k: torch.Tensor, v: torch.Tensor, k_codes: torch.Tensor, k_steps: torch.Tensor, v_codes: torch.Tensor, v_steps: torch.Tensor,
                        offsets: torch.Tensor, lengths: torch.Tensor, pages: torch.Tensor, b: int = 1, stream=None) -> None:
    """k, v: bf16 or f16 CUDA tensors [T, heads, D] (parts of longer rows too), written into codes int8 [n_pages, heads, page, D] and steps fp32 [n_pages, heads].

    offsets int32 [S + 1], lengths int32 [S] (tokens with the new ones), pages int32 [S, width].  All tensors are on the current device."""
    _fit("perq_cache_write_i8", PERQ_ERR_BLOCK, b)
    device = torch._C._cuda_getDevice()
    S, heads, D, page, n_pages, width = _cache(device, k_codes, k_steps, v_codes, v_steps, offsets, lengths, pages)
    T = k.shape[0]
    assert k.dtype is v.dtype and k.shape == (T, heads, D) == v.shape
    k_stride, v_stride = _row_stride(k, device), _row_stride(v, device)
    if _lib is None:
        load()
    args = (k.data_ptr(), v.data_ptr(), OUT_BY_DTYPE[k.dtype], k_stride, v_stride, offsets.data_ptr(), lengths.data_ptr(), pages.data_ptr(), T, S, heads, D, b, page,
            n_pages, width, k_codes.data_ptr(), k_steps.data_ptr(), v_codes.data_ptr(), v_steps.data_ptr(),
            torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream))
    try:
        rc = _cache_write_i8(*args)
    except TypeError:           # (not plain integers: what ctypes makes of them)
        rc = _lib.perq_cache_write_i8(*args)
    if rc != PERQ_OK:
        _check(rc, "perq_cache_write_i8")


def perq_cache_read_i8(k_codes: torch.Tensor, k_steps: torch.Tensor, v_codes: torch.Tensor, v_steps: torch.Tensor, offsets: torch.Tensor, lengths: torch.Tensor,
                       pages: torch.Tensor, T: int, b: int = 1, out_dtype: torch.dtype = torch.bfloat16, k: Optional[torch.Tensor] = None,
                       v: Optional[torch.Tensor] = None, stream=None):
    """The last offsets[i + 1] - offsets[i] tokens of every sequence: (k, v), each [T, heads, D] of out_dtype.

    Rows of no sequence are not written: in outputs made here they are whatever the memory holds."""
    _fit("perq_cache_read_i8", PERQ_ERR_BLOCK, b)
    device = torch._C._cuda_getDevice()
    S, heads, D, page, n_pages, width = _cache(device, k_codes, k_steps, v_codes, v_steps, offsets, lengths, pages)
    shape = (T, heads, D)
    if k is None:
        k = k_codes.new_empty(shape, dtype=out_dtype) if stream is None else _empty(shape, out_dtype, k_codes.device, stream)
    if v is None:
        v = k_codes.new_empty(shape, dtype=k.dtype) if stream is None else _empty(shape, k.dtype, k_codes.device, stream)
    assert k.get_device() == device and k.is_contiguous() and k.shape == shape and _on(v, device, k.dtype) and v.shape == shape
    if _lib is None:
        load()
    args = (k_codes.data_ptr(), k_steps.data_ptr(), v_codes.data_ptr(), v_steps.data_ptr(), offsets.data_ptr(), lengths.data_ptr(), pages.data_ptr(), T, S, heads, D, b, page,
            n_pages, width, k.data_ptr(), v.data_ptr(), OUT_BY_DTYPE[k.dtype], torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream))
    try:
        rc = _cache_read_i8(*args)
    except TypeError:           # (as above)
        rc = _lib.perq_cache_read_i8(*args)
    if rc != PERQ_OK:
        _check(rc, "perq_cache_read_i8")
    return k, v


def perq_attention_i8_workspace_bytes(T: int, S: int, heads: int, group: int, D: int, most: int) -> int:
    _fit("perq_attention_i8_workspace_bytes", PERQ_ERR_SHAPE, S, heads, group, D, most)
    n = C.c_size_t(0)
    _check(load().perq_attention_i8_workspace_bytes(T, S, heads, group, D, most, C.byref(n)), "perq_attention_i8_workspace_bytes")
    return int(n.value)


# (asked once for the sizes of a device: it takes 1.7 us, and small calls are bound by the host)
@functools.lru_cache(maxsize=1024)
def _attention_space(device: int, T: int, S: int, heads: int, group: int, D: int, most: int) -> int:
    return max(16, perq_attention_i8_workspace_bytes(T, S, heads, group, D, most))


def perq_attention_i8(q: torch.Tensor, k_codes: torch.Tensor, k_steps: torch.Tensor, v_codes: torch.Tensor, v_steps: torch.Tensor, offsets: torch.Tensor,
                      lengths: torch.Tensor, pages: torch.Tensor, most: Optional[int] = None, b: int = 1, scale: Optional[float] = None, window: int = 0,
                      sinks: int = 0, out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """q: bf16 or f16 CUDA tensor [T, heads of queries, D] (part of longer rows too); returns out [T, heads of queries, D] of q's type, or out_dtype.

    most: at least the rows of the longest sequence of the call (None: T); scale: of the logits (None: D ** -0.5).  All tensors are on the current device.  A
    workspace that the call is not given is made here.  Rows of no sequence are not written: in an `out` made here they are whatever its memory holds."""
    _fit("perq_attention_i8", PERQ_ERR_SHAPE, 1 if most is None else most, window, sinks)
    _fit("perq_attention_i8", PERQ_ERR_BLOCK, b)
    device = torch._C._cuda_getDevice()
    S, heads, D, page, n_pages, width = _cache(device, k_codes, k_steps, v_codes, v_steps, offsets, lengths, pages)
    shape = q.shape
    T, all_heads, channels = shape
    assert channels == D and all_heads % heads == 0
    q_stride, group = _row_stride(q, device), all_heads // heads
    if out is None:
        out = q.new_empty(shape, dtype=out_dtype) if stream is None else _empty(shape, out_dtype or q.dtype, q.device, stream)
    else:
        assert out.get_device() == device and out.is_contiguous() and out.shape == shape
    if most is None:
        most = T or 1
    if _lib is None:
        load()
    if workspace is None:
        n = _attention_space(device, T, S, heads, group, D, most)
        workspace = k_codes.new_empty(n) if stream is None else _empty(n, torch.uint8, q.device, stream, result=False)       # (let go on return)
    else:
        assert workspace.get_device() == device and workspace.is_contiguous()
        n = workspace.numel() * workspace.element_size()
    args = (q.data_ptr(), OUT_BY_DTYPE[q.dtype], q_stride, k_codes.data_ptr(), k_steps.data_ptr(), v_codes.data_ptr(), v_steps.data_ptr(), offsets.data_ptr(), lengths.data_ptr(),
            pages.data_ptr(), T, S, heads, group, D, b, page, n_pages, width, most, D ** -0.5 if scale is None else scale, window, sinks, out.data_ptr(), OUT_BY_DTYPE[out.dtype],
            workspace.data_ptr(), n, torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream))
    try:
        rc = _attention_i8(*args)
    except TypeError:           # (as above)
        rc = _lib.perq_attention_i8(*args)
    if rc != PERQ_OK:
        _check(rc, "perq_attention_i8")
    return out
