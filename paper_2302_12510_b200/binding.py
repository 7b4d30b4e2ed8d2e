"""ctypes binding of libdybit.so: argument marshalling only.

Function names follow include/dybit.h.  torch supplies device memory and the
current stream; every computation happens inside the library's kernels.
There is no fallback: if libdybit.so is absent the import fails.

Every device call takes `stream` (a torch stream or a stream's handle; default:
the current stream).  What it allocates itself belongs to that stream.  What it
is given follows torch's own rule: the stream has to wait for whatever filled
it, and a tensor of another stream's that is dropped before the call has run
needs record_stream.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple, Optional, Tuple

import torch

from . import _build

__all__ = [
    "Fmt", "ConvDesc", "DybitError", "lib", "CONTAINER_NAMES",
    "dybit_status_string", "dybit_packed_bytes", "dybit_row_stride_bytes", "dybit_decode_table",
    "dybit_choose_container", "dybit_gemm_workspace_bytes", "dybit_conv2d_workspace_bytes",
    "dybit_conv2d_out_hw", "dybit_absmax_scale", "dybit_quantize_pack", "dybit_quantize_pack_2d",
    "dybit_decode", "dybit_gemm", "dybit_conv2d", "dybit_last_device_status",
    "dybit_launch_count", "dybit_set_conv_lowering", "dybit_set_gemm_decode", "dybit_selftest_wait_timeout", "dybit_profile_next_gemm", "dybit_profile_next_gemm_clock", "dybit_gemm_static_ws", "STATIC_WS_BYTES",
    "dybit_gemm_requant", "dybit_conv2d_requant", "dybit_depthwise_conv2d", "dybit_gemm_batched",
    "dybit_quantize_conv2d", "dybit_quantize_conv2d_requant",
    "ConvLayers", "dybit_quantize_expand_layers", "dybit_conv2d_prepared", "dybit_conv2d_prepared_layers",
    "dybit_gemm_batched_workspace_bytes", "dybit_rmse", "dybit_rmse_sweep", "dybit_fake_quant", "dybit_fake_quant_backward",
    "dybit_search_bitwidths",
    "dybit_checkpoint_save", "dybit_checkpoint_load", "dybit_checkpoint_wgrad", "dybit_checkpoint_wgrad_workspace_bytes",
    "AdapterPlan", "dybit_adapters_plan", "dybit_adapters_plan_bytes", "dybit_adapters", "dybit_adapters_backward",
    "dybit_adapters_backward_workspace_bytes",
    "KVCache", "CachePlan", "dybit_cache_plan", "dybit_cache_plan_bytes", "dybit_cache_write", "dybit_cache_read", "dybit_cache_attention",
    "dybit_cache_attention_workspace_bytes",
]


class Fmt(NamedTuple):
    bits: int
    is_signed: bool


class _CFmt(C.Structure):
    _fields_ = [("bits", C.c_int), ("is_signed", C.c_int)]


class _CConvDesc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n", "h", "w", "c", "k", "r", "s", "stride", "pad", "dilation")]


class _CConvLayer(C.Structure):
    _fields_ = [("desc", _CConvDesc), ("X", C.c_void_p), ("fx", _CFmt), ("scale_x", C.c_void_p),
                ("scale_x_out", C.c_void_p), ("X_packed", C.c_void_p), ("W", C.c_void_p), ("fw", _CFmt),
                ("scale_w", C.c_void_p), ("ldw_bytes", C.c_int64), ("Y", C.c_void_p), ("Y_raw", C.c_void_p),
                ("ws", C.c_void_p), ("ws_bytes", C.c_size_t), ("Q", C.c_void_p), ("fq", _CFmt),
                ("scale_q", C.c_void_p), ("bias", C.c_void_p), ("relu", C.c_int)]


class _CCache(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p),
                ("pages", C.c_int64), ("page", C.c_int), ("heads", C.c_int), ("dim", C.c_int)]


class _CCacheBatch(C.Structure):
    _fields_ = [("sequences", C.c_int), ("tokens", C.c_int64), ("max_new", C.c_int), ("q_heads", C.c_int), ("table", C.c_void_p),
                ("table_stride", C.c_int64), ("max_pages", C.c_int), ("causal", C.c_int), ("window", C.c_int)]


class ConvDesc(NamedTuple):
    n: int
    h: int
    w: int
    c: int
    k: int
    r: int
    s: int
    stride: int = 1
    pad: int = 0
    dilation: int = 1


class DybitError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {dybit_status_string(status)} (status {status})")


CONTAINER_NAMES = {0: "int8", 1: "e4m3", 2: "bf16"}


def _load() -> C.CDLL:
    # DYBIT_LIBRARY=debug selects the range-checked build (libdybit_debug.so); anything else is the product library
    path = _build.DEBUG_LIB_PATH if os.environ.get("DYBIT_LIBRARY", "") == "debug" else _build.LIB_PATH
    if not os.path.exists(path):
        raise ImportError(
            f"{path} is missing: build it with `python -m paper_2302_12510_b200._build` "
            "(there is no CPU or PyTorch fallback)")
    lib = C.CDLL(path)
    i64, i32, sz, vp = C.c_int64, C.c_int, C.c_size_t, C.c_void_p
    lib.dybit_status_string.restype = C.c_char_p
    lib.dybit_status_string.argtypes = [i32]
    lib.dybit_packed_bytes.restype = sz
    lib.dybit_packed_bytes.argtypes = [i64, i32]
    lib.dybit_row_stride_bytes.restype = sz
    lib.dybit_row_stride_bytes.argtypes = [i64, i32]
    lib.dybit_decode_table.argtypes = [_CFmt, C.POINTER(C.c_float)]
    lib.dybit_choose_container.argtypes = [_CFmt, _CFmt, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)]
    lib.dybit_gemm_workspace_bytes.restype = sz
    lib.dybit_gemm_workspace_bytes.argtypes = [i64, i64, i64, _CFmt, _CFmt]
    lib.dybit_conv2d_workspace_bytes.restype = sz
    lib.dybit_conv2d_workspace_bytes.argtypes = [C.POINTER(_CConvDesc), _CFmt, _CFmt]
    lib.dybit_conv2d_out_hw.argtypes = [C.POINTER(_CConvDesc), C.POINTER(i32), C.POINTER(i32)]
    lib.dybit_absmax_scale.argtypes = [vp, i64, _CFmt, vp, vp]
    lib.dybit_quantize_pack.argtypes = [vp, i64, _CFmt, vp, vp, vp, vp]
    lib.dybit_quantize_pack_2d.argtypes = [vp, i64, i64, i64, _CFmt, vp, vp, i64, vp, vp]
    lib.dybit_decode.argtypes = [vp, i64, _CFmt, vp, vp, vp]
    lib.dybit_gemm.argtypes = [i64, i64, i64, vp, _CFmt, vp, i64, vp, _CFmt, vp, i64,
                               vp, i64, vp, vp, sz, vp]
    lib.dybit_conv2d.argtypes = [C.POINTER(_CConvDesc), vp, _CFmt, vp, vp, _CFmt, vp, i64,
                                 vp, vp, vp, sz, vp]
    lib.dybit_last_device_status.argtypes = [vp, C.POINTER(C.c_uint32)]
    lib.dybit_launch_count.restype = C.c_uint64
    lib.dybit_launch_count.argtypes = []
    lib.dybit_set_conv_lowering.argtypes = [i32]
    lib.dybit_set_gemm_decode.argtypes = [i32]
    lib.dybit_selftest_wait_timeout.argtypes = [C.c_uint64, vp, vp]
    lib.dybit_profile_next_gemm.argtypes = [vp, vp]
    lib.dybit_profile_next_gemm_clock.argtypes = [vp]
    lib.dybit_gemm_requant.argtypes = [i64, i64, i64, vp, _CFmt, vp, i64, vp, _CFmt, vp, i64,
                                       _CFmt, vp, vp, i32, vp, i64, vp, sz, vp]
    lib.dybit_conv2d_requant.argtypes = [C.POINTER(_CConvDesc), vp, _CFmt, vp, vp, _CFmt, vp, i64,
                                         _CFmt, vp, vp, i32, vp, vp, sz, vp]
    lib.dybit_quantize_conv2d_requant.argtypes = [C.POINTER(_CConvDesc), vp, _CFmt, vp, vp, vp, vp, _CFmt, vp, i64,
                                                  _CFmt, vp, vp, i32, vp, vp, sz, vp]
    lib.dybit_rmse.argtypes = [vp, i64, _CFmt, vp, vp, vp]
    lib.dybit_quantize_conv2d.argtypes = [C.POINTER(_CConvDesc), vp, _CFmt, vp, vp, vp, vp, _CFmt, vp, i64,
                                          vp, vp, vp, sz, vp]
    lib.dybit_quantize_expand_layers.argtypes = [C.POINTER(_CConvLayer), i32, vp]
    lib.dybit_conv2d_prepared.argtypes = [C.POINTER(_CConvLayer), vp]
    lib.dybit_conv2d_prepared_layers.argtypes = [C.POINTER(_CConvLayer), i32, vp]
    lib.dybit_gemm_batched_workspace_bytes.restype = sz
    lib.dybit_gemm_batched_workspace_bytes.argtypes = [i64, i64, i64, i64, _CFmt, _CFmt]
    lib.dybit_gemm_batched.argtypes = [i64, i64, i64, i64, vp, _CFmt, vp, i64, i64, vp, _CFmt, vp, i64, i64,
                                       vp, i64, i64, vp, vp, sz, vp]
    lib.dybit_depthwise_conv2d.argtypes = [C.POINTER(_CConvDesc), vp, _CFmt, vp, vp, _CFmt, vp, i64, vp, vp]
    lib.dybit_rmse_sweep.argtypes = [vp, i64, i32, C.POINTER(_CFmt), vp, vp, vp, vp]
    lib.dybit_fake_quant.argtypes = [vp, i64, _CFmt, vp, vp, vp]
    lib.dybit_fake_quant_backward.argtypes = [vp, vp, i64, _CFmt, vp, vp, vp]
    lib.dybit_search_bitwidths.argtypes = [i32, C.POINTER(C.c_double), C.POINTER(C.c_double), i32, C.c_double, i32,
                                           C.POINTER(i32), C.POINTER(i32)]
    lib.dybit_checkpoint_save.argtypes = [vp, i32, i64, i64, i64, _CFmt, i32, vp, i64, vp, vp]
    lib.dybit_checkpoint_load.argtypes = [vp, i64, vp, i64, i64, i64, _CFmt, vp, i32, i64, vp]
    lib.dybit_checkpoint_wgrad_workspace_bytes.restype = sz
    lib.dybit_checkpoint_wgrad_workspace_bytes.argtypes = [i64, i64, i64, i32]
    lib.dybit_checkpoint_wgrad.argtypes = [i64, i64, i64, vp, i32, i64, vp, i64, _CFmt, vp, i64, vp, i64, vp, sz, vp]
    lib.dybit_adapters_plan_bytes.restype = sz
    lib.dybit_adapters_plan_bytes.argtypes = [i64, i32]
    lib.dybit_adapters_plan.argtypes = [i64, vp, i32, vp, sz, vp]
    lib.dybit_adapters.argtypes = [i64, i64, i64, i32, vp, i32, i64, i32, vp, vp, i32, vp, vp, vp, i64, i32, vp, i64, vp, vp]
    lib.dybit_adapters_backward_workspace_bytes.restype = sz
    lib.dybit_adapters_backward_workspace_bytes.argtypes = [i64, i64, i64, i32, i32]
    lib.dybit_adapters_backward.argtypes = [i64, i64, i64, i32, vp, i32, i64, vp, i64, _CFmt, vp, i64, i32, vp, vp, i32,
                                            vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp]
    cache, batch = C.POINTER(_CCache), C.POINTER(_CCacheBatch)
    lib.dybit_cache_plan_bytes.restype = sz
    lib.dybit_cache_plan_bytes.argtypes = [cache, batch]
    lib.dybit_cache_plan.argtypes = [cache, batch, vp, vp, vp, sz, vp]
    lib.dybit_cache_write.argtypes = [cache, batch, vp, vp, i64, i64, vp, i64, i64, i32, i32, vp]
    lib.dybit_cache_read.argtypes = [cache, batch, vp, vp, i64, i64, vp, i64, i64, i32, vp]
    lib.dybit_cache_attention_workspace_bytes.restype = sz
    lib.dybit_cache_attention_workspace_bytes.argtypes = [cache, batch]
    lib.dybit_cache_attention.argtypes = [cache, batch, vp, vp, i32, i64, i64, vp, i64, i64, vp, C.c_float, i32, i32, vp, sz, vp]
    lib.dybit_gemm_static_ws.argtypes = [i64, i64, i64, vp, _CFmt, vp, i64, vp, _CFmt, vp, i64, vp, i64, vp, vp]
    return lib


lib = _load()


_FMT_CACHE = {}


def _fmt(f) -> _CFmt:
    bits, sg = f
    key = (int(bits), bool(sg))
    c = _FMT_CACHE.get(key)
    if c is None:
        c = _FMT_CACHE[key] = _CFmt(key[0], int(key[1]))
    return c


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


_raw_stream, _raw_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _raw_device is not None:      # 0.2 us where torch.cuda.current_stream() takes 3
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _check(status: int, where: str):
    if status != 0:
        raise DybitError(status, where)


def _torch_stream(stream, device) -> torch.cuda.Stream:
    """The torch stream of a call's `stream` argument: a torch stream, or the handle of one (0: the default stream)."""
    if isinstance(stream, torch.cuda.Stream):
        return stream
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    return torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)


def _new(like: torch.Tensor, shape, dtype: torch.dtype, stream, zero: bool = False, returned: bool = True) -> torch.Tensor:
    """A tensor that a call allocates on the device of `like`.  It belongs to the stream that the call runs on, so its memory
    is neither still in use by earlier work of another stream nor handed on before that stream is done with it.  One that
    is returned stays alive for the work that the caller's current stream does with it, too."""
    make = like.new_zeros if zero else like.new_empty
    if stream is None:
        return make(shape, dtype=dtype)
    s, current = _torch_stream(stream, like.device), torch.cuda.current_stream(like.device)
    if s == current:
        return make(shape, dtype=dtype)
    with torch.cuda.stream(s):
        t = make(shape, dtype=dtype)
    if returned:
        t.record_stream(current)
    return t


def _ws_span(ws: torch.Tensor, like: torch.Tensor) -> Tuple[int, int]:
    """(address, bytes) of the part of a workspace from its first 1024-byte boundary on; 0 bytes where it ends before."""
    if not (ws.is_cuda and ws.device == like.device and ws.is_contiguous()):
        raise ValueError("ws must be a contiguous CUDA tensor on the device of the operands")
    at = ws.data_ptr()
    off = -at % 1024
    return at + off, max(0, ws.numel() * ws.element_size() - off)


def _workspace(need: int, ws: Optional[torch.Tensor], like: torch.Tensor, stream=None):
    """(address, bytes, tensor to keep) of a 1024-byte aligned workspace on the device of `like`."""
    if ws is None:
        ws = _new(like, need + 1024, torch.uint8, stream, returned=False)
        at = ws.data_ptr()
        return at + -at % 1024, need + 1024 - -at % 1024, ws
    return (*_ws_span(ws, like), ws)


def _dev_f32(x: torch.Tensor, name: str) -> torch.Tensor:
    if not (x.is_cuda and x.dtype == torch.float32 and x.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous float32 CUDA tensor")
    return x


# ---------------------------------------------------------------- host helpers

def dybit_status_string(status: int) -> str:
    return lib.dybit_status_string(int(status)).decode()


def dybit_packed_bytes(n: int, bits: int) -> int:
    return int(lib.dybit_packed_bytes(int(n), int(bits)))


def dybit_row_stride_bytes(k: int, bits: int) -> int:
    return int(lib.dybit_row_stride_bytes(int(k), int(bits)))


def dybit_decode_table(fmt) -> list:
    buf = (C.c_float * 256)()
    _check(lib.dybit_decode_table(_fmt(fmt), buf), "dybit_decode_table")
    return list(buf)


def dybit_choose_container(fa, fb) -> Tuple[int, int, int]:
    c, ea, eb = C.c_int(-1), C.c_int(0), C.c_int(0)
    _check(lib.dybit_choose_container(_fmt(fa), _fmt(fb), C.byref(c), C.byref(ea), C.byref(eb)),
           "dybit_choose_container")
    return c.value, ea.value, eb.value


def dybit_gemm_workspace_bytes(M: int, N: int, K: int, fa, fb) -> int:
    return int(lib.dybit_gemm_workspace_bytes(int(M), int(N), int(K), _fmt(fa), _fmt(fb)))


def _cdesc(d: ConvDesc) -> _CConvDesc:
    return _CConvDesc(*[int(v) for v in d])


def dybit_conv2d_workspace_bytes(desc: ConvDesc, fx, fw) -> int:
    cd = _cdesc(desc)
    return int(lib.dybit_conv2d_workspace_bytes(C.byref(cd), _fmt(fx), _fmt(fw)))


def dybit_conv2d_out_hw(desc: ConvDesc) -> Tuple[int, int]:
    cd = _cdesc(desc)
    oh, ow = C.c_int(0), C.c_int(0)
    _check(lib.dybit_conv2d_out_hw(C.byref(cd), C.byref(oh), C.byref(ow)), "dybit_conv2d_out_hw")
    return oh.value, ow.value


# ---------------------------------------------------------------- device entry points

def dybit_absmax_scale(x: torch.Tensor, fmt, scale_out: Optional[torch.Tensor] = None, stream=None):
    _dev_f32(x, "x")
    if scale_out is None:
        scale_out = _new(x, 2, torch.float32, stream)
    _check(lib.dybit_absmax_scale(_ptr(x), x.numel(), _fmt(fmt), _ptr(scale_out), _stream(stream)),
           "dybit_absmax_scale")
    return scale_out


def dybit_quantize_pack(x: torch.Tensor, fmt, scale: Optional[torch.Tensor] = None,
                        packed: Optional[torch.Tensor] = None,
                        scale_out: Optional[torch.Tensor] = None, stream=None):
    """Returns (packed uint8 tensor, scale tensor {scale, 1/scale})."""
    _dev_f32(x, "x")
    n = x.numel()
    if packed is None:
        packed = _new(x, dybit_packed_bytes(n, fmt[0]), torch.uint8, stream)
    if scale is None and scale_out is None:
        scale_out = _new(x, 2, torch.float32, stream)
    _check(lib.dybit_quantize_pack(_ptr(x), n, _fmt(fmt), _ptr(scale), _ptr(packed), _ptr(scale_out),
                                   _stream(stream)), "dybit_quantize_pack")
    return packed, (scale if scale is not None else scale_out)


def dybit_quantize_pack_2d(x: torch.Tensor, fmt, scale: Optional[torch.Tensor] = None,
                           packed: Optional[torch.Tensor] = None, row_stride_bytes: Optional[int] = None,
                           scale_out: Optional[torch.Tensor] = None, ld: Optional[int] = None,
                           cols: Optional[int] = None, stream=None):
    """x: [rows][ld] float32 (cols <= ld used).  Returns (packed [rows][row_stride] uint8, scale)."""
    if not (x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1):
        raise ValueError("x must be a 2-D float32 CUDA tensor with unit inner stride")
    rows = x.shape[0]
    cols = x.shape[1] if cols is None else cols
    ld = x.stride(0) if ld is None else ld
    if row_stride_bytes is None:
        row_stride_bytes = dybit_row_stride_bytes(cols, fmt[0])
    if packed is None:
        packed = _new(x, (rows, row_stride_bytes), torch.uint8, stream)
    if scale is None and scale_out is None:
        scale_out = _new(x, 2, torch.float32, stream)
    _check(lib.dybit_quantize_pack_2d(_ptr(x), rows, cols, ld, _fmt(fmt), _ptr(scale), _ptr(packed),
                                      row_stride_bytes, _ptr(scale_out), _stream(stream)),
           "dybit_quantize_pack_2d")
    return packed, (scale if scale is not None else scale_out)


def dybit_decode(packed: torch.Tensor, n: int, fmt, scale: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, stream=None):
    if out is None:
        out = _new(packed, n, torch.float32, stream)
    _check(lib.dybit_decode(_ptr(packed), int(n), _fmt(fmt), _ptr(scale), _ptr(out), _stream(stream)),
           "dybit_decode")
    return out


def dybit_gemm(M: int, N: int, K: int, A: torch.Tensor, fa, scale_a: torch.Tensor,
               B: torch.Tensor, fb, scale_b: torch.Tensor, C_out: Optional[torch.Tensor] = None,
               want_raw: bool = False, C_raw: Optional[torch.Tensor] = None,
               ws: Optional[torch.Tensor] = None, lda_bytes: Optional[int] = None,
               ldb_bytes: Optional[int] = None, stream=None):
    """C = sA*sB * value(A) @ value(B)^T.  Returns (C fp32 [M][N], C_raw int32 or None)."""
    lda = A.stride(0) if lda_bytes is None else lda_bytes
    ldb = B.stride(0) if ldb_bytes is None else ldb_bytes
    if C_out is None:
        C_out = _new(A, (M, N), torch.float32, stream)
    if want_raw and C_raw is None:
        C_raw = _new(A, (M, N), torch.int32, stream)
    ws_ptr, ws_bytes, ws = _workspace(dybit_gemm_workspace_bytes(M, N, K, fa, fb), ws, A, stream)
    _check(lib.dybit_gemm(M, N, K, _ptr(A), _fmt(fa), _ptr(scale_a), lda, _ptr(B), _fmt(fb), _ptr(scale_b), ldb,
                          _ptr(C_out), C_out.stride(0), _ptr(C_raw), ws_ptr, ws_bytes, _stream(stream)),
           "dybit_gemm")
    return C_out, C_raw


def dybit_conv2d(desc: ConvDesc, X: torch.Tensor, fx, scale_x: torch.Tensor,
                 W: torch.Tensor, fw, scale_w: torch.Tensor, Y: Optional[torch.Tensor] = None,
                 want_raw: bool = False, Y_raw: Optional[torch.Tensor] = None,
                 ws: Optional[torch.Tensor] = None, ldw_bytes: Optional[int] = None, stream=None):
    """Returns (Y fp32 [n][oh][ow][k], Y_raw int32 or None)."""
    oh, ow = dybit_conv2d_out_hw(desc)
    ldw = W.stride(0) if ldw_bytes is None else ldw_bytes
    if Y is None:
        Y = _new(X, (desc.n, oh, ow, desc.k), torch.float32, stream)
    if want_raw and Y_raw is None:
        Y_raw = _new(X, (desc.n, oh, ow, desc.k), torch.int32, stream)
    ws_ptr, ws_bytes, ws = _workspace(dybit_conv2d_workspace_bytes(desc, fx, fw), ws, X, stream)
    cd = _cdesc(desc)
    _check(lib.dybit_conv2d(C.byref(cd), _ptr(X), _fmt(fx), _ptr(scale_x), _ptr(W), _fmt(fw), _ptr(scale_w), ldw,
                            _ptr(Y), _ptr(Y_raw), ws_ptr, ws_bytes, _stream(stream)), "dybit_conv2d")
    return Y, Y_raw


def dybit_last_device_status(stream=None) -> Tuple[int, int]:
    detail = C.c_uint32(0)
    st = lib.dybit_last_device_status(_stream(stream), C.byref(detail))
    return int(st), int(detail.value)


def dybit_launch_count() -> int:
    return int(lib.dybit_launch_count())


def dybit_selftest_wait_timeout(limit_ns: int, device=None) -> torch.Tensor:
    """Runs the library's bounded wait on a barrier nobody signals; returns the two result words (device tensor)."""
    result = torch.zeros(2, dtype=torch.int32, device=device or torch.device("cuda", torch.cuda.current_device()))
    _check(lib.dybit_selftest_wait_timeout(int(limit_ns), result.data_ptr(), _stream(None)), "dybit_selftest_wait_timeout")
    return result


def dybit_set_gemm_decode(mode: int) -> None:
    """0: expand pass for both operands; 1: decode B in the GEMM's main loop wherever possible; 2: by shape (default)."""
    _check(lib.dybit_set_gemm_decode(int(mode)), "dybit_set_gemm_decode")


def dybit_set_conv_lowering(mode: int) -> None:
    """0: by shape (default); 1: halo tiles wherever they apply; 2: never halo tiles."""
    _check(lib.dybit_set_conv_lowering(int(mode)), "dybit_set_conv_lowering")


def dybit_profile_next_gemm(ev_start: Optional[torch.cuda.Event], ev_stop: Optional[torch.cuda.Event]):
    """Arms event recording around the next GEMM/conv tensor-core kernel (events need enable_timing=True)."""
    if ev_start is None:
        _check(lib.dybit_profile_next_gemm(None, None), "dybit_profile_next_gemm")
        return
    for ev in (ev_start, ev_stop):
        if not ev.cuda_event:           # torch creates the handle lazily on first record
            ev.record()
    _check(lib.dybit_profile_next_gemm(C.c_void_p(ev_start.cuda_event), C.c_void_p(ev_stop.cuda_event)),
           "dybit_profile_next_gemm")


def dybit_profile_next_gemm_clock(t2: Optional[torch.Tensor]):
    """Arms device-clock recording for the next GEMM/conv tensor-core kernel: t2 is an int64 device tensor of two
    elements, initialised to {-1 (all ones), 0}, that receives {first start, last end} in nanoseconds."""
    if t2 is not None and (t2.dtype != torch.int64 or t2.numel() < 2 or not t2.is_cuda):
        raise ValueError("t2 must be an int64 CUDA tensor of two elements")
    _check(lib.dybit_profile_next_gemm_clock(_ptr(t2)), "dybit_profile_next_gemm_clock")


STATIC_WS_BYTES = 16 * 1024 * 1024   # DYBIT_STATIC_WS_BYTES in include/dybit.h


def dybit_gemm_static_ws(M: int, N: int, K: int, A: torch.Tensor, fa, scale_a: torch.Tensor,
                         B: torch.Tensor, fb, scale_b: torch.Tensor, C_out: torch.Tensor,
                         C_raw: Optional[torch.Tensor] = None, lda_bytes: Optional[int] = None,
                         ldb_bytes: Optional[int] = None, stream=None):
    """dybit_gemm without a workspace argument, for callers that cannot allocate device memory.

    The caller passes every input and output buffer (C_out too: this wrapper creates no tensor);
    the library's built-in scratch array holds the expanded operands.  Problems that need more
    than STATIC_WS_BYTES raise DybitError (status 4).  Calls share the scratch: keep them on one
    stream per device.
    """
    lda = A.stride(0) if lda_bytes is None else lda_bytes
    ldb = B.stride(0) if ldb_bytes is None else ldb_bytes
    _check(lib.dybit_gemm_static_ws(M, N, K, _ptr(A), _fmt(fa), _ptr(scale_a), lda, _ptr(B), _fmt(fb),
                                    _ptr(scale_b), ldb, _ptr(C_out), C_out.stride(0), _ptr(C_raw),
                                    _stream(stream)), "dybit_gemm_static_ws")
    return C_out, C_raw


def _bias_ptr(bias, n):
    if bias is None:
        return None
    if not (bias.is_cuda and bias.dtype == torch.float32 and bias.is_contiguous() and bias.numel() == n):
        raise ValueError("bias must be a contiguous float32 device tensor with one value per output column")
    return _ptr(bias)


def dybit_gemm_requant(M: int, N: int, K: int, A: torch.Tensor, fa, scale_a: torch.Tensor,
                       B: torch.Tensor, fb, scale_b: torch.Tensor, fq, scale_q: torch.Tensor, relu: bool = False,
                       bias: Optional[torch.Tensor] = None, Q: Optional[torch.Tensor] = None, ldq_bytes: Optional[int] = None,
                       ws: Optional[torch.Tensor] = None, stream=None):
    """GEMM whose result is written as packed DyBit codes of format fq (scale given).  Returns Q [M][ldq] uint8."""
    if ldq_bytes is None:
        ldq_bytes = N * fq[0] // 8
    if Q is None:
        Q = _new(A, (M, ldq_bytes), torch.uint8, stream, zero=True)
    wp, wn, ws = _workspace(dybit_gemm_workspace_bytes(M, N, K, fa, fb), ws, A, stream)
    _check(lib.dybit_gemm_requant(M, N, K, _ptr(A), _fmt(fa), _ptr(scale_a), A.stride(0), _ptr(B), _fmt(fb),
                                  _ptr(scale_b), B.stride(0), _fmt(fq), _ptr(scale_q), _bias_ptr(bias, N), int(bool(relu)),
                                  _ptr(Q), ldq_bytes, wp, wn, _stream(stream)), "dybit_gemm_requant")
    return Q


def dybit_conv2d_requant(desc: ConvDesc, X: torch.Tensor, fx, scale_x: torch.Tensor, W: torch.Tensor, fw,
                         scale_w: torch.Tensor, fq, scale_q: torch.Tensor, relu: bool = False,
                         bias: Optional[torch.Tensor] = None, Q: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Convolution whose result is the dense NHWK stream of packed codes (the next layer's X).  Returns Q (1-D uint8)."""
    oh, ow = dybit_conv2d_out_hw(desc)
    if Q is None:
        Q = _new(X, dybit_packed_bytes(desc.n * oh * ow * desc.k, fq[0]), torch.uint8, stream, zero=True)
    wp, wn, ws = _workspace(dybit_conv2d_workspace_bytes(desc, fx, fw), ws, X, stream)
    cd = _cdesc(desc)
    _check(lib.dybit_conv2d_requant(C.byref(cd), _ptr(X), _fmt(fx), _ptr(scale_x), _ptr(W), _fmt(fw), _ptr(scale_w),
                                    W.stride(0), _fmt(fq), _ptr(scale_q), _bias_ptr(bias, desc.k), int(bool(relu)),
                                    _ptr(Q), wp, wn,
                                    _stream(stream)), "dybit_conv2d_requant")
    return Q


def dybit_quantize_conv2d_requant(desc: ConvDesc, X: torch.Tensor, fx, W: torch.Tensor, fw, scale_w: torch.Tensor,
                                  fq, scale_q: torch.Tensor, relu: bool = False, bias: Optional[torch.Tensor] = None,
                                  scale_x: Optional[torch.Tensor] = None, scale_out: Optional[torch.Tensor] = None,
                                  packed: Optional[torch.Tensor] = None, Q: Optional[torch.Tensor] = None,
                                  ws: Optional[torch.Tensor] = None, stream=None):
    """Quantize + pack the fp32 NHWC activation X, convolve its codes with W and write the result as packed codes.
    Returns (Q uint8 dense NHWK stream, packed codes of X uint8, scale of X float32[2])."""
    _dev_f32(X, "X")
    if X.numel() != desc.n * desc.h * desc.w * desc.c:
        raise ValueError("X does not match the descriptor")
    oh, ow = dybit_conv2d_out_hw(desc)
    if Q is None:
        Q = _new(X, dybit_packed_bytes(desc.n * oh * ow * desc.k, fq[0]), torch.uint8, stream, zero=True)
    if packed is None:
        packed = _new(X, dybit_packed_bytes(X.numel(), fx[0]), torch.uint8, stream)
    if scale_out is None:
        scale_out = _new(X, 2, torch.float32, stream)
    wp, wn, ws = _workspace(dybit_conv2d_workspace_bytes(desc, fx, fw), ws, X, stream)
    cd = _cdesc(desc)
    _check(lib.dybit_quantize_conv2d_requant(C.byref(cd), _ptr(X), _fmt(fx), _ptr(scale_x), _ptr(scale_out), _ptr(packed),
                                             _ptr(W), _fmt(fw), _ptr(scale_w), W.stride(0), _fmt(fq), _ptr(scale_q),
                                             _bias_ptr(bias, desc.k), int(bool(relu)), _ptr(Q), wp, wn, _stream(stream)),
           "dybit_quantize_conv2d_requant")
    return Q, packed, scale_out


def dybit_gemm_batched_workspace_bytes(batch: int, M: int, N: int, K: int, fa, fb) -> int:
    return int(lib.dybit_gemm_batched_workspace_bytes(int(batch), int(M), int(N), int(K), _fmt(fa), _fmt(fb)))


def dybit_gemm_batched(M: int, N: int, K: int, A: torch.Tensor, fa, scale_a: torch.Tensor, B: torch.Tensor, fb,
                       scale_b: torch.Tensor, want_raw: bool = False, C: Optional[torch.Tensor] = None,
                       ws: Optional[torch.Tensor] = None, stream=None):
    """C[b] = A[b] * B[b]^T for packed A [batch][M][row bytes], B [batch][N][row bytes] (uint8, one scale per operand).
    Returns (C float32 [batch][M][N], C_raw int32 or None)."""
    if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[1] != M or B.shape[1] != N:
        raise ValueError("A must be [batch][M][row bytes] and B [batch][N][row bytes]")
    if A.stride(2) != 1 or B.stride(2) != 1:
        raise ValueError("rows of A and B must be contiguous")
    batch = A.shape[0]
    if C is None:
        C = _new(A, (batch, M, N), torch.float32, stream)
    raw = _new(A, C.shape, torch.int32, stream) if want_raw else None
    if raw is not None and not C.is_contiguous():
        raise ValueError("want_raw needs a contiguous C")
    wp, wn, ws = _workspace(dybit_gemm_batched_workspace_bytes(batch, M, N, K, fa, fb), ws, A, stream)
    _check(lib.dybit_gemm_batched(batch, M, N, K, _ptr(A), _fmt(fa), _ptr(scale_a), A.stride(1), A.stride(0),
                                  _ptr(B), _fmt(fb), _ptr(scale_b), B.stride(1), B.stride(0),
                                  _ptr(C), C.stride(1), C.stride(0), _ptr(raw), wp, wn, _stream(stream)),
           "dybit_gemm_batched")
    return C, raw


def dybit_quantize_conv2d(desc: ConvDesc, X: torch.Tensor, fx, W: torch.Tensor, fw, scale_w: torch.Tensor,
                          scale_x: Optional[torch.Tensor] = None, scale_out: Optional[torch.Tensor] = None,
                          packed: Optional[torch.Tensor] = None, want_raw: bool = False,
                          Y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Quantize + pack the fp32 NHWC activation X and convolve its codes with the packed weights W in one call.
    Returns (Y float32 [n][oh][ow][k], Y_raw int32 or None, packed codes uint8, scale float32[2])."""
    _dev_f32(X, "X")
    if X.numel() != desc.n * desc.h * desc.w * desc.c:
        raise ValueError("X does not match the descriptor")
    oh, ow = dybit_conv2d_out_hw(desc)
    if Y is None:
        Y = _new(X, (desc.n, oh, ow, desc.k), torch.float32, stream)
    raw = _new(X, Y.shape, torch.int32, stream) if want_raw else None
    if packed is None:
        packed = _new(X, dybit_packed_bytes(X.numel(), fx[0]), torch.uint8, stream)
    if scale_out is None:
        scale_out = _new(X, 2, torch.float32, stream)
    wp, wn, ws = _workspace(dybit_conv2d_workspace_bytes(desc, fx, fw), ws, X, stream)
    cd = _cdesc(desc)
    _check(lib.dybit_quantize_conv2d(C.byref(cd), _ptr(X), _fmt(fx), _ptr(scale_x), _ptr(scale_out), _ptr(packed),
                                     _ptr(W), _fmt(fw), _ptr(scale_w), W.stride(0), _ptr(Y), _ptr(raw), wp, wn,
                                     _stream(stream)), "dybit_quantize_conv2d")
    return Y, raw, packed, scale_out


class ConvLayers:
    """Arguments of dybit_quantize_conv2d for several independent layers, marshalled once into the C array that
    dybit_quantize_expand_layers / dybit_conv2d_prepared take.  Each entry of `layers` is a dict with the keyword
    arguments of dybit_quantize_conv2d (desc, X, fx, W, fw, scale_w and optionally scale_x, scale_out, packed, Y,
    want_raw, ws) or, with fq and scale_q given, of dybit_quantize_conv2d_requant (relu, bias, Q): that layer then
    leaves as packed codes in self.Q[i] instead of fp32 in self.Y[i].  Missing outputs and workspaces are allocated
    here, on the current stream, one workspace per layer; they live as long as this object, which has to outlive the
    calls that use it."""

    def __init__(self, layers):
        self.n = len(layers)
        self.array = (_CConvLayer * self.n)()
        self.Y, self.raw, self.packed, self.scale, self.Q, self._keep = [], [], [], [], [], []
        for i, a in enumerate(layers):
            desc, X, fx, W, fw = a["desc"], _dev_f32(a["X"], "X"), a["fx"], a["W"], a["fw"]
            if X.numel() != desc.n * desc.h * desc.w * desc.c:
                raise ValueError("X does not match the descriptor")
            oh, ow = dybit_conv2d_out_hw(desc)
            requant = a.get("fq") is not None
            Y, Q, raw = a.get("Y"), a.get("Q"), None
            if requant:
                if Q is None:
                    Q = torch.zeros(dybit_packed_bytes(desc.n * oh * ow * desc.k, a["fq"][0]), dtype=torch.uint8, device=X.device)
                Y = None
            else:
                if Y is None:
                    Y = torch.empty((desc.n, oh, ow, desc.k), dtype=torch.float32, device=X.device)
                if a.get("want_raw"):
                    raw = torch.empty(Y.shape, dtype=torch.int32, device=X.device)
            packed = a.get("packed")
            if packed is None:
                packed = torch.empty(dybit_packed_bytes(X.numel(), fx[0]), dtype=torch.uint8, device=X.device)
            scale_out = a.get("scale_out")
            if scale_out is None:
                scale_out = torch.empty(2, dtype=torch.float32, device=X.device)
            ws = a.get("ws")
            if ws is None:
                ws = torch.empty(dybit_conv2d_workspace_bytes(desc, fx, fw) + 1024, dtype=torch.uint8, device=X.device)
            wp, wn = _ws_span(ws, X)
            c = self.array[i]
            c.desc = _cdesc(desc)
            addr = lambda t: None if t is None else t.data_ptr()
            c.X, c.fx, c.scale_x = addr(X), _fmt(fx), addr(a.get("scale_x"))
            c.scale_x_out, c.X_packed = addr(scale_out), addr(packed)
            c.W, c.fw, c.scale_w, c.ldw_bytes = addr(W), _fmt(fw), addr(a["scale_w"]), W.stride(0)
            c.Y, c.Y_raw, c.ws, c.ws_bytes = addr(Y), addr(raw), wp, wn
            if requant:
                bias = a.get("bias")
                c.Q, c.fq, c.scale_q, c.relu = addr(Q), _fmt(a["fq"]), addr(a["scale_q"]), int(bool(a.get("relu")))
                c.bias = None if bias is None else _bias_ptr(bias, desc.k).value
                self._keep.append((a["scale_q"], bias))
            self.Q.append(Q)
            self.Y.append(Y)
            self.raw.append(raw)
            self.packed.append(packed)
            self.scale.append(scale_out)
            self._keep.append((X, W, a["scale_w"], a.get("scale_x"), ws))


def dybit_quantize_expand_layers(layers: ConvLayers, stream=None):
    """Max-abs scales, codes and expanded operands of all the layers, in few launches on one stream."""
    _check(lib.dybit_quantize_expand_layers(layers.array, layers.n, _stream(stream)), "dybit_quantize_expand_layers")


def dybit_conv2d_prepared(layers: ConvLayers, i: int, stream=None):
    """The tensor-core part of layer i, after dybit_quantize_expand_layers.  Returns (Y, Y_raw or None), or (Q, None)
    for a layer with the re-quantizing epilogue."""
    _check(lib.dybit_conv2d_prepared(C.byref(layers.array[i]), _stream(stream)), "dybit_conv2d_prepared")
    return (layers.Y[i] if layers.Q[i] is None else layers.Q[i]), layers.raw[i]


def dybit_conv2d_prepared_layers(layers: ConvLayers, stream=None):
    """The tensor-core part of all layers on one stream, layers of one kernel configuration sharing launches."""
    _check(lib.dybit_conv2d_prepared_layers(layers.array, layers.n, _stream(stream)), "dybit_conv2d_prepared_layers")


def dybit_depthwise_conv2d(desc: ConvDesc, X: torch.Tensor, fx, scale_x: torch.Tensor, W: torch.Tensor, fw,
                           scale_w: torch.Tensor, Y: Optional[torch.Tensor] = None, stream=None):
    """Depth-wise convolution (desc.k == desc.c).  X: dense NHWC code stream; W: [c][row bytes] rows of r*s codes
    (dybit_quantize_pack_2d of the [c][r*s] filter matrix).  Returns Y [n][oh][ow][c] float32."""
    oh, ow = dybit_conv2d_out_hw(desc)
    if Y is None:
        Y = _new(X, (desc.n, oh, ow, desc.c), torch.float32, stream)
    cd = _cdesc(desc)
    _check(lib.dybit_depthwise_conv2d(C.byref(cd), _ptr(X), _fmt(fx), _ptr(scale_x), _ptr(W), _fmt(fw), _ptr(scale_w),
                                      W.stride(0), _ptr(Y), _stream(stream)), "dybit_depthwise_conv2d")
    return Y


def dybit_rmse(x: torch.Tensor, fmt, scale: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None):
    """Eq. 2.  Returns a float64 device tensor {RMSE, sigma, mse, n}."""
    _dev_f32(x, "x")
    if out is None:
        out = _new(x, 4, torch.float64, stream)
    _check(lib.dybit_rmse(_ptr(x), x.numel(), _fmt(fmt), _ptr(scale), _ptr(out), _stream(stream)), "dybit_rmse")
    return out


def dybit_rmse_sweep(x: torch.Tensor, fmts, scales: torch.Tensor, stream=None):
    """Eq. 2 for several candidate (format, scale) pairs in one pass over x.  scales: float32 device tensor
    [len(fmts)][2] of {scale, 1/scale}.  Returns (float64 device tensor [len(fmts)][4] of {RMSE, sigma, mse, n},
    int32 device tensor holding the index of the smallest RMSE)."""
    _dev_f32(x, "x")
    nc = len(fmts)
    if not (scales.is_cuda and scales.dtype == torch.float32 and scales.is_contiguous() and scales.numel() == 2 * nc):
        raise ValueError("scales must be a contiguous float32 device tensor with two values per candidate")
    arr = (_CFmt * max(nc, 1))(*[_fmt(f) for f in fmts])
    out = _new(x, (nc, 4), torch.float64, stream)
    best = _new(x, 1, torch.int32, stream)
    _check(lib.dybit_rmse_sweep(_ptr(x), x.numel(), nc, arr, _ptr(scales), _ptr(out), _ptr(best), _stream(stream)),
           "dybit_rmse_sweep")
    return out, best


def dybit_fake_quant(x: torch.Tensor, fmt, scale: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None):
    """Quantize-dequantize image of x (QAT forward) in one pass; returns a float32 tensor shaped like x."""
    _dev_f32(x, "x")
    if out is None:
        out = _new(x, x.shape, x.dtype, stream)
    _dev_f32(out, "out")
    _check(lib.dybit_fake_quant(_ptr(x), x.numel(), _fmt(fmt), _ptr(scale), _ptr(out), _stream(stream)),
           "dybit_fake_quant")
    return out


def dybit_fake_quant_backward(x: torch.Tensor, grad_out: torch.Tensor, fmt, scale: torch.Tensor,
                              out: Optional[torch.Tensor] = None, stream=None):
    """Clipped straight-through gradient of dybit_fake_quant with respect to x."""
    _dev_f32(x, "x")
    _dev_f32(grad_out, "grad_out")
    if grad_out.numel() != x.numel():
        raise ValueError("grad_out must have as many elements as x")
    if out is None:
        out = _new(x, x.shape, x.dtype, stream)
    _dev_f32(out, "out")
    _check(lib.dybit_fake_quant_backward(_ptr(x), _ptr(grad_out), x.numel(), _fmt(fmt), _ptr(scale), _ptr(out),
                                         _stream(stream)), "dybit_fake_quant_backward")
    return out


def dybit_search_bitwidths(lat, rmse, num_layers: int, strategy: str, constraint: float, top_k: int):
    """Algorithm 1.  lat / rmse: flat sequences of num_layers*9 numbers, index (layer*3 + a_idx)*3 + w_idx with
    idx 0, 1, 2 <-> 8, 4, 2 bits.  strategy "speedup" (constraint = alpha) or "rmse" (constraint = beta).
    Returns (weight bits, activation bits) as two lists."""
    if len(lat) != num_layers * 9 or len(rmse) != num_layers * 9:
        raise ValueError("lat and rmse need num_layers * 9 entries")
    if strategy not in ("speedup", "rmse"):
        raise ValueError("strategy must be 'speedup' or 'rmse'")
    la = (C.c_double * len(lat))(*[float(v) for v in lat])
    ra = (C.c_double * len(rmse))(*[float(v) for v in rmse])
    w = (C.c_int * num_layers)()
    a = (C.c_int * num_layers)()
    _check(lib.dybit_search_bitwidths(num_layers, la, ra, 0 if strategy == "speedup" else 1, float(constraint),
                                      int(top_k), w, a), "dybit_search_bitwidths")
    return list(w), list(a)


# ---------------------------------------------------------------- fine-tuning a coded layer

_DTYPE_CODE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _matrix(x: torch.Tensor, name: str, rows: Optional[int] = None, cols: Optional[int] = None) -> Tuple[int, int]:
    """Checks a 2-D device matrix of real numbers with contiguous rows; returns (dybit_dtype, row stride)."""
    code, shape = _DTYPE_CODE.get(x.dtype), x.shape
    if code is None or not x.is_cuda or len(shape) != 2:
        raise ValueError(f"{name} must be a 2-D float32, bfloat16 or float16 CUDA tensor with unit inner stride")
    r, c = shape
    ld, inner = x.stride()
    if inner != 1 and c > 1:
        raise ValueError(f"{name} must be a 2-D float32, bfloat16 or float16 CUDA tensor with unit inner stride")
    if (cols is not None and c != cols) or (rows is not None and r != rows):
        raise ValueError(f"{name} has shape {(r, c)}, expected ({'any' if rows is None else rows}, {'any' if cols is None else cols})")
    return code, (ld if r > 1 or ld > c else c)       # (torch gives a single row any stride)


def _codes8(codes: torch.Tensor, rows: int, cols: int, scales: torch.Tensor, per_row: bool) -> Tuple[int, int]:
    """Checks a matrix of 8-bit codes and its scales; returns (row stride in bytes, scale stride)."""
    shape = codes.shape
    if codes.dtype != torch.uint8 or not codes.is_cuda or len(shape) != 2 or shape[0] != rows or shape[1] < cols:
        raise ValueError("codes must be a 2-D uint8 CUDA tensor [rows][row bytes >= cols] with unit inner stride")
    ld, inner = codes.stride()
    if inner != 1 and shape[1] > 1:
        raise ValueError("codes must be a 2-D uint8 CUDA tensor [rows][row bytes >= cols] with unit inner stride")
    if scales.dtype != torch.float32 or not scales.is_cuda or not scales.is_contiguous() or scales.numel() < (rows if per_row else 1):
        raise ValueError("scales must be a contiguous float32 CUDA tensor with one value per row, or the scale of the whole tensor")
    return (ld if rows > 1 or ld > shape[1] else shape[1]), 1 if per_row else 0


def dybit_checkpoint_save(x: torch.Tensor, fmt, top: int = 2, codes: Optional[torch.Tensor] = None,
                          scales: Optional[torch.Tensor] = None, stream=None):
    """8-bit codes of an activation [rows][cols] with one power-of-two scale per row; the largest magnitude of a row
    lands in (2^(top-1), 2^top].  Returns (codes uint8 [rows][row bytes], scales float32 [rows])."""
    t, ld = _matrix(x, "x")
    rows, cols = x.shape
    stride = padded = (cols + 127) // 128 * 128
    given = codes is not None or scales is not None
    if codes is None:
        codes = _new(x, (rows, padded), torch.uint8, stream)
    if scales is None:
        scales = _new(x, rows, torch.float32, stream)
    if given:
        stride, _ = _codes8(codes, rows, cols, scales, True)
        if codes.shape[1] < padded and codes.shape[1] < stride:
            raise ValueError("codes must have room for the columns rounded up to 128, or to the end of its rows")
    _check(lib.dybit_checkpoint_save(x.data_ptr(), t, rows, cols, ld, _fmt(fmt), top, codes.data_ptr(), stride,
                                     scales.data_ptr(), _stream(stream)), "dybit_checkpoint_save")
    return codes, scales


def dybit_checkpoint_load(codes: torch.Tensor, cols: int, fmt, scales: torch.Tensor, dtype: torch.dtype = torch.float32,
                          out: Optional[torch.Tensor] = None, per_row: bool = True, stream=None):
    """The activation [rows][cols] that a checkpoint stands for.  per_row=False: scales is the pair {scale, 1/scale} of
    the whole tensor, as dybit_quantize_pack_2d writes it."""
    rows = codes.shape[0]
    stride, scale_stride = _codes8(codes, rows, cols, scales, per_row)
    if out is None:
        if dtype not in _DTYPE_CODE:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        out, t, ld = _new(codes, (rows, cols), dtype, stream), _DTYPE_CODE[dtype], cols
    else:
        t, ld = _matrix(out, "out", rows, cols)
    _check(lib.dybit_checkpoint_load(codes.data_ptr(), stride, scales.data_ptr(), scale_stride, rows, cols, _fmt(fmt),
                                     out.data_ptr(), t, ld, _stream(stream)), "dybit_checkpoint_load")
    return out


def dybit_checkpoint_wgrad_workspace_bytes(T: int, N: int, K: int, dtype: torch.dtype) -> int:
    if dtype not in _DTYPE_CODE:
        raise ValueError("dtype must be float32, bfloat16 or float16")
    return int(lib.dybit_checkpoint_wgrad_workspace_bytes(int(T), int(N), int(K), _DTYPE_CODE[dtype]))


def dybit_checkpoint_wgrad(dY: torch.Tensor, codes: torch.Tensor, K: int, fmt, scales: torch.Tensor,
                           out: Optional[torch.Tensor] = None, per_row: bool = True,
                           ws: Optional[torch.Tensor] = None, stream=None):
    """dW [N][K] float32 = dY^T x^ with x^ [T][K] read from an 8-bit checkpoint.  x^ takes part as bf16 numbers: exact for the
    scales of dybit_checkpoint_save (powers of two) and with per_row=False, rounded to nearest for other row scales."""
    t, ld = _matrix(dY, "dY")
    T, N = dY.shape
    stride, scale_stride = _codes8(codes, T, K, scales, per_row)
    if out is None:
        out, ldo = _new(dY, (N, K), torch.float32, stream), K
    else:
        to, ldo = _matrix(out, "out", N, K)
        if to != 0:
            raise ValueError("out must be float32")
    at, size, ws = _workspace(lib.dybit_checkpoint_wgrad_workspace_bytes(T, N, K, t), ws, dY, stream)
    _check(lib.dybit_checkpoint_wgrad(T, N, K, dY.data_ptr(), t, ld, codes.data_ptr(), stride, _fmt(fmt), scales.data_ptr(),
                                      scale_stride, out.data_ptr(), ldo, at, size, _stream(stream)), "dybit_checkpoint_wgrad")
    return out


def dybit_adapters_plan_bytes(T: int, n_adapters: int) -> int:
    return int(lib.dybit_adapters_plan_bytes(int(T), int(n_adapters)))


def dybit_adapters_plan(ids: torch.Tensor, n_adapters: int, plan: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Groups the tokens of a batch by adapter: ids int32 [T], outside 0 .. n_adapters-1 for a token without one.
    Returns the plan's buffer (uint8)."""
    if ids.dtype != torch.int32 or not ids.is_cuda or ids.dim() != 1 or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous 1-D int32 CUDA tensor")
    T = ids.numel()
    if plan is None:
        plan = _new(ids, dybit_adapters_plan_bytes(T, n_adapters), torch.uint8, stream)
    _check(lib.dybit_adapters_plan(T, ids.data_ptr(), int(n_adapters), plan.data_ptr(), plan.numel(), _stream(stream)),
           "dybit_adapters_plan")
    return plan


class AdapterPlan:
    """The plan of one batch of tokens, for every call with the same tokens (dybit_adapters_plan).  It has to outlive the
    calls that use it (or take buffer.record_stream), as any tensor that is used on another stream than its own."""

    def __init__(self, ids: torch.Tensor, n_adapters: int, stream=None):
        self.T, self.n = ids.numel(), int(n_adapters)
        self.buffer = dybit_adapters_plan(ids, n_adapters, stream=stream)
        self.address = self.buffer.data_ptr()


def _factors(A: torch.Tensor, B: torch.Tensor, alpha: Optional[torch.Tensor], plan: AdapterPlan) -> Tuple[int, int, int, int]:
    """Checks the factors [n][R][K] and [n][R][N]; returns (R, K, N, dybit_dtype)."""
    a, b, dt = A.shape, B.shape, A.dtype
    if len(a) != 3 or len(b) != 3 or a[0] != plan.n or b[0] != plan.n or a[1] != b[1] or dt != B.dtype or \
            dt not in (torch.bfloat16, torch.float16) or not (A.is_cuda and B.is_cuda and A.is_contiguous() and B.is_contiguous()):
        raise ValueError("A and B must be contiguous 16-bit CUDA tensors [n_adapters][R][K] and [n_adapters][R][N]")
    if alpha is not None and (alpha.dtype != torch.float32 or not alpha.is_cuda or not alpha.is_contiguous() or alpha.numel() != plan.n):
        raise ValueError("alpha must be a contiguous float32 CUDA tensor with one value per adapter")
    return a[1], a[2], b[2], _DTYPE_CODE[dt]


def _dense(x: torch.Tensor, name: str, shape) -> int:
    """Checks a dense float32 device tensor of the given shape; returns its address."""
    if x.dtype != torch.float32 or not x.is_cuda or x.shape != shape or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 CUDA tensor {list(shape)}")
    return x.data_ptr()


def dybit_adapters(x: torch.Tensor, A: torch.Tensor, B: torch.Tensor, alpha: Optional[torch.Tensor], plan: AdapterPlan,
                   base: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                   want_v: bool = False, v: Optional[torch.Tensor] = None, stream=None):
    """y[t] = base[t] + alpha_a * (x[t] A_a^T) B_a with a the adapter of token t: x [T][K], A [n][R][K], B [n][R][N].
    out may be base.  Returns (y [T][N], V [T][R] float32 or None); V is what dybit_adapters_backward takes."""
    R, K, N, tw = _factors(A, B, alpha, plan)
    T = plan.T
    tx, ldx = _matrix(x, "x", T, K)
    tb, ldb = (None, 0) if base is None else _matrix(base, "base", T, N)
    if out is None:
        dtype = base.dtype if base is not None else (out_dtype or x.dtype)
        if dtype not in _DTYPE_CODE:
            raise ValueError("out_dtype must be float32, bfloat16 or float16")
        out, ty, ldy = _new(x, (T, N), dtype, stream), _DTYPE_CODE[dtype], N
    else:
        ty, ldy = _matrix(out, "out", T, N)
    if base is not None and tb != ty:
        raise ValueError("base and out must have one dtype")
    if want_v and v is None:
        v = _new(x, (T, R), torch.float32, stream)
    _check(lib.dybit_adapters(T, K, N, R, x.data_ptr(), tx, ldx, plan.n, A.data_ptr(), B.data_ptr(), tw,
                              None if alpha is None else alpha.data_ptr(), plan.address, None if base is None else base.data_ptr(),
                              ldb, ty, out.data_ptr(), ldy, None if v is None else _dense(v, "v", (T, R)), _stream(stream)),
           "dybit_adapters")
    return out, v


def dybit_adapters_backward_workspace_bytes(T: int, K: int, N: int, R: int, n_adapters: int) -> int:
    return int(lib.dybit_adapters_backward_workspace_bytes(int(T), int(K), int(N), int(R), int(n_adapters)))


def dybit_adapters_backward(dY: torch.Tensor, codes: torch.Tensor, fmt, scales: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
                            alpha: Optional[torch.Tensor], plan: AdapterPlan, v: torch.Tensor,
                            dx_base: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                            dA: Optional[torch.Tensor] = None, dB: Optional[torch.Tensor] = None,
                            per_row: bool = True, ws: Optional[torch.Tensor] = None, stream=None):
    """Gradients of dybit_adapters with its input read from an 8-bit checkpoint (codes [T][row bytes], scales).  dx may
    be dx_base.  Returns (dx [T][K] like dY, dA [n][R][K] float32, dB [n][R][N] float32)."""
    R, K, N, tw = _factors(A, B, alpha, plan)
    T, n = plan.T, plan.n
    t, ldy = _matrix(dY, "dY", T, N)
    stride, scale_stride = _codes8(codes, T, K, scales, per_row)
    tb, ldb = (t, 0) if dx_base is None else _matrix(dx_base, "dx_base", T, K)
    if dx is None:
        dx, tx, ldx = _new(dY, (T, K), dY.dtype, stream), t, K
    else:
        tx, ldx = _matrix(dx, "dx", T, K)
    if tx != t or tb != t:
        raise ValueError("dx and dx_base must have dY's dtype")
    if dA is None:
        dA = _new(dY, (n, R, K), torch.float32, stream)
    if dB is None:
        dB = _new(dY, (n, R, N), torch.float32, stream)
    at, size, ws = _workspace(lib.dybit_adapters_backward_workspace_bytes(T, K, N, R, n), ws, dY, stream)
    _check(lib.dybit_adapters_backward(T, K, N, R, dY.data_ptr(), t, ldy, codes.data_ptr(), stride, _fmt(fmt),
                                       scales.data_ptr(), scale_stride, n, A.data_ptr(), B.data_ptr(), tw,
                                       None if alpha is None else alpha.data_ptr(), plan.address, _dense(v, "v", (T, R)),
                                       None if dx_base is None else dx_base.data_ptr(), ldb, dx.data_ptr(), ldx,
                                       _dense(dA, "dA", (n, R, K)), _dense(dB, "dB", (n, R, N)), at, size, _stream(stream)),
           "dybit_adapters_backward")
    return dx, dA, dB


# ---------------------------------------------------------------- key-value cache in 8-bit codes

def _c_int(value, name: str) -> int:
    """An argument that the library takes in 32 bits, which ctypes would cut it to."""
    value = int(value)
    if not -2**31 <= value < 2**31:
        raise ValueError(f"{name} does not fit 32 bits")
    return value


def _window(window) -> int:
    """A window of any size: one of 2^31 - 1 holds every sequence whole already."""
    return _c_int(min(int(window), 2**31 - 1), "window")


class KVCache:
    """A pool of `pages` pages for the keys and values of `heads` heads of `dim` elements, `page` tokens to a page: codes
    uint8 [pages][heads][page][dim] and scales float32 [pages][heads], for keys and for values.  Buffers that are not given
    are allocated on `device`, on the current stream; a new pool reads as zeros."""

    def __init__(self, pages: int, page: int, heads: int, dim: int, device=None, k_codes: Optional[torch.Tensor] = None,
                 v_codes: Optional[torch.Tensor] = None, k_scales: Optional[torch.Tensor] = None, v_scales: Optional[torch.Tensor] = None):
        self.pages, self.page, self.heads, self.dim = int(pages), _c_int(page, "page"), _c_int(heads, "heads"), _c_int(dim, "dim")
        given = next((t for t in (k_codes, v_codes, k_scales, v_scales) if t is not None), None)
        device = given.device if given is not None else device or torch.device("cuda", torch.cuda.current_device())

        def buffer(t, name, shape, dtype):
            if t is None:
                return torch.zeros(shape, dtype=dtype, device=device) if dtype == torch.float32 else torch.empty(shape, dtype=dtype, device=device)
            if not (t.is_cuda and t.device == given.device and t.dtype == dtype and tuple(t.shape) == shape and t.is_contiguous()):
                raise ValueError(f"{name} must be a contiguous {dtype} CUDA tensor {list(shape)}, all on one device")
            return t

        codes, scales = (self.pages, self.heads, self.page, self.dim), (self.pages, self.heads)
        self.k_codes, self.v_codes = buffer(k_codes, "k_codes", codes, torch.uint8), buffer(v_codes, "v_codes", codes, torch.uint8)
        self.k_scales, self.v_scales = buffer(k_scales, "k_scales", scales, torch.float32), buffer(v_scales, "v_scales", scales, torch.float32)
        self.c = _CCache(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.k_scales.data_ptr(), self.v_scales.data_ptr(),
                         self.pages, self.page, self.heads, self.dim)
        self.ref, self.device = C.byref(self.c), self.k_codes.get_device()


def _on(device: int, *tensors: Optional[torch.Tensor]):
    """The calls run on the current device, and what they are given lies there."""
    if device != (_raw_device or torch.cuda.current_device)():
        raise ValueError(f"the cache or the table lies on device {device}, which is not the current one")
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"a tensor on {t.device} with a cache or a table on device {device}")


def _cache_ints(t: torch.Tensor, name: str, n: int):
    if not (t.dtype == torch.int32 and t.is_cuda and t.dim() == 1 and t.is_contiguous() and t.numel() == n):
        raise ValueError(f"{name} must be a contiguous int32 CUDA tensor of {n} entries")


def _cache_batch(cache: KVCache, table: torch.Tensor, tokens: int, q_heads: Optional[int], max_new: Optional[int], causal: bool = True,
                 window: int = 0) -> _CCacheBatch:
    if not (table.dtype == torch.int32 and table.is_cuda and table.dim() == 2 and (table.stride(1) == 1 or table.shape[1] <= 1)):
        raise ValueError("table must be a 2-D int32 CUDA tensor [sequences][pages] with unit inner stride")
    B, most = table.shape
    stride = table.stride(0) if B > 1 else most            # (torch gives a single row any stride)
    if stride < most:
        raise ValueError("the rows of table must not overlap: give a copy of a table that is expanded or slides over another")
    return _CCacheBatch(_c_int(B, "the number of sequences"), _c_int(tokens, "tokens"), _c_int(tokens if max_new is None else min(max_new, tokens), "max_new"),
                        cache.heads if q_heads is None else _c_int(q_heads, "q_heads"), table.data_ptr(), stride, _c_int(most, "the table's width"),
                        int(bool(causal)), _window(window))


def dybit_cache_plan_bytes(cache: KVCache, table: torch.Tensor, tokens: int, q_heads: Optional[int] = None, max_new: Optional[int] = None) -> int:
    return int(lib.dybit_cache_plan_bytes(cache.ref, C.byref(_cache_batch(cache, table, tokens, q_heads, max_new))))


def dybit_cache_plan(cache: KVCache, table: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor, tokens: int, q_heads: Optional[int] = None,
                     max_new: Optional[int] = None, causal: bool = True, window: int = 0, plan: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """Lists of the work of a batch (see CachePlan).  Returns the plan's buffer (uint8).  On another stream than their own, starts
    and lengths have to outlive the call's work, and the table that of all calls that go by the plan."""
    batch = _cache_batch(cache, table, tokens, q_heads, max_new, causal, window)
    _on(table.get_device(), starts, lengths, plan)
    _cache_ints(starts, "starts", batch.sequences + 1)
    _cache_ints(lengths, "lengths", batch.sequences)
    need = int(lib.dybit_cache_plan_bytes(cache.ref, C.byref(batch)))
    if plan is None:
        plan = _new(table, max(need, 16), torch.uint8, stream)
    elif not (plan.is_cuda and plan.is_contiguous()):
        raise ValueError("plan must be a contiguous CUDA tensor")
    _check(lib.dybit_cache_plan(cache.ref, C.byref(batch), starts.data_ptr(), lengths.data_ptr(), plan.data_ptr(), plan.numel() * plan.element_size(),
                                _stream(stream)), "dybit_cache_plan")
    return plan


class CachePlan:
    """The plan of one batch of sequences, for every call on caches of the same pages' size and heads: table int32
    [sequences][pages] with the page of every `page` tokens (rows of any stride that do not overlap), starts int32 [sequences + 1] with the rows of each sequence's
    new tokens among the batch's `tokens` rows, lengths int32 [sequences] with the tokens of each sequence, new ones
    included.  max_new bounds the new tokens of one sequence (default: tokens); the smaller, the less is launched.  causal and
    window say how the attention will mask; a call that masks otherwise takes one more launch.  The plan has to outlive the calls
    that use it (or its tensors take record_stream), as any tensor that is used on another stream than its own; it keeps
    the table, starts and lengths alive."""

    def __init__(self, cache: KVCache, table: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor, tokens: int, q_heads: Optional[int] = None,
                 max_new: Optional[int] = None, causal: bool = True, window: int = 0, buffer: Optional[torch.Tensor] = None, stream=None):
        self.table, self.starts, self.lengths, self.T, self.device = table, starts, lengths, int(tokens), table.get_device()
        self.batch = _cache_batch(cache, table, tokens, q_heads, max_new, causal, window)
        self.q_heads, self.page, self.heads = self.batch.q_heads, cache.page, cache.heads
        self.buffer = dybit_cache_plan(cache, table, starts, lengths, tokens, q_heads, max_new, causal, window, buffer, stream)
        self.address, self.ref = self.buffer.data_ptr(), C.byref(self.batch)
        self._ws_bytes = {}

    def _for(self, cache: KVCache, *tensors: Optional[torch.Tensor]):
        if cache.page != self.page or cache.heads != self.heads or cache.device != self.device:
            raise ValueError("the plan was made for a cache of other pages or heads, or on another device")
        _on(cache.device, *tensors)

    def _workspace_bytes(self, cache: KVCache) -> int:
        need = self._ws_bytes.get(cache.dim)
        if need is None:
            need = self._ws_bytes[cache.dim] = int(lib.dybit_cache_attention_workspace_bytes(cache.ref, self.ref))
        return need


def _heads3(x: torch.Tensor, name: str, T: int, heads: int, dim: int, code: Optional[int] = None) -> Tuple[int, int, int]:
    """Checks a tensor [T][heads][dim] with unit inner stride; returns (dybit_dtype, token stride, head stride)."""
    t = _DTYPE_CODE.get(x.dtype)
    st, sh, inner = x.stride() if x.dim() == 3 else (0, 0, 0)
    if t is None or not x.is_cuda or x.shape != (T, heads, dim) or inner != 1 or (code is not None and t != code):
        raise ValueError(f"{name} must be a CUDA tensor [{T}][{heads}][{dim}] with unit inner stride, of float32, bfloat16 or float16 as its fellows")
    if (T > 1 and st < dim) or (heads > 1 and sh < dim):
        raise ValueError(f"the tokens and heads of {name} must not overlap")
    # (torch gives an axis of one entry any stride)
    return t, (st if T > 1 else heads * dim), (sh if heads > 1 else dim)


def dybit_cache_write(cache: KVCache, k: torch.Tensor, v: torch.Tensor, plan: CachePlan, top: int = 2, stream=None) -> None:
    """Stores the keys and values [tokens][heads][dim] of a batch's new tokens in the pages of the plan's table."""
    plan._for(cache, k, v)
    t, kt, kh = _heads3(k, "k", plan.T, cache.heads, cache.dim)
    _, vt, vh = _heads3(v, "v", plan.T, cache.heads, cache.dim, t)
    _check(lib.dybit_cache_write(cache.ref, plan.ref, plan.address, k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, t, _c_int(top, "top"), _stream(stream)),
           "dybit_cache_write")


def dybit_cache_read(cache: KVCache, plan: CachePlan, dtype: torch.dtype = torch.float32, k: Optional[torch.Tensor] = None,
                     v: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The keys and values [tokens][heads][dim] that the cache holds for a batch's new tokens.  Rows of no sequence are
    left as they are."""
    plan._for(cache, k, v)
    if dtype not in _DTYPE_CODE:
        raise ValueError("dtype must be float32, bfloat16 or float16")
    T, H, D = shape = (plan.T, cache.heads, cache.dim)
    kt, kh, vt, vh = H * D, D, H * D, D
    if k is None and v is None:
        t, k, v = _DTYPE_CODE[dtype], _new(cache.k_codes, shape, dtype, stream), _new(cache.k_codes, shape, dtype, stream)
    else:
        if k is None:
            k = _new(cache.k_codes, shape, v.dtype, stream)
        if v is None:
            v = _new(cache.k_codes, shape, k.dtype, stream)
        t, kt, kh = _heads3(k, "k", T, H, D)
        _, vt, vh = _heads3(v, "v", T, H, D, t)
    _check(lib.dybit_cache_read(cache.ref, plan.ref, plan.address, k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, t, _stream(stream)),
           "dybit_cache_read")
    return k, v


def dybit_cache_attention_workspace_bytes(cache: KVCache, plan: CachePlan) -> int:
    return plan._workspace_bytes(cache)


def dybit_cache_attention(q: torch.Tensor, cache: KVCache, plan: CachePlan, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                          out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Attention of a batch's new tokens q [tokens][q_heads][dim] (bfloat16 or float16) over their sequences' caches; scale
    defaults to dim ** -0.5, window > 0 lets a token see the last `window` keys, its own among them.  Returns the outputs
    [tokens][q_heads][dim]; lse, float32 [tokens][q_heads], receives the logarithms of the rows' sums where it is given."""
    plan._for(cache, q, out, lse)
    t, qt, qh = _heads3(q, "q", plan.T, plan.q_heads, cache.dim)
    if t == 0:
        raise ValueError("q must be bfloat16 or float16")
    if out is None:
        out, yt, yh = _new(q, q.shape, q.dtype, stream), plan.q_heads * cache.dim, cache.dim
    else:
        _, yt, yh = _heads3(out, "out", plan.T, plan.q_heads, cache.dim, t)
    at, size, ws = _workspace(plan._workspace_bytes(cache), ws, q, stream)
    _check(lib.dybit_cache_attention(cache.ref, plan.ref, plan.address, q.data_ptr(), t, qt, qh, out.data_ptr(), yt, yh,
                                     None if lse is None else _dense(lse, "lse", (plan.T, plan.q_heads)),
                                     cache.dim ** -0.5 if scale is None else scale, int(bool(causal)), _window(window), at, size, _stream(stream)),
           "dybit_cache_attention")
    return out
