"""Thin ctypes binding of libim2win.so: argument marshalling only.

Every function mirrors the C entry point of the same name (include/im2win.h)
on torch CUDA tensors; all arithmetic runs in the CUDA kernels behind the C
ABI.  Loading fails loudly when the library cannot be built or opened: there
is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Tuple

import torch

from . import build as _build

F32 = 0
F16 = 1
BF16 = 2      # the operators on token sequences only

STATUS_NAMES = {
    0: "IM2WIN_OK", 1: "IM2WIN_ERR_INVALID_ARG", 2: "IM2WIN_ERR_NULL_POINTER", 3: "IM2WIN_ERR_MISALIGNED",
    4: "IM2WIN_ERR_WORKSPACE_TOO_SMALL", 5: "IM2WIN_ERR_UNSUPPORTED", 6: "IM2WIN_ERR_CUDA", 7: "IM2WIN_ERR_TIMEOUT",
}

EXPORTS = (
    "im2win_status_string", "im2win_workspace_size", "im2win_transform", "im2win_conv_f32", "im2win_conv_f16",
    "im2win_check_status", "im2win_layer_workspace_size", "im2win_layer_forward_host",
    "im2win_conv_f32_static", "im2win_pack_filter", "im2win_conv_packed", "im2win_conv_kernel_name", "im2win_nhwc_kernel_name",
    "im2win_nhwc_workspace_size", "im2win_transform_nhwc", "im2win_conv_f16_nhwc", "im2win_pack_filter_nhwc",
    "im2win_conv_packed_nhwc", "im2win_causal_conv1d", "im2win_linear_attention",
    "im2win_linear_attention_workspace_size", "im2win_linear_attention_kernel_name", "im2win_matvec_int4",
    "im2win_matvec_int4_kernel_name", "im2win_gated_delta_rule", "im2win_gated_delta_rule_kernel_name", "im2win_rms_norm",
    "im2win_matmul_int8", "im2win_matmul_int8_kernel_name",
)

STATIC_SCRATCH_BYTES = 4 << 20


class Shape(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("N", "C", "H", "W", "Co", "Kh", "Kw", "stride", "pad")]


NCHW = 0
NHWC = 1


class Epilogue(ctypes.Structure):
    """im2win_epilogue: bias (device pointer or NULL), relu, out_dtype (F32/F16), out_layout (NCHW/NHWC)."""

    _fields_ = [("bias", ctypes.c_void_p), ("relu", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("out_layout", ctypes.c_int32)]


class Sequences(ctypes.Structure):
    """im2win_sequences: device pointers to row numbers, pool elements and flags, each NULL or one a sequence."""

    _fields_ = [("cu_seqlens", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("resume", ctypes.c_void_p)]


class Conv1dShape(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("tokens", "sequences", "slots", "channels", "taps", "silu")] + \
               [(k, ctypes.c_int64) for k in ("x_stride", "y_stride")]


class AttentionShape(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("tokens", "sequences", "slots", "max_len", "heads", "qk_heads", "dk", "dv")] + \
               [("scale", ctypes.c_float)] + \
               [(k, ctypes.c_int64) for k in ("q_stride", "k_stride", "v_stride", "o_stride", "decay_stride")]


class Int4Shape(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("M", "N", "K", "group")] + [(k, ctypes.c_int64) for k in ("x_stride", "y_stride")]


class DeltaShape(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("tokens", "sequences", "slots", "max_len", "heads", "qk_heads", "dk", "dv", "normalize")] + \
               [("scale", ctypes.c_float)] + \
               [(k, ctypes.c_int64) for k in ("q_stride", "k_stride", "v_stride", "o_stride", "decay_stride", "beta_stride")]


class NormShape(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("rows", "channels")] + [("eps", ctypes.c_float)] + \
               [(k, ctypes.c_int64) for k in ("x_stride", "residual_stride", "residual_out_stride", "y_stride")]


class Int8Shape(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("M", "N", "K")] + [(k, ctypes.c_int64) for k in ("x_stride", "y_stride")]


class Im2winError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().im2win_status_string(code).decode()
        super().__init__(f"{where}: {STATUS_NAMES.get(code, code)} ({msg})")


_lib: Optional[ctypes.CDLL] = None
# Set with the library (which looks the switch up once per process too): its testing-aid switches may change the sizes.
_debug = True


def lib() -> ctypes.CDLL:
    """Build (if stale) and load the shared library; raises on failure."""
    global _lib, _debug
    if _lib is not None:
        return _lib
    path = _build.build_library()
    L = ctypes.CDLL(path)
    P = ctypes.POINTER
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    L.im2win_status_string.argtypes = [ctypes.c_int]
    L.im2win_status_string.restype = ctypes.c_char_p
    L.im2win_workspace_size.argtypes = [P(Shape), ctypes.c_int, P(sz), P(sz), P(i32), P(i32)]
    L.im2win_transform.argtypes = [vp, vp, P(Shape), ctypes.c_int, vp]
    L.im2win_conv_f32.argtypes = [vp, vp, vp, vp, sz, P(Shape), vp]
    L.im2win_conv_f16.argtypes = [vp, vp, vp, vp, sz, P(Shape), vp]
    L.im2win_check_status.argtypes = [vp, vp]
    L.im2win_layer_workspace_size.argtypes = [P(Shape), ctypes.c_int, P(sz)]
    L.im2win_layer_forward_host.argtypes = [vp, vp, vp, vp, sz, P(Shape), ctypes.c_int, vp]
    L.im2win_conv_f32_static.argtypes = [vp, vp, vp, P(Shape), vp]
    L.im2win_pack_filter.argtypes = [vp, vp, sz, P(Shape), ctypes.c_int, vp]
    L.im2win_conv_packed.argtypes = [vp, vp, vp, sz, P(Shape), ctypes.c_int, vp]
    L.im2win_conv_kernel_name.argtypes = [P(Shape), ctypes.c_int]
    L.im2win_nhwc_workspace_size.argtypes = [P(Shape), P(sz), P(sz), P(i32), P(i32), P(i32)]
    L.im2win_transform_nhwc.argtypes = [vp, ctypes.c_int, vp, P(Shape), vp]
    L.im2win_conv_f16_nhwc.argtypes = [vp, vp, vp, P(Epilogue), vp, sz, P(Shape), vp]
    L.im2win_pack_filter_nhwc.argtypes = [vp, vp, sz, P(Shape), vp]
    L.im2win_conv_packed_nhwc.argtypes = [vp, vp, P(Epilogue), vp, sz, P(Shape), vp]
    L.im2win_causal_conv1d.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp]
    L.im2win_linear_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, ctypes.c_int, vp]
    L.im2win_linear_attention_workspace_size.argtypes = [P(AttentionShape), ctypes.c_int, P(sz)]
    L.im2win_matvec_int4.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp]
    L.im2win_gated_delta_rule.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp]
    L.im2win_rms_norm.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp]
    L.im2win_matmul_int8.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp]
    for name in EXPORTS[1:]:
        getattr(L, name).restype = ctypes.c_int
    L.im2win_conv_kernel_name.restype = ctypes.c_char_p
    L.im2win_nhwc_kernel_name.argtypes = [P(Shape), P(Epilogue)]
    L.im2win_nhwc_kernel_name.restype = ctypes.c_char_p
    L.im2win_linear_attention_kernel_name.argtypes = [P(AttentionShape), ctypes.c_int]
    L.im2win_linear_attention_kernel_name.restype = ctypes.c_char_p
    L.im2win_matvec_int4_kernel_name.argtypes = [P(Int4Shape), ctypes.c_int]
    L.im2win_matvec_int4_kernel_name.restype = ctypes.c_char_p
    L.im2win_gated_delta_rule_kernel_name.argtypes = [P(DeltaShape), ctypes.c_int]
    L.im2win_gated_delta_rule_kernel_name.restype = ctypes.c_char_p
    L.im2win_matmul_int8_kernel_name.argtypes = [P(Int8Shape), ctypes.c_int]
    L.im2win_matmul_int8_kernel_name.restype = ctypes.c_char_p
    # the library looks at IM2WIN_DEBUG in its first plan: here, so that both sides see the same
    _debug = bool(os.environ.get("IM2WIN_DEBUG"))
    L.im2win_conv_kernel_name(ctypes.byref(Shape(1, 64, 1, 1, 1, 1, 1, 1, 0)), F32)
    _lib = L
    return L


def make_shape(N, C, H, W, Co, Kh, Kw, stride, pad) -> Shape:
    return Shape(int(N), int(C), int(H), int(W), int(Co), int(Kh), int(Kw), int(stride), int(pad))


def as_shape(shape) -> Shape:
    if isinstance(shape, Shape):
        return shape
    if isinstance(shape, dict):
        return make_shape(**shape)
    if hasattr(shape, "dims"):
        return make_shape(**shape.dims())
    return make_shape(*shape)


def _check(code: int, where: str) -> None:
    if code != 0:
        raise Im2winError(code, where)


# The handle of the current stream without a Stream object around it (0.2 us instead of 3.3; a call's launches take 3), and the
# current device without the look whether CUDA is initialised (there are CUDA tensors).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _dtype_code(t: torch.dtype) -> int:
    if t == torch.float32:
        return F32
    if t == torch.float16:
        return F16
    raise TypeError(f"unsupported dtype {t}")


_size_cache: dict = {}
_nhwc_size_cache: dict = {}


def im2win_workspace_size(shape, dtype: int) -> Tuple[int, int, int, int]:
    """Returns (window_bytes, scratch_bytes, Ho, Wo)."""
    return _sizes(as_shape(shape), dtype)[:4]


def _sizes(s: Shape, dtype: int) -> Tuple[int, ...]:
    """(window_bytes, scratch_bytes, Ho, Wo, elements of the input, the filter and the output)."""
    key = bytes(s)
    hit = _size_cache.get(key)
    if hit is not None and dtype in (F32, F16) and hit[dtype] is not None:     # (other codes are the library's to refuse)
        return hit[dtype]
    wb, sb = ctypes.c_size_t(), ctypes.c_size_t()
    ho, wo = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().im2win_workspace_size(ctypes.byref(s), dtype, ctypes.byref(wb), ctypes.byref(sb),
                                       ctypes.byref(ho), ctypes.byref(wo)), "im2win_workspace_size")
    out = (wb.value, sb.value, ho.value, wo.value, s.N * s.C * s.H * s.W, s.Co * s.C * s.Kh * s.Kw, s.N * s.Co * ho.value * wo.value)
    _remember(_size_cache, key, (out, hit[F16] if hit else None) if dtype == F32 else (hit[F32] if hit else None, out))
    return out


def _remember(cache, key, sizes) -> None:
    if _debug:
        return
    if len(cache) >= 4096:
        cache.clear()
    cache[key] = sizes


def im2win_conv_kernel_name(shape, dtype: int) -> str:
    """Name of the convolution kernel the library selects for the layer (for reports and tests)."""
    s = as_shape(shape)
    return lib().im2win_conv_kernel_name(ctypes.byref(s), dtype).decode()


def im2win_nhwc_kernel_name(shape, epilogue: Optional["Epilogue"] = None) -> str:
    """Name of the kernel im2win_conv_f16_nhwc selects for the layer and epilogue (for reports and tests)."""
    s = as_shape(shape)
    return lib().im2win_nhwc_kernel_name(ctypes.byref(s), None if epilogue is None else ctypes.byref(epilogue)).decode()


def im2win_transform(x: torch.Tensor, window: torch.Tensor, shape, stream=None) -> None:
    """x [N,C,H,W] -> window (flat tensor of window_bytes), both CUDA tensors of the same 2/4-byte dtype."""
    s = as_shape(shape)
    assert x.is_cuda and window.is_cuda and x.is_contiguous() and window.is_contiguous()
    dtype = x.dtype
    assert dtype == window.dtype
    code = _dtype_code(dtype)
    sizes = _sizes(s, code)
    assert x.numel() == sizes[4] and window.nbytes >= sizes[0]
    code = lib().im2win_transform(x.data_ptr(), window.data_ptr(), ctypes.byref(s), code, _stream(stream))
    if code:
        _check(code, "im2win_transform")


def _conv(fn_name: str, dtype: torch.dtype, code: int, window, filt, y, scratch, shape, stream):
    s = as_shape(shape)
    for t in (window, filt, y, scratch):
        assert t.is_cuda and t.is_contiguous()
    assert window.dtype == dtype and filt.dtype == dtype and y.dtype == torch.float32
    sizes = _sizes(s, code)
    assert window.nbytes >= sizes[0] and filt.numel() == sizes[5] and y.numel() == sizes[6]
    code = getattr(lib(), fn_name)(window.data_ptr(), filt.data_ptr(), y.data_ptr(), scratch.data_ptr(), scratch.nbytes,
                                   ctypes.byref(s), _stream(stream))
    if code:
        _check(code, fn_name)


def im2win_conv_f32(window, filter_oihw, y, scratch, shape, stream=None) -> None:
    _conv("im2win_conv_f32", torch.float32, F32, window, filter_oihw, y, scratch, shape, stream)


def im2win_conv_f16(window, filter_oihw, y, scratch, shape, stream=None) -> None:
    _conv("im2win_conv_f16", torch.float16, F16, window, filter_oihw, y, scratch, shape, stream)


def im2win_conv_f32_static(window, filter_oihw, y, shape, stream=None) -> None:
    """fp32 convolution for callers that cannot allocate device memory: the operation of im2win_conv_f32,
    always on CUDA cores, with the scratch in a fixed array inside the library (layers needing more than
    STATIC_SCRATCH_BYTES are rejected).  Calls that may overlap on the GPU must be serialised."""
    s = as_shape(shape)
    for t in (window, filter_oihw, y):
        assert t.is_cuda and t.is_contiguous() and t.dtype == torch.float32
    _check(lib().im2win_conv_f32_static(window.data_ptr(), filter_oihw.data_ptr(), y.data_ptr(),
                                        ctypes.byref(s), _stream(stream)), "im2win_conv_f32_static")


def im2win_pack_filter(filter_oihw, scratch, shape, stream=None) -> None:
    """Packs the filter into `scratch` once (static weights); im2win_conv_packed then reuses it."""
    s = as_shape(shape)
    assert filter_oihw.is_cuda and filter_oihw.is_contiguous() and scratch.is_cuda
    _check(lib().im2win_pack_filter(filter_oihw.data_ptr(), scratch.data_ptr(), scratch.nbytes,
                                    ctypes.byref(s), _dtype_code(filter_oihw.dtype), _stream(stream)),
           "im2win_pack_filter")


def im2win_conv_packed(window, y, scratch, shape, stream=None) -> None:
    """Convolution with the filter that im2win_pack_filter left in `scratch` (same shape and dtype)."""
    s = as_shape(shape)
    assert window.is_cuda and window.is_contiguous() and y.is_cuda and y.dtype == torch.float32 and scratch.is_cuda
    _check(lib().im2win_conv_packed(window.data_ptr(), y.data_ptr(), scratch.data_ptr(),
                                    scratch.nbytes, ctypes.byref(s),
                                    _dtype_code(window.dtype), _stream(stream)),
           "im2win_conv_packed")


def im2win_check_status(scratch: torch.Tensor, stream=None) -> None:
    """Blocks until the stream is idle; raises if a bounded device wait gave up."""
    _check(lib().im2win_check_status(scratch.data_ptr(), _stream(stream)), "im2win_check_status")


def im2win_layer_workspace_size(shape, dtype: int) -> int:
    s = as_shape(shape)
    n = ctypes.c_size_t()
    _check(lib().im2win_layer_workspace_size(ctypes.byref(s), dtype, ctypes.byref(n)), "im2win_layer_workspace_size")
    return n.value


def im2win_layer_forward_host(x_host: torch.Tensor, filter_host: torch.Tensor, y_host: torch.Tensor,
                              device_workspace: torch.Tensor, shape, stream=None) -> None:
    """Whole layer from (pinned) host tensors; y_host is float32 on the host.  Asynchronous."""
    s = as_shape(shape)
    assert not x_host.is_cuda and not filter_host.is_cuda and not y_host.is_cuda and device_workspace.is_cuda
    assert x_host.is_contiguous() and filter_host.is_contiguous() and y_host.is_contiguous()
    assert x_host.dtype == filter_host.dtype and y_host.dtype == torch.float32
    code = _dtype_code(x_host.dtype)
    _check(lib().im2win_layer_forward_host(x_host.data_ptr(), filter_host.data_ptr(), y_host.data_ptr(),
                                           device_workspace.data_ptr(),
                                           device_workspace.nbytes,
                                           ctypes.byref(s), code, _stream(stream)),
           "im2win_layer_forward_host")


# ------------------------------------------------------- channel-innermost (NHWC) form
def make_epilogue(bias: Optional[torch.Tensor] = None, relu: bool = False, out_dtype: torch.dtype = torch.float32,
                  out_layout: int = NCHW) -> Epilogue:
    if bias is not None:
        assert bias.is_cuda and bias.dtype == torch.float32 and bias.is_contiguous()
    return Epilogue(None if bias is None else bias.data_ptr(), int(bool(relu)), _dtype_code(out_dtype), int(out_layout))


def im2win_nhwc_workspace_size(shape) -> Tuple[int, int, int, int, int]:
    """Returns (window_bytes, scratch_bytes, Ho, Wo, Cp) of the NHWC form."""
    return _nhwc_sizes(as_shape(shape))


def _nhwc_sizes(s: Shape) -> Tuple[int, int, int, int, int]:
    key = bytes(s)
    hit = _nhwc_size_cache.get(key)
    if hit is not None:
        return hit
    wb, sb = ctypes.c_size_t(), ctypes.c_size_t()
    ho, wo, cp = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(lib().im2win_nhwc_workspace_size(ctypes.byref(s), ctypes.byref(wb), ctypes.byref(sb), ctypes.byref(ho),
                                            ctypes.byref(wo), ctypes.byref(cp)), "im2win_nhwc_workspace_size")
    out = (wb.value, sb.value, ho.value, wo.value, cp.value)
    _remember(_nhwc_size_cache, key, out)
    return out


def im2win_transform_nhwc(x: torch.Tensor, x_layout: int, window: torch.Tensor, shape, stream=None) -> None:
    """x (float16, [N,C,H,W] for NCHW or [N,H,W,C] for NHWC) -> NHWC window tensor (flat float16)."""
    s = as_shape(shape)
    assert x.is_cuda and window.is_cuda and x.is_contiguous() and window.is_contiguous()
    assert x.dtype == torch.float16 and window.dtype == torch.float16
    assert x.numel() == s.N * s.C * s.H * s.W and window.nbytes >= _nhwc_sizes(s)[0]
    code = lib().im2win_transform_nhwc(x.data_ptr(), int(x_layout), window.data_ptr(), ctypes.byref(s), _stream(stream))
    if code:
        _check(code, "im2win_transform_nhwc")


def _epi_ref(epilogue: Optional[Epilogue]):
    return None if epilogue is None else ctypes.byref(epilogue)


def im2win_conv_f16_nhwc(window, filter_oihw, y, scratch, shape, epilogue: Optional[Epilogue] = None, stream=None) -> None:
    s = as_shape(shape)
    for t in (window, filter_oihw, y, scratch):
        assert t.is_cuda and t.is_contiguous()
    assert window.dtype == torch.float16 and filter_oihw.dtype == torch.float16
    want = torch.float32 if epilogue is None or epilogue.out_dtype == F32 else torch.float16
    assert y.dtype == want
    _check(lib().im2win_conv_f16_nhwc(window.data_ptr(), filter_oihw.data_ptr(), y.data_ptr(), _epi_ref(epilogue),
                                      scratch.data_ptr(), scratch.nbytes, ctypes.byref(s),
                                      _stream(stream)), "im2win_conv_f16_nhwc")


def im2win_pack_filter_nhwc(filter_oihw, scratch, shape, stream=None) -> None:
    s = as_shape(shape)
    assert filter_oihw.is_cuda and filter_oihw.is_contiguous() and filter_oihw.dtype == torch.float16 and scratch.is_cuda
    _check(lib().im2win_pack_filter_nhwc(filter_oihw.data_ptr(), scratch.data_ptr(),
                                         scratch.nbytes, ctypes.byref(s), _stream(stream)),
           "im2win_pack_filter_nhwc")


def im2win_conv_packed_nhwc(window, y, scratch, shape, epilogue: Optional[Epilogue] = None, stream=None) -> None:
    s = as_shape(shape)
    assert window.is_cuda and window.dtype == torch.float16 and y.is_cuda and scratch.is_cuda
    _check(lib().im2win_conv_packed_nhwc(window.data_ptr(), y.data_ptr(), _epi_ref(epilogue), scratch.data_ptr(),
                                         scratch.nbytes, ctypes.byref(s), _stream(stream)),
           "im2win_conv_packed_nhwc")


def alloc_nhwc_buffers(shape, out_dtype: torch.dtype = torch.float32, out_layout: int = NCHW, device="cuda"):
    """Allocates (window, scratch, y) for one layer of the NHWC form with torch (device memory only)."""
    s = as_shape(shape)
    wb, sb, ho, wo, _ = im2win_nhwc_workspace_size(s)
    window = torch.empty(wb // 2, dtype=torch.float16, device=device)
    scratch = torch.empty(sb, dtype=torch.uint8, device=device)
    yshape = (s.N, s.Co, ho, wo) if out_layout == NCHW else (s.N, ho, wo, s.Co)
    y = torch.empty(yshape, dtype=out_dtype, device=device)
    return window, scratch, y


# ------------------------------------------------------- operators on token sequences
# Rows of tokens are given packed, as [tokens, ...] with `cu_seqlens`, or as [sequences, tokens of each, ...]; [tokens, ...] without
# `cu_seqlens` is one token of each of `tokens` sequences (the next token of a generation).  See include/im2win.h.
_SEQUENCE_DTYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}

# The structures above, as bytes: a call of one token is over in the time that a few ctypes structures take to fill (a whole call 13 us with
# them, 10 without).
_pack_sequences = struct.Struct("@3P").pack
_pack_conv1d = struct.Struct("@6i2q").pack
_pack_attention = struct.Struct("@8if5q").pack
_pack_int4 = struct.Struct("@4i2q").pack
_pack_delta = struct.Struct("@9if6q").pack
_pack_norm = struct.Struct("@2if4x4q").pack
_pack_int8 = struct.Struct("@3i4x2q").pack


def _sequence_dtype(dtype: torch.dtype) -> int:
    code = _SEQUENCE_DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}")
    return code


def _on_current_device(*tensors) -> None:
    """The kernels are launched on the current device: tensors of another one, or of the host, are refused."""
    device = -2
    for t in tensors:
        if t is not None and t.get_device() != device:
            at = t.get_device()
            if at < 0:
                raise ValueError("tensors have to be on a CUDA device")
            if device != -2 or at != _device():
                raise ValueError("tensors have to be on the current device (see torch.cuda.device)")
            device = at


def _row_stride(t: torch.Tensor, inner: int, name: str) -> int:
    """Elements from a row of t to the next one: its last `inner` (1 or 2) dimensions are a row, dense; those before them count rows."""
    shape = t.shape
    if t.is_contiguous():
        return shape[-1] if inner == 1 else shape[-1] * shape[-2]
    stride = t.stride()
    width = shape[-1]
    if stride[-1] != 1 and width != 1:
        raise ValueError(f"{name}: the elements of a row have to lie one behind the other")
    if inner == 2:
        if shape[-2] != 1 and stride[-2] != width:
            raise ValueError(f"{name}: the heads of a row have to lie one behind the other")
        width *= shape[-2]
    n = len(shape) - inner
    if n == 2:
        if shape[0] > 1 and shape[1] > 1:
            if stride[0] != shape[1] * stride[1]:
                raise ValueError(f"{name}: the sequences have to lie one behind the other")
            return stride[1]
        return stride[1] if shape[1] > 1 else stride[0] if shape[0] > 1 else width
    return stride[0] if shape[0] > 1 else width


def _take_sequences(rows, cu_seqlens, slots, resume, state, state_out):
    """(tokens, sequences, states in a pool, im2win_sequences as bytes or None) for tensors with the leading dimensions `rows`."""
    pool = 0
    if cu_seqlens is not None:
        if len(rows) != 1:
            raise ValueError("with cu_seqlens the tokens are the one leading dimension")
        if cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2 or not cu_seqlens.is_contiguous():
            raise ValueError("cu_seqlens: sequences + 1 int32 values")
        tokens, sequences = rows[0], cu_seqlens.numel() - 1
    else:
        sequences = rows[0]
        tokens = sequences if len(rows) == 1 else sequences * rows[1]
        if sequences < 1:
            raise ValueError("there has to be a sequence")
    if tokens >= 1 << 31:
        raise ValueError("fewer than 2^31 tokens")
    if state is not None:
        pool = state.shape[0]
        if pool < 1 or not state.is_contiguous():
            raise ValueError("state has to be contiguous, and to hold a state")
    if state_out is not None and state_out is not state:
        held = state_out.shape[0]
        if held < 1 or not state_out.is_contiguous() or (pool and held != pool):
            raise ValueError("state_out has to be contiguous, and to hold as many states as state")
        pool = held
    if slots is not None:
        if slots.dtype != torch.int32 or slots.dim() != 1 or slots.numel() != sequences or not slots.is_contiguous():
            raise ValueError("slots: an int32 value for each sequence")
        pool = pool or 0x7fffffff
    elif pool and pool < sequences:
        raise ValueError("the pool has fewer states than there are sequences")
    if resume is not None and (resume.dtype not in (torch.bool, torch.uint8) or resume.dim() != 1 or resume.numel() != sequences
                               or not resume.is_contiguous()):
        raise ValueError("resume: a flag for each sequence")
    if cu_seqlens is None and slots is None and resume is None:
        return tokens, sequences, pool, None
    return tokens, sequences, pool, _pack_sequences(_ptr(cu_seqlens) or 0, _ptr(slots) or 0, _ptr(resume) or 0)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def im2win_causal_conv1d(x, weight, y, bias=None, silu: bool = False, state=None, state_out=None, cu_seqlens=None, slots=None,
                         resume=None, stream=None) -> None:
    """Causal depthwise convolution along the tokens into y: x and y [tokens, channels] or [sequences, tokens, channels], weight
    [channels, taps], bias float32 [channels], state and state_out [slots, taps - 1, channels] (may be one tensor)."""
    dtype = x.dtype
    code = _sequence_dtype(dtype)
    _on_current_device(x, weight, y, bias, state, state_out, cu_seqlens, slots, resume)
    shape = x.shape
    if not 2 <= len(shape) <= 3 or y.shape != shape:
        raise ValueError("x and y: [tokens, channels] or [sequences, tokens, channels]")
    channels = shape[-1]
    if weight.dim() != 2 or weight.shape[0] != channels or not weight.is_contiguous():
        raise ValueError("weight: [channels, taps], contiguous")
    taps = weight.shape[1]
    if weight.dtype != dtype or y.dtype != dtype:
        raise ValueError("x, weight and y have to be of one dtype")
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != (channels,) or not bias.is_contiguous()):
        raise ValueError("bias: [channels] of float32")
    for p in (state, state_out):
        if p is not None and (p.dtype != dtype or p.dim() != 3 or p.shape[1] != taps - 1 or p.shape[2] != channels):
            raise ValueError("state and state_out: [slots, taps - 1, channels] of x's dtype")
    tokens, sequences, pool, seqs = _take_sequences(shape[:-1], cu_seqlens, slots, resume, state, state_out)
    sizes = _pack_conv1d(tokens, sequences, pool, channels, taps, 1 if silu else 0, _row_stride(x, 1, "x"), _row_stride(y, 1, "y"))
    if taps == 1:                                            # nothing is carried
        state = state_out = None
    code = (_lib or lib()).im2win_causal_conv1d(x.data_ptr(), weight.data_ptr(), _ptr(bias), y.data_ptr(), _ptr(state), _ptr(state_out), seqs,
                                                sizes, code, _stream(stream))
    if code:
        _check(code, "im2win_causal_conv1d")


def make_attention_shape(tokens, sequences, heads, qk_heads, dk, dv, max_len=0) -> AttentionShape:
    """The sizes that im2win_linear_attention's workspace depends on (all of them: fewer tokens may need more of it)."""
    return AttentionShape(int(tokens), int(sequences), 0, int(max_len), int(heads), int(qk_heads), int(dk), int(dv), 1.0, 0, 0, 0, 0, 0)


def im2win_linear_attention_workspace_size(shape: AttentionShape, dtype: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().im2win_linear_attention_workspace_size(ctypes.byref(shape), dtype, ctypes.byref(n)),
           "im2win_linear_attention_workspace_size")
    return n.value


def im2win_linear_attention_kernel_name(shape: AttentionShape, dtype: int) -> str:
    """How im2win_linear_attention runs these sizes (for reports and tests)."""
    return lib().im2win_linear_attention_kernel_name(ctypes.byref(shape), dtype).decode()


def alloc_attention_workspace(shape: AttentionShape, dtype: torch.dtype, device="cuda") -> torch.Tensor:
    """A workspace for im2win_linear_attention, with torch (device memory only)."""
    return torch.empty(im2win_linear_attention_workspace_size(shape, _sequence_dtype(dtype)), dtype=torch.uint8, device=device)


def im2win_linear_attention(q, k, v, log_decay, o, workspace, scale: float = 1.0, state=None, state_out=None, cu_seqlens=None,
                            slots=None, resume=None, max_len: int = 0, stream=None) -> None:
    """Linear attention with a decay for each head into o: q and k [tokens, qk_heads, dk] or [sequences, tokens, qk_heads, dk], v and o
    the same with heads and dv, log_decay float32 [tokens, heads] (or [sequences, tokens, heads]) or [heads], state and state_out float32
    [slots, heads, dk, dv] (may be one tensor), workspace from alloc_attention_workspace for these sizes and max_len."""
    dtype = q.dtype
    code = _sequence_dtype(dtype)
    _on_current_device(q, k, v, log_decay, o, workspace, state, state_out, cu_seqlens, slots, resume)
    if k.dtype != dtype or v.dtype != dtype or o.dtype != dtype:
        raise ValueError("q, k, v and o have to be of one dtype")
    qs, vs = q.shape, v.shape
    if not 3 <= len(qs) <= 4 or k.shape != qs or o.shape != vs or vs[:-2] != qs[:-2]:
        raise ValueError("q and k: [..., tokens, qk_heads, dk], v and o: [..., tokens, heads, dv]")
    qk_heads, dk = qs[-2:]
    heads, dv = vs[-2:]
    gs = log_decay.shape
    if log_decay.dtype != torch.float32 or (gs != vs[:-1] and gs != (heads,)):
        raise ValueError("log_decay: [..., tokens, heads] or [heads] of float32")
    for p in (state, state_out):
        if p is not None and (p.dtype != torch.float32 or p.dim() != 4 or p.shape[1] != heads or p.shape[2] != dk or p.shape[3] != dv):
            raise ValueError("state and state_out: [slots, heads, dk, dv] of float32")
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous, of uint8")
    tokens, sequences, pool, seqs = _take_sequences(qs[:-2], cu_seqlens, slots, resume, state, state_out)
    if tokens > 0 and len(gs) > 1 and log_decay.is_contiguous():
        decay_stride = heads
    elif len(gs) == 1 or (tokens > 1 and all(n == 1 or step == 0 for n, step in zip(gs[:-1], log_decay.stride()))):
        decay_stride = 0                                     # one decay for each head (it may be an expanded view)
        if heads > 1 and log_decay.stride(-1) != 1:
            raise ValueError("log_decay: the heads have to lie one behind the other")
    else:
        decay_stride = _row_stride(log_decay, 1, "log_decay")
    sizes = _pack_attention(tokens, sequences, pool, max_len, heads, qk_heads, dk, dv, scale, _row_stride(q, 2, "q"), _row_stride(k, 2, "k"),
                            _row_stride(v, 2, "v"), _row_stride(o, 2, "o"), decay_stride)
    code = (_lib or lib()).im2win_linear_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), o.data_ptr(), _ptr(state),
                                                   _ptr(state_out), seqs, workspace.data_ptr(), workspace.numel(), sizes, code,
                                                   _stream(stream))
    if code:
        _check(code, "im2win_linear_attention")


def im2win_matvec_int4(x, weight, scales, y, group: int, zeros=None, bias=None, stream=None) -> None:
    """A few rows times a matrix of 4-bit weights into y: x [M, K], weight uint8 [N, (K + 1) // 2], scales [N, ceil(K / group)], zeros
    uint8 of that shape, bias float32 [N], y [M, N]."""
    dtype = x.dtype
    code = _sequence_dtype(dtype)
    _on_current_device(x, weight, scales, y, zeros, bias)
    if x.dim() != 2 or y.dim() != 2 or x.shape[0] != y.shape[0] or y.dtype != dtype:
        raise ValueError("x: [M, K], y: [M, N] of one dtype")
    (m, k), n = x.shape, y.shape[1]
    if m < 1 or n < 1 or k < 1 or group < 1:
        raise ValueError("M, N, K and group have to be positive")
    if weight.dtype != torch.uint8 or weight.shape != (n, (k + 1) // 2) or not weight.is_contiguous():
        raise ValueError("weight: [N, (K + 1) // 2] of uint8")
    groups = (n, -(-k // group))
    if scales.dtype != dtype or scales.shape != groups or not scales.is_contiguous():
        raise ValueError("scales: [N, ceil(K / group)] of x's dtype")
    if zeros is not None and (zeros.dtype != torch.uint8 or zeros.shape != groups or not zeros.is_contiguous()):
        raise ValueError("zeros: [N, ceil(K / group)] of uint8")
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != (n,) or not bias.is_contiguous()):
        raise ValueError("bias: [N] of float32")
    sizes = _pack_int4(m, n, k, group, _row_stride(x, 1, "x"), _row_stride(y, 1, "y"))
    code = (_lib or lib()).im2win_matvec_int4(x.data_ptr(), weight.data_ptr(), scales.data_ptr(), _ptr(zeros), _ptr(bias), y.data_ptr(), sizes,
                                              code, _stream(stream))
    if code:
        _check(code, "im2win_matvec_int4")


def im2win_matvec_int4_kernel_name(m: int, n: int, k: int, group: int, dtype: int, x_stride: int = 0) -> str:
    """How im2win_matvec_int4 runs these sizes where tensors start on 16-byte boundaries (for reports and tests)."""
    return lib().im2win_matvec_int4_kernel_name(ctypes.byref(Int4Shape(m, n, k, group, x_stride or k, n)), dtype).decode()


def make_delta_shape(tokens, sequences, heads, qk_heads, dk, dv, max_len=0) -> DeltaShape:
    """The sizes that im2win_gated_delta_rule_kernel_name looks at."""
    return DeltaShape(int(tokens), int(sequences), 0, int(max_len), int(heads), int(qk_heads), int(dk), int(dv), 0, 1.0, 0, 0, 0, 0, 0, 0)


def im2win_gated_delta_rule_kernel_name(shape: DeltaShape, dtype: int) -> str:
    """How im2win_gated_delta_rule runs these sizes (for reports and tests)."""
    return lib().im2win_gated_delta_rule_kernel_name(ctypes.byref(shape), dtype).decode()


def _by_token_or_head(t, heads: int, rows, tokens: int, name: str) -> int:
    """Floats from a row of t ([..., tokens, heads], or [heads]) to the next one; 0: one value for each head."""
    shape = t.shape
    if t.dtype != torch.float32 or (shape != rows and shape != (heads,)):
        raise ValueError(f"{name}: [..., tokens, heads] or [heads] of float32")
    if tokens > 0 and len(shape) > 1 and t.is_contiguous():
        return heads
    if len(shape) == 1 or (tokens > 1 and all(n == 1 or step == 0 for n, step in zip(shape[:-1], t.stride()))):
        if heads > 1 and t.stride(-1) != 1:                  # (one value for each head may be an expanded view)
            raise ValueError(f"{name}: the heads have to lie one behind the other")
        return 0
    return _row_stride(t, 1, name)


def im2win_gated_delta_rule(q, k, v, log_decay, beta, o, scale: float = 1.0, normalize: bool = False, state=None, state_out=None,
                            cu_seqlens=None, slots=None, resume=None, max_len: int = 0, stream=None) -> None:
    """The gated delta rule into o: q and k [tokens, qk_heads, dk] or [sequences, tokens, qk_heads, dk], v and o the same with heads and dv,
    log_decay and beta float32 [tokens, heads] (or [sequences, tokens, heads]) or [heads], state and state_out float32 [slots, heads, dk,
    dv] (may be one tensor)."""
    dtype = q.dtype
    code = _sequence_dtype(dtype)
    _on_current_device(q, k, v, log_decay, beta, o, state, state_out, cu_seqlens, slots, resume)
    if k.dtype != dtype or v.dtype != dtype or o.dtype != dtype:
        raise ValueError("q, k, v and o have to be of one dtype")
    qs, vs = q.shape, v.shape
    if not 3 <= len(qs) <= 4 or k.shape != qs or o.shape != vs or vs[:-2] != qs[:-2]:
        raise ValueError("q and k: [..., tokens, qk_heads, dk], v and o: [..., tokens, heads, dv]")
    qk_heads, dk = qs[-2:]
    heads, dv = vs[-2:]
    for p in (state, state_out):
        if p is not None and (p.dtype != torch.float32 or p.dim() != 4 or p.shape[1] != heads or p.shape[2] != dk or p.shape[3] != dv):
            raise ValueError("state and state_out: [slots, heads, dk, dv] of float32")
    tokens, sequences, pool, seqs = _take_sequences(qs[:-2], cu_seqlens, slots, resume, state, state_out)
    sizes = _pack_delta(tokens, sequences, pool, max_len, heads, qk_heads, dk, dv, 1 if normalize else 0, scale, _row_stride(q, 2, "q"),
                        _row_stride(k, 2, "k"), _row_stride(v, 2, "v"), _row_stride(o, 2, "o"),
                        _by_token_or_head(log_decay, heads, vs[:-1], tokens, "log_decay"), _by_token_or_head(beta, heads, vs[:-1], tokens, "beta"))
    code = (_lib or lib()).im2win_gated_delta_rule(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), beta.data_ptr(), o.data_ptr(),
                                                   _ptr(state), _ptr(state_out), seqs, sizes, code, _stream(stream))
    if code:
        _check(code, "im2win_gated_delta_rule")


def im2win_rms_norm(x, weight, y, scales=None, residual=None, residual_out=None, eps: float = 1e-6, stream=None) -> None:
    """Root-mean-square norm of x (+ residual, their sum into residual_out) into y: all [rows, channels] of one dtype, weight [channels] or
    None.  With scales, float32 [rows], y is int8 and y * scales the normed rows."""
    dtype = x.dtype
    code = _sequence_dtype(dtype)
    _on_current_device(x, weight, y, scales, residual, residual_out)
    shape = x.shape
    if len(shape) != 2 or y.shape != shape or shape[1] < 1:
        raise ValueError("x and y: [rows, channels]")
    rows, channels = shape
    if y.dtype != (dtype if scales is None else torch.int8):
        raise ValueError("y: of x's dtype, or with scales of int8")
    if scales is not None and (scales.dtype != torch.float32 or scales.shape != (rows,) or not scales.is_contiguous()):
        raise ValueError("scales: [rows] of float32")
    if weight is not None and (weight.dtype != dtype or weight.shape != (channels,) or not weight.is_contiguous()):
        raise ValueError("weight: [channels] of x's dtype")
    if residual is None and residual_out is not None:
        raise ValueError("residual_out goes with a residual")
    for t in (residual, residual_out):
        if t is not None and (t.dtype != dtype or t.shape != shape):
            raise ValueError("residual and residual_out: like x")
    sizes = _pack_norm(rows, channels, eps, _row_stride(x, 1, "x"), 0 if residual is None else _row_stride(residual, 1, "residual"),
                       0 if residual_out is None else _row_stride(residual_out, 1, "residual_out"), _row_stride(y, 1, "y"))
    code = (_lib or lib()).im2win_rms_norm(x.data_ptr(), _ptr(residual), _ptr(weight), _ptr(residual_out), y.data_ptr(), _ptr(scales), sizes, code,
                                           _stream(stream))
    if code:
        _check(code, "im2win_rms_norm")


def im2win_matmul_int8(x, x_scales, weight, scales, y, bias=None, stream=None) -> None:
    """Rows times a matrix in 8-bit integers into y: x int8 [M, K], x_scales float32 [M], weight int8 [N, K], scales float32 [N], bias float32
    [N], y [M, N]."""
    code = _sequence_dtype(y.dtype)
    _on_current_device(x, x_scales, weight, scales, y, bias)
    if x.dim() != 2 or y.dim() != 2 or x.shape[0] != y.shape[0] or x.dtype != torch.int8:
        raise ValueError("x: int8 [M, K], y: [M, N]")
    (m, k), n = x.shape, y.shape[1]
    if n < 1 or k < 1:
        raise ValueError("N and K have to be positive")
    if weight.dtype != torch.int8 or weight.shape != (n, k) or not weight.is_contiguous():
        raise ValueError("weight: [N, K] of int8, contiguous")
    for t, size, name in ((x_scales, m, "x_scales: [M]"), (scales, n, "scales: [N]"), (bias, n, "bias: [N]")):
        if (t is not None or name[0] != "b") and (t.dtype != torch.float32 or t.shape != (size,) or not t.is_contiguous()):
            raise ValueError(name + " of float32")
    sizes = _pack_int8(m, n, k, _row_stride(x, 1, "x"), _row_stride(y, 1, "y"))
    code = (_lib or lib()).im2win_matmul_int8(x.data_ptr(), x_scales.data_ptr(), weight.data_ptr(), scales.data_ptr(), _ptr(bias), y.data_ptr(),
                                              sizes, code, _stream(stream))
    if code:
        _check(code, "im2win_matmul_int8")


def im2win_matmul_int8_kernel_name(m: int, n: int, k: int, dtype: int, x_stride: int = 0) -> str:
    """How im2win_matmul_int8 runs these sizes where tensors start on 16-byte boundaries (for reports and tests)."""
    return lib().im2win_matmul_int8_kernel_name(ctypes.byref(Int8Shape(m, n, k, x_stride or k, n)), dtype).decode()


# ---------------------------------------------------------------- conveniences
def alloc_layer_buffers(shape, dtype: torch.dtype, device="cuda"):
    """Allocates (window, scratch, y) for one layer with torch (device memory only)."""
    s = as_shape(shape)
    code = _dtype_code(dtype)
    wb, sb, ho, wo = im2win_workspace_size(s, code)
    esize = 4 if code == F32 else 2
    window = torch.empty(max(wb // esize, 1), dtype=dtype, device=device)
    scratch = torch.empty(sb, dtype=torch.uint8, device=device)
    y = torch.empty((s.N, s.Co, ho, wo), dtype=torch.float32, device=device)
    return window, scratch, y


def conv2d_im2win(x: torch.Tensor, filter_oihw: torch.Tensor, stride: int, pad: int, stream=None) -> torch.Tensor:
    """Transform + convolution through the C ABI for CUDA tensors of float32 or float16; returns y (float32)."""
    N, C, H, W = x.shape
    Co, C2, Kh, Kw = filter_oihw.shape
    assert C == C2
    dtype = x.dtype
    code = _dtype_code(dtype)
    assert x.is_cuda and filter_oihw.is_cuda and filter_oihw.dtype == dtype
    s = make_shape(N, C, H, W, Co, Kh, Kw, stride, pad)
    sizes = _sizes(s, code)
    x = x.contiguous()
    filter_oihw = filter_oihw.contiguous()
    # window and scratch in one buffer (an allocation takes as long as half a launch)
    scratch_at = (sizes[0] + 255) & ~255
    buffer = x.new_empty((scratch_at + sizes[1],), dtype=torch.uint8)
    y = x.new_empty((N, Co, sizes[2], sizes[3]), dtype=torch.float32)
    L, window, shape, queue = lib(), buffer.data_ptr(), ctypes.byref(s), _stream(stream)
    _check(L.im2win_transform(x.data_ptr(), window, shape, code, queue), "im2win_transform")
    name = "im2win_conv_f32" if code == F32 else "im2win_conv_f16"
    _check(getattr(L, name)(window, filter_oihw.data_ptr(), y.data_ptr(), window + scratch_at, sizes[1], shape, queue), name)
    return y
