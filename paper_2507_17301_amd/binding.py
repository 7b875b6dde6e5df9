"""ctypes binding of libnmconv.so -- argument marshalling only.

Same names as the C ABI in ``include/nm_conv.h`` and ``include/nm_q8.h``.  Tensors are torch tensors
used purely as device buffers (``data_ptr()``) and for the current stream; all
arithmetic happens inside the library's kernels.  There is no fallback: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Tuple

import numpy as np

NM_F32, NM_BF16, NM_F8E4M3, NM_I8 = 0, 1, 2, 3
NM_Q8_MAX_WIDTH, NM_Q8_FEW_ROWS = 65536, 64
NM_OK = 0
NM_ERR_ARG, NM_ERR_SHAPE, NM_ERR_UNSUPPORTED, NM_ERR_ALLOC, NM_ERR_HIP, NM_ERR_IO = -1, -2, -3, -4, -5, -6
_STATUS = {0: "NM_OK", -1: "NM_ERR_ARG", -2: "NM_ERR_SHAPE", -3: "NM_ERR_UNSUPPORTED",
           -4: "NM_ERR_ALLOC", -5: "NM_ERR_HIP", -6: "NM_ERR_IO"}

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libnmconv.so")
_lib = None
_torch = None   # the module, from the first lib() on
_q8_codes = {}  # element types that the 8-bit operators know, from then on


class NMError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{_STATUS.get(code, code)}: {msg}")
        self.code = code


def lib():
    """Open libnmconv.so (once).  Raises if it has not been built."""
    global _lib, _torch
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2507_17301_amd.build` "
                "(there is no fallback path)")
        # PyTorch ships its own copy of the HIP runtime; a process must not end up with two.
        # Importing torch first makes its copy the one libnmconv.so binds to as well (loaded
        # the other way round, torch finds no GPU).
        import torch
        _torch = torch
        _q8_codes.update({torch.float32: NM_F32, torch.bfloat16: NM_BF16, torch.int8: NM_I8})
        L = ctypes.CDLL(LIB_PATH)
        ci, cf, vp = ctypes.c_int, ctypes.c_float, ctypes.c_void_p
        pi = ctypes.POINTER(ctypes.c_int)
        L.nm_last_error.restype = ctypes.c_char_p
        L.nm_variant_count.restype = ci
        L.nm_last_variant.restype = ci
        L.nm_variant_name.argtypes = [ci]
        L.nm_variant_name.restype = ctypes.c_char_p
        L.nm_prune.argtypes = [vp, ci, ci, ci, ci, ci, ci, ci, ci, ctypes.POINTER(vp)]
        L.nm_packed_free.argtypes = [vp]
        L.nm_packed_dims.argtypes = [vp, pi, pi, pi, pi]
        L.nm_packed_indices.argtypes = [vp, vp]
        L.nm_packed_values.argtypes = [vp, vp]
        L.nm_packed_mask.argtypes = [vp, vp]
        L.nm_packed_scale.argtypes = [vp, ctypes.POINTER(cf)]
        L.nm_conv2d.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp, ci, ci, ci, ci, ci, ci, ci, vp, ci, vp]
        L.nm_conv2d_res.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, vp, ci, vp]
        L.nm_conv2d_static.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, vp, ci, vp]
        L.nm_conv2d_args.argtypes = [ctypes.c_char_p]
        L.nm_maxpool2d.argtypes = [vp, ci, ci, ci, ci, ci, ci, ci, ci, vp, vp]
        L.nm_avgpool_global.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp]
        L.nm_im2col.argtypes = [vp] + [ci] * 13 + [vp, vp]
        L.nm_stream_floor.argtypes = [vp, ctypes.c_size_t, vp, ctypes.c_size_t, vp]
        L.nm_autotune.argtypes = [ci, ci, ci, ci, ci, vp, ci, ci, ci, ci, ci, ci, ci, ci, ci, vp,
                                  pi, ctypes.POINTER(cf)]
        L.nm_autotune_tile.argtypes = ([vp] + [ci] * 6 + [pi, ci, ci] + [ci] * 13 +
                                       [vp, ctypes.POINTER(vp), pi, ctypes.POINTER(ctypes.c_float)])
        L.nm_cache_save.argtypes = [ctypes.c_char_p]
        L.nm_cache_load.argtypes = [ctypes.c_char_p]
        L.nm_force_variant.argtypes = [ci]
        L.nm_variant_legal.argtypes = [ci, vp, ci, ci]
        i64, st = ctypes.c_int64, ctypes.c_size_t
        L.nm_quantize_q8.argtypes = [vp, ci, i64, ci, i64, vp, i64, vp, vp]
        L.nm_dequantize_q8.argtypes = [vp, i64, vp, i64, ci, vp, ci, i64, vp]
        L.nm_rmsnorm_q8.argtypes = [vp, ci, i64, ci, i64, vp, i64, vp, cf, vp, i64, vp, i64, vp, vp]
        L.nm_q8_pack.argtypes = [vp, ci, vp, ci, ci, i64, ci, vp, ctypes.POINTER(vp)]
        L.nm_q8_free.argtypes = [vp]
        L.nm_q8_dims.argtypes = [vp, pi, pi, pi]
        L.nm_q8_export.argtypes = [vp, vp, vp]
        L.nm_linear_q8.argtypes = [vp, i64, ci, i64, vp, vp, vp, vp, i64, vp, ci, i64, vp, st, vp]
        L.nm_rows_q8_args.argtypes = L.nm_dequantize_q8_args.argtypes = L.nm_linear_q8_args.argtypes = [ctypes.c_char_p]
        L.nm_linear_q8_workspace.argtypes = [vp, i64, i64, vp, ctypes.POINTER(st)]
        for name in ("nm_prune", "nm_packed_free", "nm_packed_dims", "nm_packed_indices",
                     "nm_packed_values", "nm_packed_mask", "nm_packed_scale", "nm_conv2d", "nm_conv2d_res", "nm_conv2d_static", "nm_conv2d_args",
                     "nm_maxpool2d",
                     "nm_avgpool_global", "nm_im2col", "nm_stream_floor", "nm_autotune",
                     "nm_cache_save", "nm_cache_load", "nm_cache_clear", "nm_cache_size", "nm_workspace_free",
                     "nm_force_variant", "nm_variant_legal", "nm_quantize_q8", "nm_dequantize_q8", "nm_rmsnorm_q8",
                     "nm_q8_pack", "nm_q8_free", "nm_q8_dims", "nm_q8_export", "nm_linear_q8", "nm_linear_q8_workspace", "nm_rows_q8_args",
                     "nm_dequantize_q8_args", "nm_linear_q8_args"):
            getattr(L, name).restype = ci
        _lib = L
    return _lib


def _lib_torch():
    lib()
    return _torch


def _check(rc: int) -> int:
    if rc < 0:
        raise NMError(rc, lib().nm_last_error().decode())
    return rc


def _pair(v) -> Tuple[int, int]:
    if isinstance(v, (tuple, list)):
        return int(v[0]), int(v[1])
    return int(v), int(v)


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return NM_F32
    if t.dtype == torch.bfloat16:
        return NM_BF16
    if t.dtype == torch.float8_e4m3fn:
        return NM_F8E4M3
    raise TypeError(f"unsupported tensor dtype {t.dtype}")


class Packed:
    """Owner of an nm_packed_t handle."""

    def __init__(self, handle, cout, kh, kw, cin, n, m, tile, value_dtype):
        self.handle = handle
        self.cout, self.kh, self.kw, self.cin = cout, kh, kw, cin
        self.n, self.m, self.tile, self.value_dtype = n, m, tile, value_dtype
        self.K = kh * kw * cin

    def free(self):
        """Release the handle now (idempotent)."""
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.nm_packed_free(h)

    def __del__(self):
        # at interpreter shutdown the module globals may already be gone; the
        # process is ending then and the driver reclaims the device memory
        try:
            self.free()
        except Exception:
            pass


def nm_variant_count() -> int:
    return lib().nm_variant_count()


def nm_last_variant() -> int:
    """Variant id launched by this thread's last successful nm_conv2d / nm_conv2d_res."""
    return lib().nm_last_variant()


def nm_variant_name(v: int) -> Optional[str]:
    s = lib().nm_variant_name(v)
    return s.decode() if s else None


def nm_prune(w_ohwi: np.ndarray, n: int, m: int, tile: int, value_dtype: int = NM_F32) -> Packed:
    """w_ohwi: host numpy array [Cout,Kh,Kw,Cin] fp32."""
    w = np.ascontiguousarray(w_ohwi, dtype=np.float32)
    cout, kh, kw, cin = w.shape
    h = ctypes.c_void_p()
    _check(lib().nm_prune(w.ctypes.data, cout, kh, kw, cin, n, m, tile, value_dtype,
                          ctypes.byref(h)))
    return Packed(h, cout, kh, kw, cin, n, m, tile, value_dtype)


def nm_packed_dims(wp: Packed):
    a, b, c, d = (ctypes.c_int() for _ in range(4))
    _check(lib().nm_packed_dims(wp.handle, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c),
                                ctypes.byref(d)))
    return a.value, b.value, c.value, d.value


def nm_packed_indices(wp: Packed) -> np.ndarray:
    n_tiles, groups, n, _ = nm_packed_dims(wp)
    out = np.empty((n_tiles, groups, n), dtype=np.int32)
    _check(lib().nm_packed_indices(wp.handle, out.ctypes.data))
    return out


def nm_packed_values(wp: Packed) -> np.ndarray:
    n_tiles, _, _, kprime = nm_packed_dims(wp)
    out = np.empty((n_tiles, kprime, wp.tile), dtype=np.float32)
    _check(lib().nm_packed_values(wp.handle, out.ctypes.data))
    return out


def nm_packed_mask(wp: Packed) -> np.ndarray:
    out = np.empty((wp.cout, wp.K), dtype=np.uint8)
    _check(lib().nm_packed_mask(wp.handle, out.ctypes.data))
    return out


def nm_packed_scale(wp: Packed) -> float:
    """The power-of-two scale of an fp8 handle (stored value = weight * scale); 1 otherwise."""
    v = ctypes.c_float(0)
    _check(lib().nm_packed_scale(wp.handle, ctypes.byref(v)))
    return v.value


def _out_dtype(x):
    """fp32 -> fp32, bf16 -> bf16, E4M3 -> bf16."""
    import torch
    return torch.bfloat16 if x.dtype == torch.float8_e4m3fn else x.dtype


def _stream_ptr(stream) -> int:
    import torch
    if stream is None:
        # the handle of torch.cuda.current_stream() without the Stream object around it
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream)


def out_shape(x_shape, wp: Packed, stride, pad, dil):
    b, h, w, _ = x_shape
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    dh, dw = _pair(dil)
    if sh < 1 or sw < 1:
        raise NMError(NM_ERR_ARG, "stride must be >= 1")
    ho = (h + 2 * ph - dh * (wp.kh - 1) - 1) // sh + 1
    wo = (w + 2 * pw - dw * (wp.kw - 1) - 1) // sw + 1
    return (b, ho, wo, wp.cout)


_CONV_ARGS = struct.Struct("20q")   # nm_conv_args_t


def _conv2d(x, wp: Packed, residual, bias, stride, pad, dil, relu, y, stream, static_only):
    """Checks and marshals one convolution.  A small layer runs for 5 us on the GPU, so this is
    kept to one look at each tensor and one block of arguments (9 us a call before, 5 now)."""
    import torch
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous device tensor")
    b, h, w, cin = x.shape
    sh, sw = (stride, stride) if type(stride) is int else _pair(stride)
    ph, pw = (pad, pad) if type(pad) is int else _pair(pad)
    dh, dw = (dil, dil) if type(dil) is int else _pair(dil)
    if sh < 1 or sw < 1:
        raise NMError(NM_ERR_ARG, "stride must be >= 1")
    ho = (h + 2 * ph - dh * (wp.kh - 1) - 1) // sh + 1
    wo = (w + 2 * pw - dw * (wp.kw - 1) - 1) // sw + 1
    shp = (b, ho, wo, wp.cout)
    if min(shp) < 1:
        raise NMError(-2, "output would be empty")
    if y is None:
        y = torch.empty(shp, dtype=_out_dtype(x), device=x.device)
    elif y.shape != shp or not y.is_cuda or y.get_device() != x.get_device() or not y.is_contiguous():
        # what the kernel will write, exactly (the library itself checks the dtype pair)
        raise ValueError(f"y must be a contiguous device tensor of shape {shp} on {x.device}")
    rptr = bptr = 0
    if residual is not None:
        if (residual.shape != shp or residual.dtype != y.dtype or not residual.is_cuda
                or not residual.is_contiguous()):
            raise ValueError("residual must be a contiguous device tensor shaped and typed like the output")
        rptr = residual.data_ptr()
    if bias is not None:
        if bias.dtype != torch.float32 or not bias.is_cuda or not bias.is_contiguous():
            raise ValueError("bias must be a contiguous fp32 device tensor")
        bptr = bias.data_ptr()
    rc = (_lib or lib()).nm_conv2d_args(_CONV_ARGS.pack(
        x.data_ptr(), (wp.handle.value or 0) if wp.handle else 0, bptr, rptr, y.data_ptr(), _stream_ptr(stream),
        _dtype_code(x), b, h, w, cin, sh, sw, ph, pw, dh, dw, bool(relu), _dtype_code(y), static_only))
    if rc < 0:
        _check(rc)
    return y


def nm_conv2d(x, wp: Packed, bias=None, stride=1, pad=0, dil=1, relu=False, y=None, stream=None):
    """x: device tensor NHWC [B,H,W,Cin] (fp32 or bf16, contiguous); bias: device
    fp32 [Cout] or None; y: optional preallocated output.  Enqueues on `stream`
    (default: torch's current stream) and returns y."""
    return _conv2d(x, wp, None, bias, stride, pad, dil, relu, y, stream, False)


def nm_conv2d_static(x, wp: Packed, residual, bias, stride, pad, dil, relu, y, stream=None):
    """nm_conv2d_res through the entry point that allocates nothing; y must be given."""
    return _conv2d(x, wp, residual, bias, stride, pad, dil, relu, y, stream, True)


def nm_conv2d_res(x, wp: Packed, residual, bias=None, stride=1, pad=0, dil=1, relu=False, y=None,
                  stream=None, _entry="nm_conv2d_res"):
    """nm_conv2d with a residual (device tensor shaped and typed like the output, or None)
    added before the activation."""
    return _conv2d(x, wp, residual, bias, stride, pad, dil, relu, y, stream, _entry == "nm_conv2d_static")


def nm_maxpool2d(x, k: int, stride: int, pad: int, y=None, stream=None):
    """Max pooling of a contiguous NHWC device tensor (fp32 or bf16)."""
    import torch
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous device tensor")
    b, h, w, c = x.shape
    ho, wo = (h + 2 * pad - k) // stride + 1, (w + 2 * pad - k) // stride + 1
    if y is None:
        if min(ho, wo) < 1:
            raise NMError(-2, "output would be empty")
        y = torch.empty((b, ho, wo, c), dtype=x.dtype, device=x.device)
    _check(lib().nm_maxpool2d(x.data_ptr(), _dtype_code(x), b, h, w, c, k, stride, pad, y.data_ptr(),
                              _stream_ptr(stream)))
    return y


def nm_avgpool_global(x, y=None, stream=None):
    """Mean over all positions of a contiguous NHWC device tensor: [B,H,W,C] -> [B,C]."""
    import torch
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous device tensor")
    b, h, w, c = x.shape
    if y is None:
        y = torch.empty((b, c), dtype=x.dtype, device=x.device)
    _check(lib().nm_avgpool_global(x.data_ptr(), _dtype_code(x), b, h, w, c, y.data_ptr(),
                                   _stream_ptr(stream)))
    return y


def nm_im2col(x, kh: int, kw: int, stride=1, pad=0, dil=1, a=None, stream=None):
    """The im2col matrix of a contiguous NHWC device tensor, as the NHWC tensor
    [B,Hout,Wout,kh*kw*Cin] (k order (kh, kw, ci))."""
    import torch
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous device tensor")
    b, h, w, c = x.shape
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    dh, dw = _pair(dil)
    ho = (h + 2 * ph - dh * (kh - 1) - 1) // sh + 1
    wo = (w + 2 * pw - dw * (kw - 1) - 1) // sw + 1
    if a is None:
        if min(ho, wo) < 1:
            raise NMError(-2, "output would be empty")
        a = torch.empty((b, ho, wo, kh * kw * c), dtype=x.dtype, device=x.device)
    _check(lib().nm_im2col(x.data_ptr(), _dtype_code(x), b, h, w, c, kh, kw, sh, sw, ph, pw, dh, dw,
                           a.data_ptr(), _stream_ptr(stream)))
    return a


def nm_stream_floor(x, y, stream=None):
    """Reads all of x and overwrites all of y (contents unspecified) with one plain
    streaming kernel: the cost of a layer's traffic alone."""
    if not (x.is_cuda and y.is_cuda and x.is_contiguous() and y.is_contiguous()):
        raise ValueError("x and y must be contiguous device tensors")
    _check(lib().nm_stream_floor(x.data_ptr(), x.numel() * x.element_size(), y.data_ptr(),
                                 y.numel() * y.element_size(), _stream_ptr(stream)))


def nm_autotune(x_dtype: int, b: int, h: int, w: int, cin: int, wp: Packed, has_bias=True,
                stride=1, pad=0, dil=1, relu=True, y_dtype: Optional[int] = None, stream=None):
    """Returns (chosen variant id, its time in ms)."""
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    dh, dw = _pair(dil)
    v, ms = ctypes.c_int(-1), ctypes.c_float(0)
    _check(lib().nm_autotune(x_dtype, b, h, w, cin, wp.handle, int(bool(has_bias)), sh, sw, ph, pw,
                             dh, dw, int(bool(relu)),
                             (NM_BF16 if x_dtype == NM_F8E4M3 else x_dtype) if y_dtype is None else y_dtype,
                             _stream_ptr(stream), ctypes.byref(v), ctypes.byref(ms)))
    return v.value, ms.value


def nm_autotune_tile(w_ohwi: np.ndarray, n: int, m: int, tiles, x_dtype: int, b: int, h: int, w: int,
                     has_bias=True, stride=1, pad=0, dil=1, relu=True, value_dtype: Optional[int] = None,
                     stream=None):
    """Prunes at every candidate tile size, tunes each and returns
    (handle of the fastest, its tile size, [ms per candidate])."""
    wt = np.ascontiguousarray(w_ohwi, dtype=np.float32)
    cout, kh, kw, cin = wt.shape
    sh, sw = _pair(stride)
    ph, pw = _pair(pad)
    dh, dw = _pair(dil)
    vd = x_dtype if value_dtype is None else value_dtype
    cand = (ctypes.c_int * len(tiles))(*[int(t) for t in tiles])
    ms = (ctypes.c_float * len(tiles))()
    hnd, best = ctypes.c_void_p(), ctypes.c_int(0)
    _check(lib().nm_autotune_tile(wt.ctypes.data, cout, kh, kw, cin, n, m, cand, len(tiles), vd,
                                  x_dtype, b, h, w, int(bool(has_bias)), sh, sw, ph, pw, dh, dw,
                                  int(bool(relu)), x_dtype, _stream_ptr(stream),
                                  ctypes.byref(hnd), ctypes.byref(best), ms))
    return Packed(hnd, cout, kh, kw, cin, n, m, best.value, vd), best.value, list(ms)


def nm_cache_save(path: str):
    _check(lib().nm_cache_save(path.encode()))


def nm_cache_load(path: str):
    _check(lib().nm_cache_load(path.encode()))


def nm_workspace_free():
    _check(lib().nm_workspace_free())


def nm_cache_clear():
    _check(lib().nm_cache_clear())


def nm_cache_size() -> int:
    return _check(lib().nm_cache_size())


def nm_force_variant(v: int):
    _check(lib().nm_force_variant(v))


def nm_variant_legal(v: int, wp: Packed, x_dtype: int = NM_F32, y_dtype: int = NM_F32) -> bool:
    return _check(lib().nm_variant_legal(v, wp.handle, x_dtype, y_dtype)) == 1


# ---------------------------------------------------------------- 8-bit feed-forward operators (nm_q8.h)
# A single token's call runs for a few us on the GPU, so these keep what they ask of a tensor short, and do not look at outputs
# that they have allocated themselves.  A given stream is made the current one for the call: what is allocated then belongs to it.
# All tensors lie on the current device (or the given stream's).
def _rows_of(t, name: str):
    """(rows, width, row stride) of a device tensor whose last axis is the row: two axes with any row stride, or any
    number of them whose rows lie at one stride."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    shape = t.shape
    if len(shape) == 2:
        rows, width = shape
        ld, inner = t.stride()
        if inner != 1 and width > 1:
            raise ValueError(f"the values of a row of {name} must be adjacent")
        return rows, width, ld if rows > 1 else width
    if len(shape) < 1:
        raise ValueError(f"{name} must have rows")
    width = shape[-1]
    if t.is_contiguous():
        return (t.numel() // width if width else 0), width, width
    try:
        return _rows_of(t.view(-1, width), name)
    except RuntimeError:
        raise ValueError(f"the rows of {name} must lie at one stride") from None


def _q8_code(dtype, name: str) -> int:
    code = _q8_codes.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype} of {name}")
    return code


def _q8_stride(t, name: str, shape, dtype, dev: int) -> int:
    """Row stride of a tensor that the caller gave and that has to have this shape and type, on device `dev`."""
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on device {dev}")
    return _rows_of(t, name)[2]


def _q8_vector(t, name: str, n: int, dev: int) -> int:
    """Pointer of a contiguous fp32 vector of n values on device `dev`."""
    if t.dtype != _torch.float32 or t.numel() != n or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 tensor of {n} values on device {dev}")
    return t.data_ptr()


def _q8_like(x, dtype):
    """A new tensor of x's shape, contiguous."""
    if x.is_contiguous():
        return _torch.empty_like(x, dtype=dtype)
    return _torch.empty_like(x, dtype=dtype, memory_format=_torch.contiguous_format)


def _q8_new(x, rows: int, width: int):
    """(new 8-bit rows for x, their stride): the rows start at multiples of 16 bytes, where nm_linear_q8 reads them in place."""
    if width % 16 == 0 or rows == 1:
        return _q8_like(x, _torch.int8), width
    ld = (width + 15) // 16 * 16
    if x.dim() == 2:
        return x.new_empty_strided((rows, width), (ld, 1), dtype=_torch.int8), ld
    return x.new_empty(x.shape[:-1] + (ld,), dtype=_torch.int8)[..., :width], ld


def _q8_stream(dev: int) -> int:
    """The current stream, for tensors on device `dev`: the library launches on the current device, in no order with another's streams."""
    current = _torch._C._cuda_getDevice()
    if dev != current:
        raise ValueError(f"the tensors are on device {dev}, the current device is {current}")
    return _torch._C._cuda_getCurrentRawStream(dev)


_ROWS_ARGS = struct.Struct("15qd")       # nm_rows_q8_args_t
_DEQUANTIZE_ARGS = struct.Struct("9q")   # nm_dequantize_q8_args_t
_LINEAR_ARGS = struct.Struct("15q")      # nm_linear_q8_args_t


def _q8_rows(norm: bool, x, gamma, residual, eps, q, scales, residual_out):
    L = _lib or lib()
    rows, width, ld = _rows_of(x, "x")
    dtype, dev = x.dtype, x.get_device()
    code = _q8_code(dtype, "x")
    gptr = rptr = optr = ldr = 0
    ldo = width
    if gamma is not None:
        gptr = _q8_vector(gamma, "gamma", width, dev)
    if residual is not None:
        ldr, rptr = _q8_stride(residual, "residual", x.shape, dtype, dev), residual.data_ptr()
    if residual_out is not None:
        ldo, optr = _q8_stride(residual_out, "residual_out", x.shape, dtype, dev), residual_out.data_ptr()
    elif residual is not None:
        residual_out = _q8_like(x, dtype)
        optr = residual_out.data_ptr()
    if q is None:
        q, ldq = _q8_new(x, rows, width)
    else:
        ldq = _q8_stride(q, "q", x.shape, _torch.int8, dev)
    if scales is None:
        scales = x.new_empty_strided((rows,), (1,), dtype=_torch.float32) if x.dim() == 2 else x.new_empty(x.shape[:-1], dtype=_torch.float32)
        sptr = scales.data_ptr()
    else:
        if scales.shape != x.shape[:-1]:
            raise ValueError(f"scales must have the shape {tuple(x.shape[:-1])}")
        sptr = _q8_vector(scales, "scales", rows, dev)
    rc = L.nm_rows_q8_args(_ROWS_ARGS.pack(x.data_ptr(), rptr, gptr, optr, q.data_ptr(), sptr, _q8_stream(dev), code, rows, width, ld, ldr, ldo,
                                           ldq, norm, eps))
    if rc < 0:
        _check(rc)
    return q, scales, residual_out


def nm_quantize_q8(x, q=None, scales=None, stream=None):
    """Rows of x (fp32 or bf16, the last axis) rounded to 8 bits: (q int8 like x, scales fp32 [rows...]) with x ~ q * scales.
    A new q of an odd width has gaps between its rows."""
    if stream is not None:
        with _lib_torch().cuda.stream(stream):
            return _q8_rows(False, x, None, None, 0.0, q, scales, None)[:2]
    return _q8_rows(False, x, None, None, 0.0, q, scales, None)[:2]


def nm_rmsnorm_q8(x, gamma=None, residual=None, eps: float = 1e-6, q=None, scales=None, residual_out=None, stream=None):
    """h = x + residual; rows of gamma * h / sqrt(mean(h^2) + eps) rounded to 8 bits.  Returns (q, scales, h rounded to x's
    dtype); the last is None without a residual unless residual_out is given.  residual_out may be x or residual.  A new q of
    an odd width has gaps between its rows."""
    if stream is not None:
        with _lib_torch().cuda.stream(stream):
            return _q8_rows(True, x, gamma, residual, eps, q, scales, residual_out)
    return _q8_rows(True, x, gamma, residual, eps, q, scales, residual_out)


def nm_dequantize_q8(q, scales, dtype=None, y=None, stream=None):
    """The values that 8-bit rows stand for, q * scales, in fp32 or bf16 (`dtype`; default fp32 or y's)."""
    if stream is not None:
        with _lib_torch().cuda.stream(stream):
            return nm_dequantize_q8(q, scales, dtype, y)
    L = _lib or lib()
    rows, width, ld = _rows_of(q, "q")
    if q.dtype != _torch.int8:
        raise TypeError(f"q must be int8, not {q.dtype}")
    dev, ldy = q.get_device(), width
    if y is None:
        dtype = dtype or _torch.float32
        y = _q8_like(q, dtype)
    else:
        dtype = dtype or y.dtype
        ldy = _q8_stride(y, "y", q.shape, dtype, dev)
    rc = L.nm_dequantize_q8_args(_DEQUANTIZE_ARGS.pack(q.data_ptr(), _q8_vector(scales, "scales", rows, dev), y.data_ptr(), _q8_stream(dev),
                                                       _q8_code(dtype, "y"), rows, width, ld, ldy))
    if rc < 0:
        _check(rc)
    return y


class Q8Weights:
    """Owner of an nm_q8_t handle: [channels, width] weights in 8 bits."""

    def __init__(self, handle, channels: int, width: int, gated: bool):
        self.handle = handle
        self.channels, self.width, self.gated = channels, width, gated
        self.outs = channels // 2 if gated else channels

    def free(self):
        """Release the handle now (idempotent)."""
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.nm_q8_free(h)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def nm_q8_pack(w, scales=None, gated: bool = False, stream=None) -> Q8Weights:
    """Weights [channels, width] on the device: int8 with fp32 scales [channels], or fp32 / bf16, which are rounded here
    (a scale for each channel).  gated: the first half of the channels gates the second."""
    if stream is not None:
        with _lib_torch().cuda.stream(stream):
            return nm_q8_pack(w, scales, gated)
    L = _lib or lib()
    if w.dim() != 2:
        raise ValueError("w must have two axes")
    channels, width, ld = _rows_of(w, "w")
    sptr = 0 if scales is None else _q8_vector(scales, "scales", channels, w.get_device())
    h = ctypes.c_void_p()
    _check(L.nm_q8_pack(w.data_ptr(), _q8_code(w.dtype, "w"), sptr, channels, width, ld, int(bool(gated)), _q8_stream(w.get_device()), ctypes.byref(h)))
    return Q8Weights(h, channels, width, bool(gated))


def nm_q8_export(w: Q8Weights):
    """(int8 [channels, width], fp32 scales [channels]) as numpy arrays."""
    a, s = np.empty((w.channels, w.width), dtype=np.int8), np.empty(w.channels, dtype=np.float32)
    _check(lib().nm_q8_export(w.handle, a.ctypes.data, s.ctypes.data))
    return a, s


def nm_linear_q8(q, scales, w: Q8Weights, bias=None, residual=None, dtype=None, y=None, stream=None):
    """8-bit rows times 8-bit weights: (q @ w.T) * scales * channel scales + bias + residual, or the gated form
    silu(gate) * up.  y: [..., channels] (gated: half of them) in bf16 (default) or fp32; residual is typed and shaped
    like y and may be y."""
    if stream is not None:
        with _lib_torch().cuda.stream(stream):
            return nm_linear_q8(q, scales, w, bias, residual, dtype, y)
    L = _lib or lib()
    rows, width, ld = _rows_of(q, "q")
    if q.dtype != _torch.int8:
        raise TypeError(f"q must be int8, not {q.dtype}")
    dev, outs = q.get_device(), w.outs
    shape = (rows, outs) if q.dim() == 2 else q.shape[:-1] + (outs,)
    ldy = outs
    if y is None:
        dtype = dtype or _torch.bfloat16
        y = q.new_empty(shape, dtype=dtype)
    else:
        dtype = dtype or y.dtype
        ldy = _q8_stride(y, "y", shape, dtype, dev)
    bptr = rptr = ldr = 0
    if bias is not None:
        bptr = _q8_vector(bias, "bias", w.channels, dev)
    if residual is not None:
        ldr, rptr = _q8_stride(residual, "residual", shape, dtype, dev), residual.data_ptr()
    qptr, handle = q.data_ptr(), w.handle.value if w.handle else 0
    wptr = nbytes = 0
    if rows > NM_Q8_FEW_ROWS or qptr % 16 or (rows > 1 and ld % 16):   # (else none is needed)
        need = ctypes.c_size_t(0)
        rc = L.nm_linear_q8_workspace(qptr, rows, ld, handle, ctypes.byref(need))
        if rc < 0:
            _check(rc)
        nbytes = need.value
        if nbytes:
            ws = q.new_empty(nbytes)
            wptr = ws.data_ptr()
    rc = L.nm_linear_q8_args(_LINEAR_ARGS.pack(qptr, _q8_vector(scales, "scales", rows, dev), handle, bptr, rptr, y.data_ptr(), wptr,
                                               _q8_stream(dev), _q8_code(dtype, "y"), rows, width, ld, ldr, ldy, nbytes))
    if rc < 0:
        _check(rc)
    return y
