"""Python binding of include/apt_mx.h (in libapt.so): argument marshalling only.

Every function named ``apt_*`` calls the C entry point of the same name with
plain integers and device pointers.  The torch helpers below (``mx4_quantize``,
``mx4_gemm``, ``rmsnorm_codes``, ...) check the tensors, allocate outputs and
workspace with torch and pass pointers, strides and the HIP stream; every step
of the computation runs in the library's kernels.  They run on their tensors'
device, whichever is current, on its current stream or the one that is passed.
"""
from __future__ import annotations

import ctypes
import os
import re
from dataclasses import dataclass

from . import apt as _apt
from .apt import APT_ERR_INVALID_ARG, AptError, _on_stream, _torch, check

HEADER_PATH = os.path.join(os.path.dirname(_apt.HEADER_PATH), "apt_mx.h")

APT_TYPE_FP16 = 1
APT_TYPE_BF16 = 2
APT_TYPE_FP32 = 3

_vp, _int, _i64, _size = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
_SIGNATURES = {
    "apt_mx4_bytes": (_size, [_int, _int]),
    "apt_mx4_quantize": (_int, [_vp, _int, _int, _int, _i64, _vp, _vp]),
    "apt_mx4_dequantize": (_int, [_vp, _int, _int, _int, _vp, _vp]),
    "apt_mx4_pack": (_int, [_vp, _vp, _int, _int, _vp, _vp]),
    "apt_mx4_unpack": (_int, [_vp, _int, _int, _vp, _vp, _vp]),
    "apt_mx4_gemm": (_int, [_int, _int, _int, _vp, _vp, _int, _vp, _vp]),
    "apt_mx4_select": (_int, [_int, _int, _int, ctypes.POINTER(_int), ctypes.POINTER(_int)]),
    "apt_mx4_gemm_act_workspace_bytes": (_size, [_int, _int, _int]),
    "apt_mx4_gemm_act": (_int, [_int, _int, _int, _vp, _int, _i64, _vp, _int, _vp, _vp, _size, _vp]),
    "apt_rmsnorm_codes": (_int, [_int, _int, _int, _vp, _i64, _vp, _i64, _vp, ctypes.c_double, _int, _vp, _vp, _vp,
                                 _vp, _vp]),
    "apt_rmsnorm_mx4": (_int, [_int, _int, _int, _vp, _i64, _vp, _i64, _vp, ctypes.c_double, _vp, _vp, _vp, _vp]),
    "apt_dequantize_codes": (_int, [_vp, _vp, _int, _int, _int, _vp, _vp]),
}
_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = _apt.lib()
        for name, (restype, argtypes) in _SIGNATURES.items():
            f = getattr(L, name)
            f.restype, f.argtypes = restype, argtypes
        _lib = L
    return _lib


def mx_header_functions() -> list:
    """Names of the functions include/apt_mx.h declares."""
    text = re.sub(r"/\*.*?\*/", "", open(HEADER_PATH).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(apt_[a-z0-9_]+)\s*\(", text)))


# ---- C entry points, same names -------------------------------------------------
#
# (ctypes passes an int modulo 2^32: 2^32 + 16 rows would be 16)

_MOST = 2 ** 31 - 1  # that an int of C holds


def _ints(*numbers):
    """Whether ints of C hold the numbers."""
    return max(numbers) <= _MOST and min(numbers) >= -_MOST - 1


def apt_mx4_bytes(rows, K) -> int:
    if not _ints(rows, K):
        return 0
    return int(lib().apt_mx4_bytes(rows, K))


def apt_mx4_quantize(x, type, rows, K, stride, mx, stream) -> int:
    if not _ints(type, rows, K):
        return APT_ERR_INVALID_ARG
    return lib().apt_mx4_quantize(x, type, rows, K, stride, mx, stream)


def apt_mx4_dequantize(mx, rows, K, type, out, stream) -> int:
    if not _ints(rows, K, type):
        return APT_ERR_INVALID_ARG
    return lib().apt_mx4_dequantize(mx, rows, K, type, out, stream)


def apt_mx4_pack(codes, scales, rows, K, mx, stream) -> int:
    if not _ints(rows, K):
        return APT_ERR_INVALID_ARG
    return lib().apt_mx4_pack(codes, scales, rows, K, mx, stream)


def apt_mx4_unpack(mx, rows, K, codes, scales, stream) -> int:
    if not _ints(rows, K):
        return APT_ERR_INVALID_ARG
    return lib().apt_mx4_unpack(mx, rows, K, codes, scales, stream)


def apt_mx4_gemm(M, N, K, a_mx, w_mx, type, c, stream) -> int:
    if not _ints(M, N, K, type):
        return APT_ERR_INVALID_ARG
    return lib().apt_mx4_gemm(M, N, K, a_mx, w_mx, type, c, stream)


def apt_mx4_select(M, N, K):
    """(status, rows, columns)."""
    if not _ints(M, N, K):
        return APT_ERR_INVALID_ARG, 0, 0
    rows, columns = _int(0), _int(0)
    st = lib().apt_mx4_select(M, N, K, ctypes.byref(rows), ctypes.byref(columns))
    return st, rows.value, columns.value


def apt_mx4_gemm_act_workspace_bytes(M, N, K) -> int:
    if not _ints(M, N, K):
        return 0
    return int(lib().apt_mx4_gemm_act_workspace_bytes(M, N, K))


def apt_mx4_gemm_act(M, N, K, x, x_type, x_stride, w_mx, type, c, workspace, workspace_bytes, stream) -> int:
    if not _ints(M, N, K, x_type, type):
        return APT_ERR_INVALID_ARG
    return lib().apt_mx4_gemm_act(M, N, K, x, x_type, x_stride, w_mx, type, c, workspace, workspace_bytes, stream)


def apt_rmsnorm_codes(M, K, type, x, x_stride, residual, residual_stride, gain, eps, q, h, y, codes, scale,
                      stream) -> int:
    if not _ints(M, K, type, q):
        return APT_ERR_INVALID_ARG
    return lib().apt_rmsnorm_codes(M, K, type, x, x_stride, residual, residual_stride, gain, eps, q, h, y, codes,
                                   scale, stream)


def apt_rmsnorm_mx4(M, K, type, x, x_stride, residual, residual_stride, gain, eps, h, y, mx, stream) -> int:
    if not _ints(M, K, type):
        return APT_ERR_INVALID_ARG
    return lib().apt_rmsnorm_mx4(M, K, type, x, x_stride, residual, residual_stride, gain, eps, h, y, mx, stream)


def apt_dequantize_codes(codes, scale, M, K, type, out, stream) -> int:
    if not _ints(M, K, type):
        return APT_ERR_INVALID_ARG
    return lib().apt_dequantize_codes(codes, scale, M, K, type, out, stream)


# ---- torch helpers (checks, allocation, pointers) -------------------------------
#
# A small call's time is the host's (a launch 3.3 us, each allocation 1.2 to 1.7),
# so these keep to what a call needs: the C functions are called without the
# wrappers above, new tensors are made like given ones, and devices are compared
# by number.

_types = None


def _type(dtype, where):
    """The library's number of a torch type."""
    global _types
    if _types is None:
        torch = _torch()
        _types = {torch.float16: APT_TYPE_FP16, torch.bfloat16: APT_TYPE_BF16, torch.float32: APT_TYPE_FP32}
    t = _types.get(dtype)
    if t is None:
        raise AptError(APT_ERR_INVALID_ARG, "%s: type %s" % (where, dtype))
    return t


def _refuse(where, what):
    raise AptError(APT_ERR_INVALID_ARG, "%s: %s" % (where, what))


_raw_stream = _device = None  # torch's, once it is there


def _call(name, index, stream, *args):
    """The C function `name` of the arguments and the raw stream, on the device of number `index`."""
    global _raw_stream, _device
    if _device is None:
        C = _torch()._C
        _raw_stream, _device = C._cuda_getCurrentRawStream, C._cuda_getDevice
    if stream is None:
        raw = _raw_stream(index)
    else:
        if stream.device_index != index:
            _refuse(name, "a stream of another device")
        raw = stream.cuda_stream
    f = getattr(_lib or lib(), name)
    if _device() == index:
        status = f(*args, raw)
    else:
        with _torch().cuda.device(index):
            status = f(*args, raw)
    if status:
        check(status, name)


def _new(like, shape, dtype, stream):
    """A new tensor on the device of `like`, of the call's stream."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with _on_stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _new_like(x, dtype, stream):
    """A new contiguous tensor of x's shape, of the call's stream."""
    if stream is None:
        if x.is_contiguous():
            return _torch().empty_like(x, dtype=dtype)
        return x.new_empty(x.shape, dtype=dtype)
    with _on_stream(stream):
        return x.new_empty(x.shape, dtype=dtype)


def _rows(x, where, stream):
    """x, or a copy (made on the call's stream), as rows of adjacent elements: (rows, the stride from one
    to the next, their number, their length, the number of their device)."""
    index = x.get_device()  # (below 0 in host memory)
    if index < 0 or x.dim() != 2:
        _refuse(where, "a CUDA tensor of two dimensions is wanted")
    M, K = x.shape
    if M > _MOST or K > _MOST:
        _refuse(where, "%d rows of %d values" % (M, K))
    if x.is_contiguous():
        return x, K, M, K, index
    if (x.stride(1) == 1 or K == 1) and (x.stride(0) >= K or M == 1):
        return x, (x.stride(0) if M > 1 else K), M, K, index
    with _on_stream(stream):
        return x.contiguous(), K, M, K, index


@dataclass
class Mx4:
    """An MX4 operand on the device: `rows` rows of K values in apt_mx4_bytes(rows, K) bytes (uint8)."""
    data: "object"
    rows: int
    K: int


def _bytes(rows, K):
    """apt_mx4_bytes (a call into C takes longer)."""
    return (rows + 15 >> 4) * (K + 255 >> 8) * 2176 if rows >= 1 and K >= 1 else 0


_uint8 = None  # torch's, once it is there


def _data_of(a, where):
    """The data of an operand and the number of its device, checked at each use: its sizes and its
    tensor may have changed since the last."""
    global _uint8
    if _uint8 is None:
        _uint8 = _torch().uint8
    d, rows, K = a.data, a.rows, a.K
    index = d.get_device()  # (below 0 in host memory)
    if not (index >= 0 and 0 < rows <= _MOST and 0 < K <= _MOST and d.dtype is _uint8 and d.is_contiguous() and
            d.numel() >= (rows + 15 >> 4) * (K + 255 >> 8) * 2176):
        _refuse(where, "an operand of %d rows of %d values is %d bytes (uint8) on the device" % (rows, K, _bytes(rows, K)))
    return d, index


def _new_mx4(rows, K, like, stream, where) -> Mx4:
    """An operand on the device of `like`."""
    n = _bytes(rows, K)
    if n == 0:
        _refuse(where, "%d rows of %d values" % (rows, K))
    return Mx4(_new(like, n, _torch().uint8, stream), rows, K)


def mx4_quantize(x, stream=None) -> Mx4:
    """Quantizes rows x [M][K] (fp16, bf16 or fp32, a CUDA tensor) to an MX4 operand."""
    x, stride, M, K, index = _rows(x, "mx4_quantize", stream)
    t = _type(x.dtype, "mx4_quantize")
    out = _new_mx4(M, K, x, stream, "mx4_quantize")
    _call("apt_mx4_quantize", index, stream, x.data_ptr(), t, M, K, stride, out.data.data_ptr())
    return out


def mx4_dequantize(a: Mx4, dtype=None, stream=None):
    """The values of an MX4 operand, [rows][K] of `dtype` (by default bf16, which holds all that quantizing gives)."""
    dtype = _torch().bfloat16 if dtype is None else dtype
    t = _type(dtype, "mx4_dequantize")
    data, index = _data_of(a, "mx4_dequantize")
    out = _new(data, (a.rows, a.K), dtype, stream)
    _call("apt_mx4_dequantize", index, stream, data.data_ptr(), a.rows, a.K, t, out.data_ptr())
    return out


def mx4_pack(codes, scales, K: int, stream=None) -> Mx4:
    """Lays row-major codes uint8 [rows][ceil(K / 2)] (the even element in the low nibble) and scale
    bytes uint8 [rows][ceil(K / 32)] out as an MX4 operand."""
    u8 = _torch().uint8
    if not (codes.is_cuda and scales.device == codes.device and codes.dtype == u8 and scales.dtype == u8 and K >= 1 and
            codes.dim() == 2 and tuple(scales.shape) == (codes.shape[0], -(-K // 32)) and
            codes.shape[1] == -(-K // 2)):
        _refuse("mx4_pack", "codes [rows][ceil(K / 2)] and scales [rows][ceil(K / 32)]")
    rows = codes.shape[0]
    if rows > _MOST or K > _MOST:
        _refuse("mx4_pack", "%d rows of %d values" % (rows, K))
    out = _new_mx4(rows, K, codes, stream, "mx4_pack")
    with _on_stream(stream):
        codes, scales = codes.contiguous(), scales.contiguous()
    _call("apt_mx4_pack", codes.get_device(), stream, codes.data_ptr(), scales.data_ptr(), rows, K, out.data.data_ptr())
    return out


def mx4_unpack(a: Mx4, stream=None):
    """(codes, scales) of an MX4 operand as mx4_pack takes them."""
    data, index = _data_of(a, "mx4_unpack")
    codes = _new(data, (a.rows, -(-a.K // 2)), data.dtype, stream)
    scales = _new(data, (a.rows, -(-a.K // 32)), data.dtype, stream)
    _call("apt_mx4_unpack", index, stream, data.data_ptr(), a.rows, a.K, codes.data_ptr(), scales.data_ptr())
    return codes, scales


def mx4_gemm(a: Mx4, w: Mx4, dtype=None, stream=None):
    """C = A W^T of two MX4 operands, [a.rows][w.rows] of `dtype` (fp16 by default)."""
    dtype = _torch().float16 if dtype is None else dtype
    t = _type(dtype, "mx4_gemm")
    ad, index = _data_of(a, "mx4_gemm")
    wd, at = _data_of(w, "mx4_gemm")
    M, N, K = a.rows, w.rows, a.K
    if K != w.K or at != index:
        _refuse("mx4_gemm", "operands of %d and %d values a row on %s and %s" % (K, w.K, ad.device, wd.device))
    c = _new(ad, (M, N), dtype, stream)
    _call("apt_mx4_gemm", index, stream, M, N, K, ad.data_ptr(), wd.data_ptr(), t, c.data_ptr())
    return c


def mx4_gemm_act(x, w: Mx4, dtype=None, stream=None, workspace=None):
    """C = A W^T for unpacked activations x [M][K] (fp16, bf16 or fp32), quantized to MX4 inside the
    call; [M][w.rows] of `dtype` (by default x's).  A workspace of apt_mx4_gemm_act_workspace_bytes is
    allocated with torch unless one is passed."""
    x, stride, M, K, index = _rows(x, "mx4_gemm_act", stream)
    dtype = x.dtype if dtype is None else dtype
    tx, t = _type(x.dtype, "mx4_gemm_act"), _type(dtype, "mx4_gemm_act")
    wd, at = _data_of(w, "mx4_gemm_act")
    if K != w.K or at != index:
        _refuse("mx4_gemm_act", "rows of %d values on %s for weights of %d on %s" % (K, x.device, w.K, wd.device))
    N = w.rows
    if workspace is None:
        n = (_lib or lib()).apt_mx4_gemm_act_workspace_bytes(M, N, K)
        if n:
            workspace = _new(wd, n, wd.dtype, stream)
    else:
        if workspace.get_device() != index or not workspace.is_contiguous():
            _refuse("mx4_gemm_act", "a contiguous workspace on the rows' device is wanted")
        n = workspace.numel() * workspace.element_size()
    c = _new(x, (M, N), dtype, stream)
    _call("apt_mx4_gemm_act", index, stream, M, N, K, x.data_ptr(), tx, stride, wd.data_ptr(), t, c.data_ptr(),
          None if workspace is None else workspace.data_ptr(), n)
    return c


def _norm_inputs(x, gain, residual, h, stream, where):
    """Checked inputs of a norm: x, the residual, the gain, h (given, or made where there is a residual,
    or None), the number of their device and the C arguments up to the gain."""
    torch = _torch()
    dtype = x.dtype
    t = APT_TYPE_FP16 if dtype is torch.float16 else APT_TYPE_BF16 if dtype is torch.bfloat16 else 0
    if not t:
        _refuse(where, "fp16 or bf16 rows are wanted")
    x, xs, M, K, index = _rows(x, where, stream)
    shape = x.shape
    rp, rs, gp = None, 0, None
    if residual is not None:
        if residual.dtype is not dtype or residual.shape != shape or residual.get_device() != index:
            _refuse(where, "a residual like x is wanted")
        if residual.is_contiguous():
            rs = K
        else:
            residual, rs = _rows(residual, where, stream)[:2]
        rp = residual.data_ptr()
    if gain is not None:
        if gain.dtype is not dtype or gain.dim() != 1 or gain.numel() != K or gain.get_device() != index:
            _refuse(where, "a gain of x's width, type and device is wanted")
        if not gain.is_contiguous():
            with _on_stream(stream):
                gain = gain.contiguous()
        gp = gain.data_ptr()
    if h is not None:
        if h.dtype is not dtype or h.shape != shape or h.get_device() != index or not h.is_contiguous():
            _refuse(where, "a contiguous h like x is wanted")
    elif residual is not None:
        h = _new_like(x, dtype, stream)
    return x, residual, gain, h, index, (M, K, t, x.data_ptr(), xs, rp, rs, gp)


def rmsnorm_codes(x, gain, q: int, eps: float, residual=None, h=None, out_y: bool = False, stream=None):
    """RMS norm of x + residual (fp16 or bf16 [M][K]) with `gain` [K] (or None), quantized per row to
    q-bit codes as gemm_act and gemm_decode take them.  Returns (codes int8 [M][K], fp16 scales [M],
    h), and y behind them with out_y: h is x + residual, written to `h` where one is given (x or the
    residual itself, or a tensor that overlaps no input), to a new tensor where there is a residual,
    else None.  The residual and the gain have x's type; rows in more dimensions are for the caller to
    flatten."""
    torch = _torch()
    if not 1 <= q <= 8:
        _refuse("rmsnorm_codes", "codes of %s bits" % (q, ))
    # (copies that were made stay alive until the call has been enqueued)
    x, residual, gain, h, index, args = _norm_inputs(x, gain, residual, h, stream, "rmsnorm_codes")
    y = _new_like(x, x.dtype, stream) if out_y else None
    codes = _new_like(x, torch.int8, stream)
    scale = _new(x, args[0], torch.float16, stream)
    _call("apt_rmsnorm_codes", index, stream, *args, eps, q, None if h is None else h.data_ptr(),
          None if y is None else y.data_ptr(), codes.data_ptr(), scale.data_ptr())
    return (codes, scale, h, y) if out_y else (codes, scale, h)


def rmsnorm_mx4(x, gain, eps: float, residual=None, h=None, out_y: bool = False, stream=None):
    """As rmsnorm_codes with the row quantized to MX4.  Returns (Mx4, h), and y behind them with out_y."""
    # (copies that were made stay alive until the call has been enqueued)
    x, residual, gain, h, index, args = _norm_inputs(x, gain, residual, h, stream, "rmsnorm_mx4")
    y = _new_like(x, x.dtype, stream) if out_y else None
    out = _new_mx4(args[0], args[1], x, stream, "rmsnorm_mx4")
    _call("apt_rmsnorm_mx4", index, stream, *args, eps, None if h is None else h.data_ptr(),
          None if y is None else y.data_ptr(), out.data.data_ptr())
    return (out, h, y) if out_y else (out, h)


def dequantize(codes, scale, dtype=None, stream=None):
    """The values (2 code + 1) scale of int8 codes [M][K] with fp16 scales [M], of `dtype` (fp16 by default)."""
    torch = _torch()
    dtype = torch.float16 if dtype is None else dtype
    t = _type(dtype, "dequantize")
    if not (codes.is_cuda and codes.dim() == 2 and codes.dtype is torch.int8 and scale.dtype is torch.float16 and
            scale.dim() == 1 and scale.shape[0] == codes.shape[0] and scale.device == codes.device):
        _refuse("dequantize", "int8 codes [M][K] and fp16 scales [M] are wanted")
    M, K = codes.shape
    if M > _MOST or K > _MOST:
        _refuse("dequantize", "%d rows of %d values" % (M, K))
    if not (codes.is_contiguous() and scale.is_contiguous()):
        with _on_stream(stream):
            codes, scale = codes.contiguous(), scale.contiguous()
    out = _new_like(codes, dtype, stream)
    _call("apt_dequantize_codes", codes.get_device(), stream, codes.data_ptr(), scale.data_ptr(), M, K, t, out.data_ptr())
    return out
