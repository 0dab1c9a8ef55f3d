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
    "apt_mx4_gemm_workspace_bytes": (_size, [_int, _int, _int]),
    "apt_mx4_gemm": (_int, [_int, _int, _int, _vp, _vp, _int, _vp, _vp, _size, _vp]),
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

def apt_mx4_bytes(rows, K) -> int:
    return int(lib().apt_mx4_bytes(rows, K))


def apt_mx4_quantize(x, type, rows, K, stride, mx, stream) -> int:
    return lib().apt_mx4_quantize(x, type, rows, K, stride, mx, stream)


def apt_mx4_dequantize(mx, rows, K, type, out, stream) -> int:
    return lib().apt_mx4_dequantize(mx, rows, K, type, out, stream)


def apt_mx4_pack(codes, scales, rows, K, mx, stream) -> int:
    return lib().apt_mx4_pack(codes, scales, rows, K, mx, stream)


def apt_mx4_unpack(mx, rows, K, codes, scales, stream) -> int:
    return lib().apt_mx4_unpack(mx, rows, K, codes, scales, stream)


def apt_mx4_gemm_workspace_bytes(M, N, K) -> int:
    return int(lib().apt_mx4_gemm_workspace_bytes(M, N, K))


def apt_mx4_gemm(M, N, K, a_mx, w_mx, type, c, workspace, workspace_bytes, stream) -> int:
    return lib().apt_mx4_gemm(M, N, K, a_mx, w_mx, type, c, workspace, workspace_bytes, stream)


def apt_mx4_gemm_act_workspace_bytes(M, N, K) -> int:
    return int(lib().apt_mx4_gemm_act_workspace_bytes(M, N, K))


def apt_mx4_gemm_act(M, N, K, x, x_type, x_stride, w_mx, type, c, workspace, workspace_bytes, stream) -> int:
    return lib().apt_mx4_gemm_act(M, N, K, x, x_type, x_stride, w_mx, type, c, workspace, workspace_bytes, stream)


def apt_rmsnorm_codes(M, K, type, x, x_stride, residual, residual_stride, gain, eps, q, h, y, codes, scale,
                      stream) -> int:
    return lib().apt_rmsnorm_codes(M, K, type, x, x_stride, residual, residual_stride, gain, eps, q, h, y, codes,
                                   scale, stream)


def apt_rmsnorm_mx4(M, K, type, x, x_stride, residual, residual_stride, gain, eps, h, y, mx, stream) -> int:
    return lib().apt_rmsnorm_mx4(M, K, type, x, x_stride, residual, residual_stride, gain, eps, h, y, mx, stream)


def apt_dequantize_codes(codes, scale, M, K, type, out, stream) -> int:
    return lib().apt_dequantize_codes(codes, scale, M, K, type, out, stream)


# ---- torch helpers (checks, allocation, pointers) -------------------------------

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


def _require(ok, where, what):
    if not ok:
        raise AptError(APT_ERR_INVALID_ARG, "%s: %s" % (where, what))


def _call(fn, device, stream, args):
    """fn(*args, raw stream) on `device`."""
    C = _torch()._C
    if stream is not None:
        _require(stream.device == device, fn.__name__, "a stream of another device")
        raw = stream.cuda_stream
    else:
        raw = C._cuda_getCurrentRawStream(device.index)
    if C._cuda_getDevice() == device.index:
        check(fn(*args, raw), fn.__name__)
    else:
        with _torch().cuda.device(device):
            check(fn(*args, raw), fn.__name__)


def _rows(x, where, stream):
    """x, or a copy (made on the call's stream), as rows of adjacent elements, and the stride of its rows."""
    _require(x.is_cuda and x.dim() == 2, where, "a CUDA tensor of two dimensions is wanted")
    M, K = x.shape
    if (x.stride(1) == 1 or K == 1) and (x.stride(0) >= K or M == 1):
        return x, (x.stride(0) if M > 1 else K)
    with _on_stream(stream):
        return x.contiguous(), K


@dataclass
class Mx4:
    """An MX4 operand on the device: `rows` rows of K values."""
    data: "object"
    rows: int
    K: int


def _new_mx4(rows, K, device, stream, where) -> Mx4:
    n = apt_mx4_bytes(rows, K)
    _require(n > 0, where, "%d rows of %d values" % (rows, K))
    with _on_stream(stream):
        return Mx4(_torch().empty(n, dtype=_torch().uint8, device=device), rows, K)


def mx4_quantize(x, stream=None) -> Mx4:
    """Quantizes rows x [M][K] (fp16, bf16 or fp32, a CUDA tensor) to an MX4 operand."""
    x, stride = _rows(x, "mx4_quantize", stream)
    M, K = x.shape
    t = _type(x.dtype, "mx4_quantize")
    out = _new_mx4(M, K, x.device, stream, "mx4_quantize")
    _call(apt_mx4_quantize, x.device, stream, (x.data_ptr(), t, M, K, stride, out.data.data_ptr()))
    return out


def mx4_dequantize(a: Mx4, dtype=None, stream=None):
    """The values of an MX4 operand, [rows][K] of `dtype` (by default bf16, which holds them all)."""
    torch = _torch()
    dtype = torch.bfloat16 if dtype is None else dtype
    t = _type(dtype, "mx4_dequantize")
    with _on_stream(stream):
        out = torch.empty((a.rows, a.K), dtype=dtype, device=a.data.device)
    _call(apt_mx4_dequantize, a.data.device, stream, (a.data.data_ptr(), a.rows, a.K, t, out.data_ptr()))
    return out


def mx4_pack(codes, scales, K: int, stream=None) -> Mx4:
    """Lays row-major codes uint8 [rows][ceil(K / 2)] (the even element in the low nibble) and scale
    bytes uint8 [rows][ceil(K / 32)] out as an MX4 operand."""
    u8 = _torch().uint8
    _require(codes.is_cuda and scales.device == codes.device and codes.dtype == u8 and scales.dtype == u8 and K >= 1 and
             codes.dim() == 2 and tuple(scales.shape) == (codes.shape[0], -(-K // 32)) and
             codes.shape[1] == -(-K // 2), "mx4_pack", "codes [rows][ceil(K / 2)] and scales [rows][ceil(K / 32)]")
    rows = codes.shape[0]
    out = _new_mx4(rows, K, codes.device, stream, "mx4_pack")
    with _on_stream(stream):
        codes, scales = codes.contiguous(), scales.contiguous()
    _call(apt_mx4_pack, codes.device, stream, (codes.data_ptr(), scales.data_ptr(), rows, K, out.data.data_ptr()))
    return out


def mx4_unpack(a: Mx4, stream=None):
    """(codes, scales) of an MX4 operand as mx4_pack takes them."""
    torch = _torch()
    with _on_stream(stream):
        codes = torch.empty((a.rows, -(-a.K // 2)), dtype=torch.uint8, device=a.data.device)
        scales = torch.empty((a.rows, -(-a.K // 32)), dtype=torch.uint8, device=a.data.device)
    _call(apt_mx4_unpack, a.data.device, stream, (a.data.data_ptr(), a.rows, a.K, codes.data_ptr(), scales.data_ptr()))
    return codes, scales


def _product(M, w, dtype, need, device, stream, workspace, where):
    """The output and the workspace (tensor or None, its bytes) of a product."""
    torch = _torch()
    _require(w.data.device == device, where, "the operands are on different devices")
    with _on_stream(stream):
        c = torch.empty((M, w.rows), dtype=dtype, device=device)
        if workspace is None and need > 0:
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
    if workspace is None:
        return c, None, 0
    _require(workspace.device == device and workspace.is_contiguous(), where, "a contiguous workspace on the device")
    return c, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def mx4_gemm(a: Mx4, w: Mx4, dtype=None, stream=None, workspace=None):
    """C = A W^T of two MX4 operands, [a.rows][w.rows] of `dtype` (fp16 by default).  A workspace of
    apt_mx4_gemm_workspace_bytes is allocated with torch unless one is passed."""
    dtype = _torch().float16 if dtype is None else dtype
    t = _type(dtype, "mx4_gemm")
    _require(a.K == w.K, "mx4_gemm", "operands of %d and %d values a row" % (a.K, w.K))
    device = a.data.device
    c, ws, n = _product(a.rows, w, dtype, apt_mx4_gemm_workspace_bytes(a.rows, w.rows, a.K), device, stream, workspace,
                        "mx4_gemm")
    _call(apt_mx4_gemm, device, stream,
          (a.rows, w.rows, a.K, a.data.data_ptr(), w.data.data_ptr(), t, c.data_ptr(), ws, n))
    return c


def mx4_gemm_act(x, w: Mx4, dtype=None, stream=None, workspace=None):
    """C = A W^T for unpacked activations x [M][K] (fp16, bf16 or fp32), quantized to MX4 inside the
    call; [M][w.rows] of `dtype` (by default x's).  A workspace of apt_mx4_gemm_act_workspace_bytes is
    allocated with torch unless one is passed."""
    x, stride = _rows(x, "mx4_gemm_act", stream)
    M, K = x.shape
    dtype = x.dtype if dtype is None else dtype
    tx, t = _type(x.dtype, "mx4_gemm_act"), _type(dtype, "mx4_gemm_act")
    _require(K == w.K, "mx4_gemm_act", "rows of %d values for weights of %d" % (K, w.K))
    c, ws, n = _product(M, w, dtype, apt_mx4_gemm_act_workspace_bytes(M, w.rows, K), x.device, stream, workspace,
                        "mx4_gemm_act")
    _call(apt_mx4_gemm_act, x.device, stream,
          (M, w.rows, K, x.data_ptr(), tx, stride, w.data.data_ptr(), t, c.data_ptr(), ws, n))
    return c


def _norm_inputs(x, gain, residual, h, out_y, stream, where):
    """Checked inputs of a norm: (x, the arguments up to `gain`, h, y).  h is given, allocated where
    there is a residual, or None."""
    torch = _torch()
    _require(x.dtype in (torch.float16, torch.bfloat16), where, "fp16 or bf16 rows are wanted")
    x, xs = _rows(x, where, stream)
    M, K = x.shape
    r, rs = None, 0
    if residual is not None:
        _require(residual.shape == x.shape and residual.dtype == x.dtype and residual.device == x.device, where,
                 "a residual like x")
        r, rs = _rows(residual, where, stream)
    if gain is not None:
        _require(tuple(gain.shape) == (K,) and gain.dtype == x.dtype and gain.device == x.device, where,
                 "a gain of x's width, type and device")
    with _on_stream(stream):
        if gain is not None:
            gain = gain.contiguous()
        if h is not None:
            _require(h.shape == x.shape and h.dtype == x.dtype and h.device == x.device and h.is_contiguous(), where,
                     "a contiguous h like x")
        elif residual is not None:
            h = torch.empty((M, K), dtype=x.dtype, device=x.device)
        y = torch.empty((M, K), dtype=x.dtype, device=x.device) if out_y else None
    args = (M, K, _type(x.dtype, where), x.data_ptr(), xs, r.data_ptr() if r is not None else None, rs,
            gain.data_ptr() if gain is not None else None)
    # (copies made here stay alive until the call has been enqueued)
    return (x, r, gain), args, h, y


def rmsnorm_codes(x, gain, q: int, eps: float, residual=None, h=None, out_y: bool = False, stream=None):
    """RMS norm of x + residual (fp16 or bf16 [M][K]) with `gain` [K] (or None), quantized per row to
    q-bit codes as gemm_act and gemm_decode take them.  Returns (codes int8 [M][K], fp16 scales [M],
    h), and y behind them with out_y: h is x + residual, written to `h` where one is given (x or the
    residual themselves among them), to a new tensor where there is a residual, else None."""
    torch = _torch()
    keep, args, h, y = _norm_inputs(x, gain, residual, h, out_y, stream, "rmsnorm_codes")
    M, K = x.shape
    with _on_stream(stream):
        codes = torch.empty((M, K), dtype=torch.int8, device=x.device)
        scale = torch.empty(M, dtype=torch.float16, device=x.device)
    _call(apt_rmsnorm_codes, x.device, stream,
          args + (eps, q, h.data_ptr() if h is not None else None, y.data_ptr() if y is not None else None,
                  codes.data_ptr(), scale.data_ptr()))
    del keep
    return (codes, scale, h, y) if out_y else (codes, scale, h)


def rmsnorm_mx4(x, gain, eps: float, residual=None, h=None, out_y: bool = False, stream=None):
    """As rmsnorm_codes with the row quantized to MX4.  Returns (Mx4, h), and y behind them with out_y."""
    keep, args, h, y = _norm_inputs(x, gain, residual, h, out_y, stream, "rmsnorm_mx4")
    M, K = x.shape
    out = _new_mx4(M, K, x.device, stream, "rmsnorm_mx4")
    _call(apt_rmsnorm_mx4, x.device, stream,
          args + (eps, h.data_ptr() if h is not None else None, y.data_ptr() if y is not None else None,
                  out.data.data_ptr()))
    del keep
    return (out, h, y) if out_y else (out, h)


def dequantize(codes, scale, dtype=None, stream=None):
    """The values (2 code + 1) scale of int8 codes [M][K] with fp16 scales [M], of `dtype` (fp16 by default)."""
    torch = _torch()
    dtype = torch.float16 if dtype is None else dtype
    t = _type(dtype, "dequantize")
    _require(codes.is_cuda and codes.dim() == 2 and codes.dtype == torch.int8 and scale.dtype == torch.float16 and
             tuple(scale.shape) == (codes.shape[0],) and scale.device == codes.device, "dequantize",
             "int8 codes [M][K] and fp16 scales [M]")
    M, K = codes.shape
    with _on_stream(stream):
        codes, scale = codes.contiguous(), scale.contiguous()
        out = torch.empty((M, K), dtype=dtype, device=codes.device)
    _call(apt_dequantize_codes, codes.device, stream, (codes.data_ptr(), scale.data_ptr(), M, K, t, out.data_ptr()))
    return out
