"""Microscaled 4-bit floating point (include/quick_mx.h): quantisation and
products with weights in that format.  Argument marshalling only, as in the
package's own module.

* ``mxfp4_quantize(x)`` -> (codes, scales), ``mxfp4_dequantize(codes, scales, dtype)``
* ``mxfp4_pack(codes, scales, gate_up=False)`` -> (packed, packed_scales), once per weight matrix
* ``mxfp4_gemm(codes, scales, packed, packed_scales, N, ...)``
* ``mxfp4_linear(x, packed, packed_scales, N, ...)`` on 16-bit activations
* ``mxfp4_grouped_gemm(codes, scales, offsets, packed, packed_scales, N, ...)`` over experts

    codes, scales = Q.mxfp4_quantize(weight)              # weight [N][K], f16 / bf16 / f32
    packed = Q.mxfp4_pack(codes, scales)
    y = Q.mxfp4_linear(x, *packed, N)                     # x [M][K], f16 / bf16
"""
from __future__ import annotations

import ctypes

import torch

import paper_2402_10076_amd as _q

MX_BLOCK = 32

# element types of the library (QUICK_F16, QUICK_BF16, QUICK_F32)
_TYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_TYPES16 = {torch.float16: 0, torch.bfloat16: 1}


def _declare(L):
    P, I64, SZ, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
    L.quick_mxfp4_quantize.argtypes = [P, I, I64, I64, I64, P, P, P]
    L.quick_mxfp4_dequantize.argtypes = [P, P, I, I64, I64, P, P]
    L.quick_mxfp4_packed_sizes.argtypes = [I64, I64, ctypes.POINTER(SZ), ctypes.POINTER(SZ)]
    L.quick_mxfp4_pack.argtypes = [P, P, I64, I64, I64, I, P, P, P]
    L.quick_mxfp4_gemm.argtypes = [P, P, P, P, P, I, I64, I64, I64, P, I, P]
    L.quick_mxfp4_linear.argtypes = [P, P, P, P, I, I64, I64, I64, P, I, P, SZ, P]
    L.quick_mxfp4_linear_workspace_bytes.argtypes = [I64, I64, I64]
    L.quick_mxfp4_linear_workspace_bytes.restype = SZ
    L.quick_mxfp4_grouped_gemm.argtypes = [P, P, P, P, P, P, P, I, I64, I64, I64, I64, I64, P, I, P]


EXPORTED = ("quick_mxfp4_quantize", "quick_mxfp4_dequantize", "quick_mxfp4_packed_sizes", "quick_mxfp4_pack",
            "quick_mxfp4_gemm", "quick_mxfp4_linear", "quick_mxfp4_linear_workspace_bytes",
            "quick_mxfp4_grouped_gemm")


def _fail(status, text, *a):
    raise _q.QuickError(status, text % a)


def _new(stream, ref, shape, dtype):
    """An empty tensor for a call on a given stream (on the current one a small
    call, bound by the host, asks for it without this detour)."""
    return _q._taken(stream, ref, lambda: (ref.new_empty(shape, dtype=dtype),))[0]


def _plain(t, device, dtype):
    """Whether _dev has nothing to say against t, for the usual case (a small
    call is bound by the host; _dev takes three times as long)."""
    return (type(t) is torch.Tensor and t.dtype is dtype and t.is_cuda and t.get_device() == device
            and t.is_contiguous())


def _gpu(what, name, t):
    if type(t) is torch.Tensor and t.is_cuda:
        return
    if not isinstance(t, torch.Tensor) or t.device.type != _q._DEVICE_TYPE:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: %s must be a tensor on the GPU", what, name)


def _type(what, name, dtype, types):
    code = types.get(dtype)
    if code is None:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: %s must be one of %s, not %s", what, name,
              ", ".join(str(d) for d in types), dtype)
    return code


def _channels(what, K):
    if K <= 0 or K % MX_BLOCK:
        _fail(_q.QUICK_ERR_SHAPE, "%s: the channels must be a positive multiple of 32 (K=%d)", what, K)


def _check_codes(what, codes, scales, ref=None):
    """Rows and channels of a contiguous pair codes [..., K/2], scales [..., K/32]."""
    _gpu(what, "codes", codes)
    if codes.dtype is not torch.uint8 or codes.dim() < 2 or not codes.is_contiguous():
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: codes must be a contiguous uint8 tensor [rows][K/2]", what)
    if ref is not None and codes.device != ref.device:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: codes must be on %s, not %s", what, ref.device, codes.device)
    K = codes.shape[-1] * 2
    _channels(what, K)
    if _plain(scales, codes.get_device(), torch.uint8) and scales.shape == (*codes.shape[:-1], K // MX_BLOCK):
        return K
    _q._dev(what, "scales", scales, codes, dtype=torch.uint8, shape=(*codes.shape[:-1], K // MX_BLOCK))
    return K


def mxfp4_quantize(x: torch.Tensor, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None,
                   stream=None):
    """quick_mxfp4_quantize: x [rows][K] (f16, bf16 or f32; rows may be apart
    by any stride of a multiple of 16 bytes) -> uint8 (codes [rows][K/2],
    scales [rows][K/32])."""
    what = "mxfp4_quantize"
    _gpu(what, "x", x)
    dtype = _type(what, "x", x.dtype, _TYPES)
    if x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: x must be [rows][K] with consecutive channels", what)
    rows, K = x.shape
    _channels(what, K)
    ldx = x.stride(0) if rows > 1 else K
    if ldx < K:
        _fail(_q.QUICK_ERR_SHAPE, "%s: rows of x overlap (stride %d, K=%d)", what, ldx, K)
    if codes is None:
        shape = (rows, K // 2)
        codes = x.new_empty(shape, dtype=torch.uint8) if stream is None else _new(stream, x, shape, torch.uint8)
    else:
        _q._dev(what, "codes", codes, x, dtype=torch.uint8, shape=(rows, K // 2))
    if scales is None:
        shape = (rows, K // MX_BLOCK)
        scales = x.new_empty(shape, dtype=torch.uint8) if stream is None else _new(stream, x, shape, torch.uint8)
    else:
        _q._dev(what, "scales", scales, x, dtype=torch.uint8, shape=(rows, K // MX_BLOCK))
    _q._check(_q.lib().quick_mxfp4_quantize(x.data_ptr(), dtype, ldx, rows, K, codes.data_ptr(), scales.data_ptr(),
                                            _q._stream(stream, x)), "quick_mxfp4_quantize")
    return codes, scales


def mxfp4_dequantize(codes: torch.Tensor, scales: torch.Tensor, dtype: torch.dtype = torch.float16,
                     y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """quick_mxfp4_dequantize: the values [..., K] of codes [..., K/2] and scales [..., K/32]."""
    what = "mxfp4_dequantize"
    K = _check_codes(what, codes, scales)
    code = _type(what, "dtype", dtype, _TYPES)
    shape = (*codes.shape[:-1], K)
    if y is None:
        y = codes.new_empty(shape, dtype=dtype) if stream is None else _new(stream, codes, shape, dtype)
    else:
        _q._dev(what, "y", y, codes, dtype=dtype, shape=shape)
    _q._check(_q.lib().quick_mxfp4_dequantize(codes.data_ptr(), scales.data_ptr(), code,
                                              codes.numel() // codes.shape[-1], K, y.data_ptr(),
                                              _q._stream(stream, codes)), "quick_mxfp4_dequantize")
    return y


def mxfp4_packed_sizes(N: int, K: int):
    """Bytes of one packed N x K weight matrix and of its packed scales."""
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _q._check(_q.lib().quick_mxfp4_packed_sizes(N, K, ctypes.byref(a), ctypes.byref(b)), "quick_mxfp4_packed_sizes")
    return a.value, b.value


def _matrix_bytes(what, N, K):
    """quick_mxfp4_packed_sizes' formulas."""
    if N <= 0 or N > 1 << 24 or K > 1 << 22 or N * K >= 1 << 33:
        _fail(_q.QUICK_ERR_SHAPE, "%s: unsupported weight matrix (N=%d, K=%d)", what, N, K)
    tiles = -(-N // 16)
    return tiles * -(-K // 128) * 1024, tiles * -(-K // 512) * 256


def mxfp4_pack(codes: torch.Tensor, scales: torch.Tensor, gate_up: bool = False, stream=None):
    """quick_mxfp4_pack: the form the products read of weights [N][K] or of E
    experts' [E][N][K], given as codes and scales; uint8 (packed,
    packed_scales), [E][...] for experts.  gate_up: the first N/2 rows are the
    gate, the others the up projection of a gated SiLU."""
    what = "mxfp4_pack"
    K = _check_codes(what, codes, scales)
    if codes.dim() > 3:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: codes must be [N][K/2] or [E][N][K/2]", what)
    N = codes.shape[-2]
    E = codes.shape[0] if codes.dim() == 3 else 1
    pb, sb = _matrix_bytes(what, N, K)
    lead = (E,) if codes.dim() == 3 else ()
    packed, pscales = (_new(stream, codes, (*lead, n), torch.uint8) for n in (pb, sb))
    _q._check(_q.lib().quick_mxfp4_pack(codes.data_ptr(), scales.data_ptr(), E, N, K, int(bool(gate_up)),
                                        packed.data_ptr(), pscales.data_ptr(), _q._stream(stream, codes)),
              "quick_mxfp4_pack")
    return packed, pscales


def _check_packed(what, ref, packed, pscales, N, K, E=1):
    pb, sb = _matrix_bytes(what, N, K)
    if (isinstance(packed, torch.Tensor) and isinstance(pscales, torch.Tensor) and ref.is_cuda and packed.is_cuda
            and pscales.is_cuda and ref.get_device() == packed.get_device() == pscales.get_device()
            and packed.is_contiguous() and pscales.is_contiguous() and packed.nbytes >= E * pb
            and pscales.nbytes >= E * sb):
        return
    _q._dev(what, "packed", packed, ref, nbytes=E * pb)
    _q._dev(what, "packed_scales", pscales, ref, nbytes=E * sb)


def _out(what, y, ref, rows, N, activation, dtype, stream):
    if activation == _q.ACT_SILU_GATE:
        if N % 32:
            _fail(_q.QUICK_ERR_SHAPE, "%s: gated columns come in tiles of 32 (N=%d)", what, N)
        N //= 2
    if y is None:
        return ref.new_empty((rows, N), dtype=dtype) if stream is None else _new(stream, ref, (rows, N), dtype)
    _q._dev(what, "y", y, ref, dtype=dtype, shape=(rows, N))
    return y


def _bias(what, bias, ref, n, dtype):
    if bias is None:
        return None
    _q._dev(what, "bias", bias, ref, dtype=dtype, nbytes=2 * n)
    return bias.data_ptr()


def mxfp4_gemm(codes: torch.Tensor, scales: torch.Tensor, packed: torch.Tensor, packed_scales: torch.Tensor, N: int,
               bias: torch.Tensor | None = None, activation: int = 0, y: torch.Tensor | None = None,
               dtype: torch.dtype = torch.float16, stream=None) -> torch.Tensor:
    """quick_mxfp4_gemm: y = epilogue(x . W^T + bias), x [M][K] given as codes
    and scales, W [N][K] packed; bias of y's ``dtype`` in the logical column
    order; ``activation`` = ACT_SILU_GATE (weights packed with gate_up) gives
    [M][N/2]."""
    what = "mxfp4_gemm"
    K = _check_codes(what, codes, scales)
    if codes.dim() != 2:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: codes must be [M][K/2]", what)
    if y is not None:
        dtype = y.dtype
    code = _type(what, "dtype", dtype, _TYPES16)
    M = codes.shape[0]
    _check_packed(what, codes, packed, packed_scales, N, K)
    b = _bias(what, bias, codes, N, dtype)
    y = _out(what, y, codes, M, N, activation, dtype, stream)
    _q._check(_q.lib().quick_mxfp4_gemm(codes.data_ptr(), scales.data_ptr(), packed.data_ptr(),
                                        packed_scales.data_ptr(), y.data_ptr(), code, M, N, K, b, int(activation),
                                        _q._stream(stream, codes)), "quick_mxfp4_gemm")
    return y


def mxfp4_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(_q.lib().quick_mxfp4_linear_workspace_bytes(M, N, K))


def mxfp4_linear(x: torch.Tensor, packed: torch.Tensor, packed_scales: torch.Tensor, N: int,
                 bias: torch.Tensor | None = None, activation: int = 0, y: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """quick_mxfp4_linear: mxfp4_gemm of 16-bit activations x [M][K], which the
    call quantises; y and bias have x's type.  ``workspace``: a tensor of
    mxfp4_linear_workspace_bytes(M, N, K); one is taken from torch's allocator
    if none is given."""
    what = "mxfp4_linear"
    _gpu(what, "x", x)
    code = _type(what, "x", x.dtype, _TYPES16)
    if x.dim() != 2 or not x.is_contiguous():
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: x must be a contiguous [M][K] tensor", what)
    M, K = x.shape
    _channels(what, K)
    _check_packed(what, x, packed, packed_scales, N, K)
    b = _bias(what, bias, x, N, x.dtype)
    y = _out(what, y, x, M, N, activation, x.dtype, stream)
    L = _q.lib()
    hs = _q._stream(stream, x)
    if workspace is None:
        wsb = L.quick_mxfp4_linear_workspace_bytes(M, N, K)
        if wsb:
            if stream is None:
                workspace = x.new_empty(wsb, dtype=torch.uint8)
            else:
                workspace = _q._taken(stream, x, lambda: x.new_empty(wsb, dtype=torch.uint8), kept=False)
    else:
        _q._dev(what, "workspace", workspace, x)
        wsb = workspace.nbytes
    _q._check(L.quick_mxfp4_linear(x.data_ptr(), packed.data_ptr(), packed_scales.data_ptr(), y.data_ptr(), code, M, N,
                                   K, b, int(activation), workspace.data_ptr() if wsb else None, wsb, hs),
              "quick_mxfp4_linear")
    return y


def mxfp4_grouped_gemm(codes: torch.Tensor, scales: torch.Tensor, offsets: torch.Tensor, packed: torch.Tensor,
                       packed_scales: torch.Tensor, N: int, rows: torch.Tensor | None = None, R: int | None = None,
                       bias: torch.Tensor | None = None, activation: int = 0, y: torch.Tensor | None = None,
                       dtype: torch.dtype = torch.float16, stream=None) -> torch.Tensor:
    """quick_mxfp4_grouped_gemm: y[r] = epilogue(x[rows[r]] . W_e^T + bias_e)
    for offsets[e] <= r < offsets[e+1]; offsets int32 [E+1], rows int32 [R]
    (None: row r reads x[r]; R defaults to x's rows), bias [E][N]."""
    what = "mxfp4_grouped_gemm"
    K = _check_codes(what, codes, scales)
    if codes.dim() != 2:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: codes must be [T][K/2]", what)
    T = codes.shape[0]
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.numel() < 2:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: offsets must be an int32 vector of E+1 entries", what)
    _q._dev(what, "offsets", offsets, codes, dtype=torch.int32)
    E = offsets.numel() - 1
    if rows is not None:
        if not isinstance(rows, torch.Tensor) or rows.dim() != 1:
            _fail(_q.QUICK_ERR_INVALID_ARG, "%s: rows must be an int32 vector", what)
        _q._dev(what, "rows", rows, codes, dtype=torch.int32)
        if R is not None and R != rows.numel():
            _fail(_q.QUICK_ERR_SHAPE, "%s: R disagrees with rows", what)
        R = rows.numel()
    elif R is None:
        R = T
    if y is not None:
        dtype = y.dtype
    code = _type(what, "dtype", dtype, _TYPES16)
    _check_packed(what, codes, packed, packed_scales, N, K, E)
    b = _bias(what, bias, codes, E * N, dtype)
    y = _out(what, y, codes, R, N, activation, dtype, stream)
    _q._check(_q.lib().quick_mxfp4_grouped_gemm(
        codes.data_ptr(), scales.data_ptr(), rows.data_ptr() if rows is not None else None, offsets.data_ptr(),
        packed.data_ptr(), packed_scales.data_ptr(), y.data_ptr(), code, T, R, E, N, K, b, int(activation),
        _q._stream(stream, codes)), "quick_mxfp4_grouped_gemm")
    return y
