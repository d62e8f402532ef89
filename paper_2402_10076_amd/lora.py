"""Low-rank adapters of many requests beside a projection that they share
(include/quick_lora.h).  Argument marshalling only, as in the package's own
module.

* ``lora_group(ids, E)`` -> (offsets, rows), once a step
* ``lora_add(y, x, a, b, offsets, rows, scales=None)``, for each projection

    offsets, rows = Q.lora_group(ids, E)                 # ids int32 [T], -1: no adapter
    y = Q.w4a16_gemm(x, *w, N)
    y = Q.lora_add(y, x, a, b, offsets, rows, scales, out=y)
"""
from __future__ import annotations

import ctypes
import functools

import torch

import paper_2402_10076_amd as _q
from paper_2402_10076_amd.attention import _int32, _run
from paper_2402_10076_amd.mx import _TYPES16, _fail, _gpu, _new, _plain, _type

LORA_MAX_RANK = 128


def _declare(L):
    P, I64, SZ, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
    L.quick_lora_group.argtypes = [P, I64, I64, P, P, P]
    L.quick_lora_add.argtypes = [P, I64, I, I64, I64, I64, I64, I64, P, P, P, P, P, I64, P, I64, P, I64, P, SZ, P]
    L.quick_lora_workspace_bytes.argtypes = [I64, I64, I64, I64]
    L.quick_lora_workspace_bytes.restype = SZ


EXPORTED = ("quick_lora_group", "quick_lora_add", "quick_lora_workspace_bytes")


def lora_group(ids: torch.Tensor, E: int, stream=None):
    """quick_lora_group: int32 (offsets [E+1], rows [T]) of the tokens' adapters
    ids (int32 [T]; outside 0..E-1: none)."""
    what = "lora_group"
    _gpu(what, "ids", ids)
    if ids.dim() != 1:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: ids must be an int32 vector", what)
    _int32(what, "ids", ids, ids, ids.shape)
    if not 1 <= E <= _q.MAX_EXPERTS:
        _fail(_q.QUICK_ERR_SHAPE, "%s: 1 to %d adapters, not %d", what, _q.MAX_EXPERTS, E)
    T = ids.shape[0]
    if stream is None:
        offsets, rows = ids.new_empty(E + 1), ids.new_empty(T)
    else:
        offsets, rows = _q._taken(stream, ids, lambda: (ids.new_empty(E + 1), ids.new_empty(T)))
    _run(ids, "quick_lora_group", ids.data_ptr(), T, E, offsets.data_ptr(), rows.data_ptr(), _q._stream(stream, ids))
    return offsets, rows


def _rows(what, name, t, ref, T, n):
    """Row stride of t [T][n] (rows of consecutive values) of ref's type."""
    if not isinstance(t, torch.Tensor) or t.device != ref.device:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: %s must be a tensor on %s", what, name, ref.device)
    if t.dtype is not ref.dtype or t.dim() != 2 or t.shape != (T, n) or (n > 1 and t.stride(1) != 1):
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: %s must be %s [%d][%d] with consecutive columns", what, name, ref.dtype, T, n)
    ld = t.stride(0) if T > 1 else n
    if ld < n:
        _fail(_q.QUICK_ERR_SHAPE, "%s: rows of %s overlap", what, name)
    return ld


@functools.lru_cache(maxsize=256)
def lora_workspace_bytes(R: int, K: int, E: int, rank: int) -> int:
    return int(_q.lib().quick_lora_workspace_bytes(R, K, E, rank))


def _usual(x, y, a, b, offsets, rows, scales):
    """Whether the checks have nothing to say against a call of contiguous
    tensors (a small call is bound by the host; one by one they take 3 us)."""
    if not (x.is_cuda and y.is_cuda and a.is_cuda and b.is_cuda and offsets.is_cuda and rows.is_cuda):
        return False
    dev, dtype, i32 = x.get_device(), x.dtype, torch.int32
    if not (y.get_device() == a.get_device() == b.get_device() == offsets.get_device() == rows.get_device() == dev
            and y.dtype is dtype and a.dtype is dtype and b.dtype is dtype and offsets.dtype is i32 and rows.dtype is i32
            and x.is_contiguous() and y.is_contiguous() and a.is_contiguous() and b.is_contiguous()
            and offsets.is_contiguous() and rows.is_contiguous()):
        return False
    if not (x.dim() == y.dim() == 2 and a.dim() == b.dim() == 3 and offsets.dim() == rows.dim() == 1):
        return False
    (T, K), (E, rank, k), (e, N, r) = x.shape, a.shape, b.shape
    return (k == K and e == E and r == rank and y.shape == (T, N) and offsets.shape[0] == E + 1 and rows.shape[0] <= T
            and (scales is None or (_plain(scales, dev, torch.float32) and scales.shape == (E,))))


def lora_add(y: torch.Tensor, x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, offsets: torch.Tensor,
             rows: torch.Tensor, scales: torch.Tensor | None = None, out: torch.Tensor | None = None,
             workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """quick_lora_add: y [T][N] + scales[e] * (x [T][K] . a[e]^T) . b[e]^T for
    the tokens of each adapter e, y for those without one; f16 or bf16, a
    [E][rank][K], b [E][N][rank], scales f32 [E] (None: 1), offsets and rows of
    lora_group.  Rows of x, y and out may be apart by any multiple of 8.  out: y
    itself or another tensor of its shape, whose rows keep their values where
    ``rows`` does not list them; a new one if none is given, with y's there."""
    what = "lora_add"
    _gpu(what, "x", x)
    code = _type(what, "x", x.dtype, _TYPES16)
    if all(type(t) is torch.Tensor for t in (y, a, b, offsets, rows)) and _usual(x, y, a, b, offsets, rows, scales):
        (T, K), (E, N, rank), R = x.shape, b.shape, rows.shape[0]
        ldx, ldy = K, N
    else:
        if x.dim() != 2 or not isinstance(y, torch.Tensor) or y.dim() != 2:
            _fail(_q.QUICK_ERR_INVALID_ARG, "%s: x and y must be [T][K] and [T][N]", what)
        (T, K), N = x.shape, y.shape[1]
        ldx, ldy = _rows(what, "x", x, x, T, K), _rows(what, "y", y, x, T, N)
        if not isinstance(a, torch.Tensor) or a.dim() != 3:
            _fail(_q.QUICK_ERR_INVALID_ARG, "%s: a must be [E][rank][K]", what)
        E, rank = a.shape[:2]
        _q._dev(what, "a", a, x, dtype=x.dtype, shape=(E, rank, K))
        _q._dev(what, "b", b, x, dtype=x.dtype, shape=(E, N, rank))
        if scales is not None:
            _q._dev(what, "scales", scales, x, dtype=torch.float32, shape=(E,))
        _int32(what, "offsets", offsets, x, (E + 1,))
        if not isinstance(rows, torch.Tensor) or rows.dim() != 1 or rows.shape[0] > T:
            _fail(_q.QUICK_ERR_INVALID_ARG, "%s: rows must be an int32 vector of the tokens", what)
        R = rows.shape[0]
        _int32(what, "rows", rows, x, (R,))
    if out is None:
        if R < T:
            # the rows that are not listed
            out = _q._taken(stream, x, lambda: (y.clone(memory_format=torch.contiguous_format),))[0]
        else:
            out = x.new_empty((T, N)) if stream is None else _new(stream, x, (T, N), x.dtype)
        ldo = N
    else:
        ldo = _rows(what, "out", out, x, T, N)
        if out.data_ptr() == y.data_ptr() and ldo != ldy and y.numel():
            _fail(_q.QUICK_ERR_INVALID_ARG, "%s: out must be y with y's strides, or apart from it", what)
    if workspace is None:
        need = lora_workspace_bytes(R, K, E, rank)
        if need:
            if stream is None:
                workspace = x.new_empty(need, dtype=torch.uint8)
            else:
                workspace = _q._taken(stream, x, lambda: x.new_empty(need, dtype=torch.uint8), kept=False)
    else:
        _q._dev(what, "workspace", workspace, x)
        need = workspace.nbytes
    _run(x, "quick_lora_add", x.data_ptr(), ldx, code, T, K, N, E, rank, a.data_ptr(), b.data_ptr(),
         scales.data_ptr() if scales is not None else None, offsets.data_ptr(), rows.data_ptr(), R, y.data_ptr(), ldy,
         out.data_ptr(), ldo, workspace.data_ptr() if workspace is not None else None, need, _q._stream(stream, x))
    return out
