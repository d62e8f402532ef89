"""Around the grouped products of a mixture-of-experts layer
(include/quick_moe.h).  Argument marshalling only, as in the package's own
module.

* ``moe_route(logits, topk, ...)`` -> Routing(ids, weights, offsets, rows, slots)
* ``moe_combine(y, slots, weights, residual=None)``

    r = Q.moe_route(logits, 2)
    h = Q.grouped_gemm_fused(x, r.offsets, *w13, 2 * F, rows=r.rows, activation=Q.ACT_SILU_GATE)
    out = Q.moe_combine(Q.grouped_gemm(h, r.offsets, *w2, D), r.slots, r.weights)
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple

import torch

import paper_2402_10076_amd as _q
from paper_2402_10076_amd.mx import _TYPES, _TYPES16, _fail, _gpu, _new, _plain, _type

SCORE_SOFTMAX = 0
SCORE_SIGMOID = 1
MAX_TOPK = 16
MAX_GROUPS = 64
MAX_EXPERTS = 512


class QuickRoute(ctypes.Structure):
    _fields_ = [("score", ctypes.c_int), ("topk", ctypes.c_int), ("groups", ctypes.c_int),
                ("topk_groups", ctypes.c_int), ("group_best", ctypes.c_int), ("renormalize", ctypes.c_int),
                ("scale", ctypes.c_float)]


class Routing(NamedTuple):
    """ids int32 and weights f32 [T][topk]; offsets int32 [E+1] and rows int32
    [T*topk] for the grouped products; slots int32 [T][topk] for moe_combine."""
    ids: torch.Tensor
    weights: torch.Tensor
    offsets: torch.Tensor
    rows: torch.Tensor
    slots: torch.Tensor


def _declare(L):
    P, I64, SZ, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
    L.quick_moe_route.argtypes = [P, I, I64, I64, ctypes.POINTER(QuickRoute), P, P, P, P, P, P, P, SZ, P]
    L.quick_moe_route_workspace_bytes.argtypes = [I64, I64, I64]
    L.quick_moe_route_workspace_bytes.restype = SZ
    L.quick_moe_combine.argtypes = [P, I, I64, I64, P, P, I64, I64, P, P, P]


EXPORTED = ("quick_moe_route", "quick_moe_route_workspace_bytes", "quick_moe_combine")


@functools.lru_cache(maxsize=64)
def _options(*fields):
    """The C struct of a set of options (building it takes as long as a check of all arguments)."""
    return QuickRoute(*fields)


def _routing(dev, T, E, topk):
    ids = torch.empty((T, topk), dtype=torch.int32, device=dev)
    return Routing(ids, torch.empty((T, topk), dtype=torch.float32, device=dev), ids.new_empty(E + 1),
                   ids.new_empty(T * topk), ids.new_empty((T, topk)))


def moe_route_workspace_bytes(T: int, E: int, topk: int) -> int:
    return int(_q.lib().quick_moe_route_workspace_bytes(T, E, topk))


def moe_route(logits: torch.Tensor, topk: int, score: int = SCORE_SOFTMAX, bias: torch.Tensor | None = None,
              groups: int = 1, topk_groups: int = 1, group_best: int = 1, renormalize: bool = True,
              scale: float = 1.0, out: Routing | None = None, workspace: torch.Tensor | None = None,
              stream=None) -> Routing:
    """quick_moe_route: logits [T][E] (f16, bf16 or f32, contiguous) -> Routing.

    score: SCORE_SOFTMAX or SCORE_SIGMOID; bias: f32 [E], added for the choice
    alone; groups / topk_groups / group_best: only the topk_groups best of
    that many groups of consecutive experts are chosen from, by the sum of
    their group_best (1 or 2) largest choices; weights are divided by their
    sum with ``renormalize`` and multiplied by ``scale``."""
    what = "moe_route"
    _gpu(what, "logits", logits)
    dtype = _type(what, "logits", logits.dtype, _TYPES)
    if logits.dim() != 2 or not logits.is_contiguous():
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: logits must be a contiguous [T][E] tensor", what)
    T, E = logits.shape
    if not 1 <= E <= MAX_EXPERTS or not 1 <= topk <= MAX_TOPK or T > 1 << 30 or T * topk >= 1 << 31:
        _fail(_q.QUICK_ERR_SHAPE, "%s: unsupported sizes (T=%d, E=%d, topk=%d)", what, T, E, topk)
    if bias is not None:
        _q._dev(what, "bias", bias, logits, dtype=torch.float32, shape=(E,))
    if out is None:
        if stream is None:
            out = _routing(logits.device, T, E, topk)
        else:
            out = _q._taken(stream, logits, lambda: _routing(logits.device, T, E, topk))
    else:
        for name, shape in (("ids", (T, topk)), ("weights", (T, topk)), ("offsets", (E + 1,)), ("rows", (T * topk,)),
                            ("slots", (T, topk))):
            _q._dev(what, name, getattr(out, name), logits,
                    dtype=torch.float32 if name == "weights" else torch.int32, shape=shape)
    L = _q.lib()
    hs = _q._stream(stream, logits)
    if workspace is None:
        wsb = L.quick_moe_route_workspace_bytes(T, E, topk)
        if wsb:
            if stream is None:
                workspace = torch.empty(wsb, dtype=torch.uint8, device=logits.device)
            else:
                workspace = _q._taken(stream, logits, lambda: logits.new_empty(wsb, dtype=torch.uint8), kept=False)
    else:
        _q._dev(what, "workspace", workspace, logits)
        wsb = workspace.nbytes
    r = _options(score, topk, groups, topk_groups, group_best, int(bool(renormalize)), scale)
    _q._check(L.quick_moe_route(logits.data_ptr(), dtype, T, E, ctypes.byref(r),
                                bias.data_ptr() if bias is not None else None, out.ids.data_ptr(),
                                out.weights.data_ptr(), out.offsets.data_ptr(), out.rows.data_ptr(),
                                out.slots.data_ptr(), workspace.data_ptr() if wsb else None, wsb, hs),
              "quick_moe_route")
    return out


def moe_combine(y: torch.Tensor, slots: torch.Tensor, weights: torch.Tensor, residual: torch.Tensor | None = None,
                out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """quick_moe_combine: out[t] = residual[t] + sum_j weights[t][j] *
    y[slots[t][j]]; y [R][D] f16 or bf16, slots int32 and weights f32
    [T][topk] (a Routing's); a slot outside y adds nothing."""
    what = "moe_combine"
    _gpu(what, "y", y)
    dtype = _type(what, "y", y.dtype, _TYPES16)
    if y.dim() != 2 or not y.is_contiguous():
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: y must be a contiguous [R][D] tensor", what)
    if not isinstance(slots, torch.Tensor) or slots.dim() != 2:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: slots must be an int32 [T][topk] tensor", what)
    R, D = y.shape
    T, topk = slots.shape
    dev = y.get_device()
    if not (_plain(slots, dev, torch.int32) and _plain(weights, dev, torch.float32) and weights.shape == slots.shape):
        _q._dev(what, "slots", slots, y, dtype=torch.int32)
        _q._dev(what, "weights", weights, y, dtype=torch.float32, shape=(T, topk))
    if residual is not None and not (_plain(residual, dev, y.dtype) and residual.shape == (T, D)):
        _q._dev(what, "residual", residual, y, dtype=y.dtype, shape=(T, D))
    if out is None:
        out = y.new_empty((T, D)) if stream is None else _new(stream, y, (T, D), y.dtype)
    else:
        _q._dev(what, "out", out, y, dtype=y.dtype, shape=(T, D))
    _q._check(_q.lib().quick_moe_combine(y.data_ptr(), dtype, R, D, slots.data_ptr(), weights.data_ptr(), T, topk,
                                         residual.data_ptr() if residual is not None else None, out.data_ptr(),
                                         _q._stream(stream, y)), "quick_moe_combine")
    return out
