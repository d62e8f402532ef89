"""Plain binary64 forms of the microscaled 4-bit floating-point and
mixture-of-experts operators, in numpy, element by element from their
definitions.  Test infrastructure: shares no code with the library."""
from __future__ import annotations

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def bf16_values(bits):
    return (np.asarray(bits, np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)


def quantize(x):
    """(codes [m][k/2], scales [m][k/32]) uint8 of binary64 values that a 16- or 32-bit type holds."""
    m, k = x.shape
    b = np.abs(x.reshape(m, k // 32, 32))
    neg = np.signbit(x.reshape(m, k // 32, 32))
    bad = ~np.isfinite(b).all(2)
    a = np.where(bad[..., None], 0, b).max(2)
    # binary32 exponent field of a: 0 below 2^-126
    with np.errstate(divide="ignore"):
        e = np.where(a >= 2.0 ** -126, np.floor(np.log2(np.where(a > 0, a, 1))), -127) + 127
    e = np.where((a >= 2.0 ** -126) & (np.ldexp(1.0, (e - 127).astype(int)) > a), e - 1, e)   # log2's last bit
    e = np.where((a >= 2.0 ** -126) & (np.ldexp(1.0, (e - 126).astype(int)) <= a), e + 1, e)
    s = np.maximum(e - 2, 0).astype(int)
    v = np.where(bad[..., None], 0, b) * np.ldexp(1.0, 127 - s)[..., None]
    # nearest grid value; of two equally near ones the even code
    d = np.abs(v[..., None] - GRID)
    near = d == d.min(-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = np.where(bad[..., None], 0, code + 8 * neg).reshape(m, k // 2, 2).astype(np.uint8)
    return code[..., 0] | code[..., 1] << 4, np.where(bad, 255, s).astype(np.uint8)


def values(codes, scales):
    """Binary64 values [..., k]; NaN where the scale is."""
    codes = np.asarray(codes)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*scales.shape, 32)
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return (v * unit[..., None]).reshape(*scales.shape[:-1], -1)


def silu_gate(h):
    n = h.shape[-1] // 2
    g, u = h[..., :n], h[..., n:]
    return g / (1 + np.exp(-g)) * u


def packed(codes, scales, gate_up=False):
    """The packed form of one matrix, from the layout's definition."""
    N, K = codes.shape[0], codes.shape[1] * 2
    if gate_up:
        t = np.arange(N)
        src = (t // 32) * 16 + t % 16 + np.where(t % 32 >= 16, N // 2, 0)
        codes, scales = codes[src], scales[src]
    nt, ks, kq = -(-N // 16), -(-K // 128), -(-K // 512)
    c = np.zeros((nt * 16, ks * 64), np.uint8)
    c[:N, :K // 2] = codes
    s = np.zeros((nt * 16, kq * 16), np.uint8)
    s[:N, :K // 32] = scales
    c = c.reshape(nt, 16, ks, 4, 16).transpose(0, 2, 3, 1, 4)      # tile, step, block, row, byte
    s = s.reshape(nt, 16, kq, 4, 4).transpose(0, 2, 4, 1, 3)       # tile, quad, block, row, step
    return np.ascontiguousarray(c).reshape(-1), np.ascontiguousarray(s).reshape(-1)


def route(logits, topk, sigmoid=False, bias=None, groups=1, topk_groups=1, group_best=1, renormalize=True, scale=1.0):
    """(ids, weights, c) of binary64 logits [T][E]."""
    T, E = logits.shape
    with np.errstate(all="ignore"):
        if sigmoid:
            s = 1 / (1 + np.exp(-logits))
        else:
            m = np.where(np.isnan(logits), -np.inf, logits).max(1, keepdims=True)
            ex = np.where(logits == -np.inf, 0, np.exp(logits - m))
            total = ex.sum(1, keepdims=True)
            s = np.where(total == 0, 0, ex / total)
        c = s if sigmoid or bias is not None or (groups > 1 and group_best > 1) else logits
        if bias is not None:
            c = c + bias
        c = np.where(np.isnan(c), -np.inf, c)
        keep = np.ones((T, E), bool)
        if groups > 1:
            g = np.sort(c.reshape(T, groups, -1), 2)[:, :, ::-1][:, :, :group_best].sum(2)
            order = np.argsort(-np.where(np.isnan(g), -np.inf, g), axis=1, kind="stable")
            kept = np.zeros((T, groups), bool)
            np.put_along_axis(kept, order[:, :topk_groups], True, 1)
            keep = np.repeat(kept, E // groups, 1)
        # kept experts first, by descending c, then by index
        ids = np.lexsort((np.broadcast_to(np.arange(E), (T, E)), -c, ~keep), axis=1)[:, :topk]
        w = np.take_along_axis(s, ids, 1)
        if renormalize:
            total = w.sum(1, keepdims=True)
            w = np.where(total == 0, 0, w / total)
    return ids, w * scale, c


def sort_rows(ids, E):
    """(offsets, rows, slots) of the routed rows, by expert, then by token and choice."""
    T, k = ids.shape
    flat = ids.reshape(-1)
    order = np.argsort(flat, kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E))])
    slots = np.empty(T * k, np.int64)
    slots[order] = np.arange(T * k)
    return offsets, order // k, slots.reshape(T, k)
