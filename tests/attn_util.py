"""Plain binary64 forms of rotary positions, the paged 4-bit cache, attention
over it and low-rank adapters, from their definitions, on the CPU.  Test
infrastructure: shares no code with the library."""
from __future__ import annotations

import math

import numpy as np
import torch

import mx_util as U

PAGE = 64
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# half a step of each type, relative to the value
STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def gen(*seed):
    g = torch.Generator()
    g.manual_seed(sum((i + 1) * 7919 * int(s) for i, s in enumerate(seed)) % (1 << 31))
    return g


def normal(g, *shape, scale=1.0, dtype=torch.float16):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def rotated(x, positions, freqs, interleaved=False, factor=1.0, inverse=False):
    """(values, bound of the error of binary32 arithmetic) of x [T][H][D] float64."""
    r = 2 * freqs.shape[0]
    angle = positions.double().view(-1, 1, 1) * freqs.double()
    c, s = torch.cos(angle) * factor, torch.sin(angle) * factor
    if inverse:
        s = -s
    out, size = x.clone(), torch.zeros_like(x)
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    p, q = x[..., a], x[..., b]
    out[..., a], out[..., b] = p * c - q * s, q * c + p * s
    size[..., a] = size[..., b] = p.abs() + q.abs()
    # cosine and sine: half a turn's angle in binary32 (pi * 2^-25) and the functions' last places; two products, a sum
    return out, size * abs(factor) * (math.pi * 2.0 ** -25 + 6 * 2.0 ** -24)


def record(k, v, dim):
    """One page's head [68 * dim] of codes and scales, from the layout's definition.  k, v: 64 rows of (codes, scales)."""
    rec = np.zeros(68 * dim, np.uint8)
    w = min(dim, 128) // 16
    for t in range(PAGE):
        for c in range(0, dim, 2):
            rec[t * dim // 2 + c // 2] = k[0][t][c // 2]
            x = c % 128
            rec[34 * dim + c // 128 * 4096 + t // 4 * 32 * w + ((x // w) * 4 + t % 4) * w // 2 + x % w // 2] = v[0][t][c // 2]
        for b in range(dim // 32):
            rec[32 * dim + 64 * b + 4 * (t % 16) + t // 16] = k[1][t][b]
            rec[66 * dim + 64 * b + 16 * (t % 16 // 4) + 4 * (t // 16) + t % 4] = v[1][t][b]
    return rec


def rounded(x):
    """Binary64 values that a 16-bit tensor [..., d] has in the cache."""
    if not x.numel():
        return x.double()
    flat = x.double().reshape(-1, x.shape[-1]).numpy()
    return torch.from_numpy(U.values(*U.quantize(flat))).view(x.shape)


def attention(q, k, v, lengths, offsets, group, dtype, scale=None, window=0, causal=True, known=None):
    """(out, lse, tolerance) of q [T][HQ][D] float64 over k[b], v[b] [tokens][H][D] float64 of each sequence.
    ``known``: [b] of booleans, tokens whose page the cache has."""
    T, HQ, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((T, HQ), -math.inf, dtype=torch.float64)
    step = STEP[dtype]
    for b, n in enumerate(lengths):
        rows = slice(offsets[b], offsets[b + 1])
        m = offsets[b + 1] - offsets[b]
        if m == 0:
            continue
        at = torch.arange(n).view(1, -1)
        pos = torch.arange(n - m, n).view(-1, 1)
        seen = torch.ones(m, n, dtype=torch.bool)
        if causal:
            seen = at <= pos
            if window:
                seen = seen & (at > pos - window)
        if known is not None:
            seen = seen & known[b].view(1, -1)
        for h in range(HQ):
            if n == 0:
                continue
            kk, vv, qq = k[b][:, h // group], v[b][:, h // group], q[rows, h]
            s = qq @ kk.t() * scale
            # binary32 sums of D products, two more roundings; and of s log2(e)
            off = (qq.abs() @ kk.abs().t() * abs(scale)) * (D + 4) * 2.0 ** -24
            s = s.masked_fill(~seen, -math.inf)
            top = s.amax(1, keepdim=True)
            p = torch.exp(s - torch.where(top > -math.inf, top, 0))
            total = p.sum(1, keepdim=True)
            p = p / torch.where(total > 0, total, 1)
            p = torch.where(seen, p, 0)
            # what is hidden does not enter, whatever it is
            one = torch.stack([p[i][seen[i]] @ vv[seen[i]] for i in range(m)]) if m else p @ vv
            size = torch.stack([p[i][seen[i]] @ vv[seen[i]].abs() for i in range(m)])
            far = torch.where(seen, off, 0).amax(1, keepdim=True) + 2.0 ** -20   # of a weight: its score, exp2
            out[rows, h] = one
            # weights rounded to the type; they and their sum off by `far`; binary32 sums of n; weights that f16
            # holds below its normal range (2^-25 of a largest of 2^6 or more); the result rounded
            # (f16: steps of 2^-24 below 2^-14, so that half of one, 2^-25, is the least: a result of 4.0745e-6 became
            # 68 * 2^-24 = 4.0531e-6, off by 2.14e-8 of 2^-25 = 2.98e-8)
            least = 2.0 ** -25 if dtype is torch.float16 else 0.0
            tol[rows, h] = (size * (step + 2 * far + n * 2.0 ** -23)
                            + n * 2.0 ** -31 * vv[:, :].abs().nan_to_num(0).amax() + (one.abs() * step).clamp(min=least)
                            + 1e-30)
            lse[rows, h] = torch.where(total > 0, top + torch.log(total), -math.inf).squeeze(1)
    return out, lse, tol


def adapters(y, x, a, b, ids, scales, dtype):
    """(out, tolerance) in binary64."""
    out, tol = y.double().clone(), y.double().abs() * 0
    step, r, K = STEP[dtype], a.shape[1], x.shape[1]
    for t in range(x.shape[0]):
        e = int(ids[t])
        if 0 <= e < a.shape[0]:
            s = float(scales[e]) if scales is not None else 1.0
            low = s * (a[e].double() @ x[t].double())
            size = abs(s) * (a[e].double().abs() @ x[t].double().abs())
            off = low.abs() * step + size * (K + 2) * 2.0 ** -24 + 2.0 ** -25 * (dtype == torch.float16)
            out[t] += b[e].double() @ low
            tol[t] = b[e].double().abs() @ (off + low.abs() * (r + 2) * 2.0 ** -24) + y[t].double().abs() * 2.0 ** -23
    return out, tol + out.abs() * step + 1e-30
