"""Between the projections of an attention layer (include/quick_attention.h):
rotary positions, a paged cache of keys and values in 4 bits, and attention
over it.  Argument marshalling only, as in the package's own module.

* ``rotary_frequencies(dim, ...)`` -> (freqs, factor), ``rotary(x, positions, freqs, ...)``
* ``kv4_cache(pages, heads, dim)``; ``kv4_write(cache, k, v, slots)``, ``kv4_read(cache, slots)`` -> (k, v)
* ``kv4_attention(q, cache, table, lengths, ...)``

    qkv = Q.w4a16_gemm(x, *w, (HQ + 2 * H) * D).view(T, HQ + 2 * H, D)
    qk = Q.rotary(qkv[:, :HQ + H], positions, freqs)
    Q.kv4_write(cache, qk[:, HQ:], qkv[:, HQ + H:], slots)
    o = Q.kv4_attention(qk[:, :HQ], cache, table, lengths)       # [T][HQ][D]
"""
from __future__ import annotations

import ctypes
import functools
import math

import torch

import paper_2402_10076_amd as _q
from paper_2402_10076_amd.mx import _TYPES, _TYPES16, _fail, _gpu, _new, _plain, _type

KV4_PAGE = 64
KV4_DIMS = (64, 128, 256)


class QuickAttention(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("T", "q_heads", "heads", "D", "pages", "seqs", "table_width", "most",
                                               "q_token", "q_head", "window")] +
                [("causal", ctypes.c_int), ("scale", ctypes.c_float)])


def _declare(L):
    P, I64, SZ, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
    A = ctypes.POINTER(QuickAttention)
    L.quick_rotary.argtypes = [P, I, I64, I64, I64, I64, I64, P, P, I64, I, I, ctypes.c_float, P, I64, I64, P]
    L.quick_kv4_write.argtypes = [P, P, I, I64, I64, I64, I64, P, I64, I64, I64, P, I64, P]
    L.quick_kv4_read.argtypes = [P, I64, P, I64, I64, I64, I, P, P, P]
    L.quick_kv4_attention.argtypes = [A, P, I, P, P, P, P, P, P, P, SZ, P]
    L.quick_kv4_attention_workspace_bytes.argtypes = [A]
    L.quick_kv4_attention_workspace_bytes.restype = SZ


EXPORTED = ("quick_rotary", "quick_kv4_write", "quick_kv4_read", "quick_kv4_attention",
            "quick_kv4_attention_workspace_bytes")

_device_now = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _run(ref, name, *args):
    """The library's call, on the device of ``ref`` (its streams' handles mean nothing on another one)."""
    f = getattr(_q.lib(), name)
    if ref.is_cuda and _device_now() != ref.get_device():
        with torch.cuda.device(ref.device):
            st = f(*args)
    else:
        st = f(*args)
    if st:
        _q._check(st, name)


def _int32(what, name, t, ref, shape):
    if _plain(t, ref.get_device(), torch.int32) and t.shape == shape:
        return
    _q._dev(what, name, t, ref, dtype=torch.int32, shape=shape)


def rotary_frequencies(dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                       original: int = 0, low: float = 1.0, high: float = 32.0, device="cuda"):
    """(freqs, attention factor): f64 [dim/2], the angle by which pair i turns
    from one position to the next, base^(-2i/dim), for contexts ``factor``
    times as long as ``original``, the one it was made for, by ``scaling``:

    * ``none``; ``linear``: all frequencies divided by ``factor``;
    * ``base``: the base raised so that the slowest pair turns ``factor`` times
      slower and the fastest as before;
    * ``ramp``: pairs that turn more than ``high`` times over ``original`` keep
      their frequency, those that turn less than ``low`` times are divided by
      ``factor``, with a ramp over the pair's number between them; the attention
      factor is 0.1 ln(factor) + 1 (1 for factors up to 1);
    * ``bands``: the same with a ramp over the turns, and no attention factor."""
    if dim < 2 or dim % 2 or base <= 0 or factor <= 0:
        _fail(_q.QUICK_ERR_SHAPE, "rotary_frequencies: dim must be even and positive, base and factor positive (dim=%d)",
              dim)
    half, pi2 = dim // 2, 2 * math.pi
    if scaling == "base":
        base = base * factor ** (dim / max(dim - 2, 1))
    freqs = [base ** (-2 * i / dim) for i in range(half)]
    attention = 1.0
    if scaling == "linear":
        freqs = [f / factor for f in freqs]
    elif scaling in ("ramp", "bands"):
        if original <= 0 or not 0 < low < high:
            _fail(_q.QUICK_ERR_INVALID_ARG, "rotary_frequencies: %s needs original > 0 and 0 < low < high", scaling)
        if scaling == "ramp" and base <= 1:
            _fail(_q.QUICK_ERR_INVALID_ARG, "rotary_frequencies: a ramp needs pairs that turn slower from one to the next")

        def pair(turns):
            # number of the pair that turns so often over `original`
            return dim * math.log(original / (turns * pi2)) / (2 * math.log(base))
        out = []
        if scaling == "ramp":
            first, last = max(0, math.floor(pair(high))), min(dim - 1, math.ceil(pair(low)))
            attention = 0.1 * math.log(factor) + 1 if factor > 1 else 1.0
        for i, f in enumerate(freqs):
            if scaling == "ramp":
                keep = 1 - min(1.0, max(0.0, (i - first) / max(last - first, 0.001)))
            else:
                keep = min(1.0, max(0.0, (original * f / pi2 - low) / (high - low)))
            out.append(f * keep + f / factor * (1 - keep))
        freqs = out
    elif scaling not in ("none", "base"):
        _fail(_q.QUICK_ERR_INVALID_ARG, "rotary_frequencies: unknown scaling %s", scaling)
    return torch.tensor(freqs, dtype=torch.float64, device=device), attention


def _heads(what, name, x, types, ref=None):
    """Type code of x [T][H][D] with consecutive channels (any strides of tokens and heads)."""
    _gpu(what, name, x)
    code = _type(what, name, x.dtype, types)
    if x.dim() != 3 or (x.shape[2] > 1 and x.stride(2) != 1):
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: %s must be [T][H][D] with consecutive channels", what, name)
    if ref is not None and x.device != ref.device:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: %s must be on %s, not %s", what, name, ref.device, x.device)
    return code


def _strides(x):
    """Strides of tokens and heads; 0 where there is no second one to reach."""
    t, h, _ = x.stride()
    T, H, _ = x.shape
    return t if T > 1 else 0, h if H > 1 else 0


def rotary(x: torch.Tensor, positions: torch.Tensor, freqs: torch.Tensor, factor: float = 1.0,
           interleaved: bool = False, inverse: bool = False, out: torch.Tensor | None = None,
           stream=None) -> torch.Tensor:
    """quick_rotary: the first 2 * len(freqs) channels of x [T][H][D] (f16, bf16
    or f32; a slice of a projection's output, say) turned by positions (int32
    [T]) times freqs (f64), halves of those channels paired or, ``interleaved``,
    neighbours; ``inverse``: by the negated angle, which takes the gradient of
    the result to that of x.  ``out``: of x's shape and type, x itself among
    them."""
    what = "rotary"
    dtype = _heads(what, "x", x, _TYPES)
    T, H, D = x.shape
    _int32(what, "positions", positions, x, (T,))
    if not isinstance(freqs, torch.Tensor) or freqs.dim() != 1:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: freqs must be a float64 vector", what)
    if not _plain(freqs, x.get_device(), torch.float64):
        _q._dev(what, "freqs", freqs, x, dtype=torch.float64)
    R = 2 * freqs.shape[0]
    if R > D or D < 1 or H < 1:
        _fail(_q.QUICK_ERR_SHAPE, "%s: %d channels cannot turn in a head of %d (H=%d)", what, R, D, H)
    xs = _strides(x)
    if out is None:
        out = x.new_empty((T, H, D)) if stream is None else _new(stream, x, (T, H, D), x.dtype)
        os = H * D if T > 1 else 0, D if H > 1 else 0
    else:
        _heads(what, "out", out, {x.dtype: dtype}, x)
        if out.shape != x.shape:
            _fail(_q.QUICK_ERR_INVALID_ARG, "%s: out must have shape %s, not %s", what, tuple(x.shape), tuple(out.shape))
        os = _strides(out)
        if (T > 1 and os[0] < D) or (H > 1 and os[1] < D):
            _fail(_q.QUICK_ERR_SHAPE, "%s: rows of out overlap", what)
        if out.data_ptr() == x.data_ptr() and os != xs and x.numel():
            _fail(_q.QUICK_ERR_INVALID_ARG, "%s: out must be x with x's strides, or apart from it", what)
    _run(x, "quick_rotary", x.data_ptr(), dtype, *xs, T, H, D, positions.data_ptr(), freqs.data_ptr(), R,
         int(bool(interleaved)), int(bool(inverse)), factor, out.data_ptr(), *os, _q._stream(stream, x))
    return out


def kv4_cache(pages: int, heads: int, dim: int, device="cuda") -> torch.Tensor:
    """A zeroed cache: uint8 [pages][heads][68 * dim], pages of KV4_PAGE tokens.
    (Nothing has to be zero: kv4_attention reads no slot behind a sequence's
    length.)"""
    if dim not in KV4_DIMS:
        _fail(_q.QUICK_ERR_UNSUPPORTED, "kv4_cache: dim must be one of %s, not %s", KV4_DIMS, dim)
    return torch.zeros((pages, heads, 68 * dim), dtype=torch.uint8, device=device)


def _cache(what, cache, ref):
    """(pages, heads, D) of a cache."""
    if not (type(cache) is torch.Tensor and cache.is_cuda and cache.get_device() == ref.get_device()
            and cache.dtype is torch.uint8 and cache.is_contiguous()):
        _q._dev(what, "cache", cache, ref, dtype=torch.uint8)
    if cache.dim() != 3 or cache.shape[2] % 68 or cache.shape[2] // 68 not in KV4_DIMS:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: cache must be [pages][heads][68 * D] as kv4_cache makes it", what)
    return cache.shape[0], cache.shape[1], cache.shape[2] // 68


def kv4_write(cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, stream=None) -> torch.Tensor:
    """quick_kv4_write: token i's keys and values (k, v [T][heads][D], f16 or
    bf16; strides of tokens and heads multiples of 8) to slot slots[i] (int32
    [T]: page * KV4_PAGE + place; negative: passed over).  Returns the cache."""
    what = "kv4_write"
    dtype = _heads(what, "k", k, _TYPES16)
    _heads(what, "v", v, {k.dtype: dtype}, k)
    pages, heads, D = _cache(what, cache, k)
    T = k.shape[0]
    if k.shape != (T, heads, D) or v.shape != k.shape:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: k and v must be [T][%d][%d] for this cache", what, heads, D)
    _int32(what, "slots", slots, k, (T,))
    _run(k, "quick_kv4_write", k.data_ptr(), v.data_ptr(), dtype, *_strides(k), *_strides(v), slots.data_ptr(), T, heads,
         D, cache.data_ptr(), pages, _q._stream(stream, k))
    return cache


def kv4_read(cache: torch.Tensor, slots: torch.Tensor, dtype: torch.dtype = torch.float16,
             k: torch.Tensor | None = None, v: torch.Tensor | None = None, stream=None):
    """quick_kv4_read: (k, v) [T][heads][D] of ``dtype``, the values of slots
    (int32 [T]; zeros for one outside the cache)."""
    what = "kv4_read"
    _gpu(what, "cache", cache)
    pages, heads, D = _cache(what, cache, cache)
    code = _type(what, "dtype", dtype, _TYPES)
    if not isinstance(slots, torch.Tensor) or slots.dim() != 1:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: slots must be an int32 vector", what)
    _int32(what, "slots", slots, cache, slots.shape)
    shape = (slots.shape[0], heads, D)
    out = []
    for name, t in (("k", k), ("v", v)):
        if t is None:
            t = cache.new_empty(shape, dtype=dtype) if stream is None else _new(stream, cache, shape, dtype)
        else:
            _q._dev(what, name, t, cache, dtype=dtype, shape=shape)
        out.append(t)
    _run(cache, "quick_kv4_read", cache.data_ptr(), pages, slots.data_ptr(), shape[0], heads, D, code,
         out[0].data_ptr(), out[1].data_ptr(), _q._stream(stream, cache))
    return out[0], out[1]


@functools.lru_cache(maxsize=256)
def _attention(*fields):
    """The C struct of a call and its workspace's bytes (a small call is bound by the host)."""
    a = QuickAttention(*fields)
    return ctypes.byref(a), int(_q.lib().quick_kv4_attention_workspace_bytes(ctypes.byref(a)))


def _usual(q, cache, table, lengths, offsets):
    """Sizes (T, q_heads, pages, heads, D, seqs, width) of a call that the checks
    have nothing to say against, else None (a small call is bound by the host;
    one by one they take twice as long)."""
    if not (type(q) is type(cache) is type(table) is type(lengths) is torch.Tensor):
        return None
    dev, i32 = q.get_device(), torch.int32
    if not (dev == cache.get_device() == table.get_device() == lengths.get_device() and q.is_cuda and q.dim() == 3
            and cache.dim() == 3 and table.dim() == 2 and q.dtype in _TYPES16 and cache.dtype is torch.uint8
            and table.dtype is i32 and lengths.dtype is i32 and cache.is_contiguous() and table.is_contiguous()
            and lengths.is_contiguous() and q.stride(2) == 1):
        return None
    (T, HQ, D), (pages, heads, wide), (B, width) = q.shape, cache.shape, table.shape
    if wide != 68 * D or D not in KV4_DIMS or not heads or HQ % heads or not HQ or lengths.shape != (B,):
        return None
    if T != B if offsets is None else not (_plain(offsets, dev, i32) and offsets.shape == (B + 1,)):
        return None
    return T, HQ, pages, heads, D, B, width


def _checked(q, cache, table, lengths, offsets):
    """The same sizes, or what is wrong with the call."""
    what = "kv4_attention"
    _heads(what, "q", q, _TYPES16)
    pages, heads, D = _cache(what, cache, q)
    T, HQ, QD = q.shape
    if QD != D or HQ % heads or HQ == 0:
        _fail(_q.QUICK_ERR_SHAPE, "%s: q must be [T][a multiple of %d][%d] for this cache, not %s", what, heads, D,
              tuple(q.shape))
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        _fail(_q.QUICK_ERR_INVALID_ARG, "%s: table must be an int32 [seqs][width] tensor", what)
    B, width = table.shape
    _int32(what, "table", table, q, (B, width))
    _int32(what, "lengths", lengths, q, (B,))
    if offsets is not None:
        _int32(what, "offsets", offsets, q, (B + 1,))
    elif T != B:
        _fail(_q.QUICK_ERR_SHAPE, "%s: without offsets q has a row for each of the %d sequences, not %d", what, B, T)
    return T, HQ, pages, heads, D, B, width


def kv4_attention(q: torch.Tensor, cache: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                  offsets: torch.Tensor | None = None, most: int | None = None, scale: float | None = None,
                  window: int = 0, causal: bool = True, out: torch.Tensor | None = None,
                  lse: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """quick_kv4_attention: softmax(scale q . K^T) . V [T][q_heads][D] of q
    [T][q_heads][D] (f16 or bf16; strides of tokens and heads multiples of 8)
    over the cache, q_heads a multiple of its heads.

    table int32 [seqs][width]: pages of each sequence; lengths int32 [seqs]:
    its tokens in the cache, those of its queries among them; offsets int32
    [seqs + 1]: its queries' rows in q (None: row b is sequence b's, T = seqs),
    the last of which stands at the last token.  most: the most queries of a
    sequence (without it T is taken, and a call for a few is slower than it
    could be; rows behind it are not written).  It chooses the kernels for all:
    prompts beside many single tokens are faster as two calls (512 queries of
    one sequence beside 63 tokens of others, 32 heads on 8: 289 us as one, 127
    as two).  scale: 1 / sqrt(D) by default.
    window: a query sees its own token and the window - 1 before it.  causal:
    a query sees no token behind its own; else all of the sequence's.

    A row that sees nothing is zero; rows of no sequence are left as they
    were (in a new result: undefined).  lse: f32 [T][q_heads], filled with the
    logarithm of the softmax's sum.  workspace: a tensor of
    kv4_attention_workspace_bytes(); one is taken from torch's allocator if
    none is given."""
    what = "kv4_attention"
    sizes = _usual(q, cache, table, lengths, offsets)
    if sizes is None:
        sizes = _checked(q, cache, table, lengths, offsets)
    T, HQ, pages, heads, D, B, width = sizes
    dtype = _TYPES16[q.dtype]
    if offsets is None:
        most = 1
    elif most is None:
        most = max(1, T)
    if out is None:
        out = q.new_empty((T, HQ, D)) if stream is None else _new(stream, q, (T, HQ, D), q.dtype)
    elif not (_plain(out, q.get_device(), q.dtype) and out.shape == (T, HQ, D)):
        _q._dev(what, "out", out, q, dtype=q.dtype, shape=(T, HQ, D))
    if lse is not None:
        _q._dev(what, "lse", lse, q, dtype=torch.float32, shape=(T, HQ))
    a, need = _attention(T, HQ, heads, D, pages, B, width, most, *_strides(q), window, int(bool(causal)),
                         D ** -0.5 if scale is None else scale)
    if workspace is None:
        if need:
            if stream is None:
                workspace = q.new_empty(need, dtype=torch.uint8)
            else:
                workspace = _q._taken(stream, q, lambda: q.new_empty(need, dtype=torch.uint8), kept=False)
    else:
        _q._dev(what, "workspace", workspace, q)
        need = workspace.nbytes
    _run(q, "quick_kv4_attention", a, q.data_ptr(), dtype, cache.data_ptr(), table.data_ptr(), lengths.data_ptr(),
         offsets.data_ptr() if offsets is not None else None, out.data_ptr(), lse.data_ptr() if lse is not None else None,
         workspace.data_ptr() if workspace is not None else None, need, _q._stream(stream, q))
    return out


def kv4_attention_workspace_bytes(T: int, q_heads: int, heads: int, D: int, pages: int, seqs: int, width: int,
                                  most: int = 1, window: int = 0, causal: bool = True) -> int:
    return _attention(T, q_heads, heads, D, pages, seqs, width, most, 0, 0, window, int(bool(causal)), 1.0)[1]
