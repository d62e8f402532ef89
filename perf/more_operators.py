"""What is measured of an attention layer's operators around the 4-bit products.

Kinds of case, each one pass through an operator as a serving program calls it:

* ``rotary``     rotary positions of the query and key heads of a projection's output;
* ``cache``      keys and values to the paged 4-bit cache (blocks of 32 channels, E2M1 codes, one E8M0 scale each) and
                 back to values;
* ``attention``  queries over the paged 4-bit cache of their sequences: single tokens, a few drafted ones, or prompts;
* ``lora``       the low-rank adapters of many requests, each token with its own or none, added to the output of the
                 projection that all share.

The plain forms are elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 64       # tokens of a cache page

_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"f16": 2, "bf16": 2, "f32": 4}


def _rotary(name, tokens, heads, dim, part, far, dtype="f16", interleaved=False, factor=1.0):
    # part: channels of a head that turn; far: positions are below it; factor: that many times longer contexts than
    # the frequencies were made for
    return {"name": name, "kind": "rotary", "tokens": tokens, "heads": heads, "dim": dim, "part": part, "far": far,
            "dtype": dtype, "interleaved": interleaved, "factor": factor}


def _cache(name, tokens, heads, dim, dtype="f16"):
    return {"name": name, "kind": "cache", "tokens": tokens, "heads": heads, "dim": dim, "dtype": dtype}


def _attention(name, seqs, heads, group, dim, least, most, new=1, new_most=1, dtype="f16", causal=True, window=0):
    # heads: of keys and values, each read by `group` query heads; least, most: tokens of a sequence in the cache, the
    # new ones among them; new, new_most: fewest and most new tokens (queries) of a sequence
    return {"name": name, "kind": "attention", "seqs": seqs, "heads": heads, "group": group, "dim": dim,
            "least": least, "most": most, "new": new, "new_most": new_most, "dtype": dtype, "causal": causal,
            "window": window}


def _lora(name, tokens, k, n, adapters, rank, dtype="f16", bare=0):
    # bare: of 8 tokens so many have no adapter
    return {"name": name, "kind": "lora", "tokens": tokens, "k": k, "n": n, "adapters": adapters, "rank": rank,
            "dtype": dtype, "bare": bare}


def listed():
    return [
        # one user's token in a 7B model, queries and keys at once: latency counts
        _rotary("rotary_t1_7b", 1, 64, 128, 128, 4096),
        # a prompt in a 70B model, half of each head turning, pairs side by side, stretched to long contexts
        _rotary("rotary_t8192_70b_part", 8192, 72, 128, 64, 131072, dtype="bf16", interleaved=True, factor=8.0),
        # the new tokens of a decode batch in a 70B model
        _cache("cache_t20_70b", 20, 8, 128),
        # a prompt of a 7B model, one key and value head a query head
        _cache("cache_t8192_7b", 8192, 32, 128, dtype="bf16"),
        # one user's token after a thousand others, 4 query heads for each of 8 key and value heads
        _attention("decode_s1_l1000", 1, 8, 4, 128, 1000, 1000),
        # an ordinary decode batch of a 7B model, lengths as they come
        _attention("decode_s32_7b", 32, 32, 1, 128, 37, 4096, dtype="bf16"),
        # a decode batch of a 70B model at long contexts: what a 4-bit cache is for
        _attention("decode_s64_70b_long", 64, 8, 8, 128, 512, 32768),
        # five drafted tokens of each of 8 sequences, looked over at once
        _attention("verify_s8_q5", 8, 8, 4, 128, 2000, 9000, new=5, new_most=5, dtype="bf16"),
        # chunks of prompts beside single tokens, small heads, a sliding window
        _attention("mixed_s16_window", 16, 8, 4, 64, 600, 5000, new=1, new_most=501, window=1024),
        # a whole prompt of a 70B model
        _attention("prompt_t8192_70b", 1, 8, 8, 128, 8192, 8192, new=8192, new_most=8192, dtype="bf16"),
        # a decode batch, three tokens to an adapter and three without one, at a 7B model's QKV projection
        _lora("lora_t27_7b_qkv", 27, 4096, 12288, 8, 16, bare=1),
        # prompts of four requests at a 13B model's QKV projection
        _lora("lora_t4096_13b_qkv", 4096, 5120, 15360, 4, 64, dtype="bf16"),
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step) * step))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        kind = rng.choice(["rotary", "cache", "attention", "attention", "attention", "lora", "lora"])
        dtype = rng.choice(["f16", "bf16"])
        if kind == "rotary":
            dim = rng.choice([64, 80, 96, 128, 256])
            c = {"kind": kind, "tokens": _log_int(rng, 1, 16384), "heads": _log_int(rng, 1, 128), "dim": dim,
                 "part": rng.choice([dim, dim // 2, dim // 4]), "far": rng.choice([4096, 32768, 1048576]),
                 "dtype": rng.choice(["f16", "bf16", "f32"]), "interleaved": rng.random() < 0.5,
                 "factor": rng.choice([1.0, 1.0, 4.0, 32.0])}
        elif kind == "cache":
            c = {"kind": kind, "tokens": _log_int(rng, 1, 16384), "heads": rng.choice([1, 2, 4, 5, 8, 32, 40]),
                 "dim": rng.choice([64, 128, 128, 256]), "dtype": dtype}
        elif kind == "attention":
            c = {"kind": kind, "seqs": _log_int(rng, 1, 128), "heads": rng.choice([1, 2, 4, 8, 8, 32]),
                 "group": rng.choice([1, 2, 4, 5, 8, 16]), "dim": rng.choice([64, 128, 128, 256]),
                 "most": _log_int(rng, 1, 32768), "dtype": dtype, "causal": rng.random() < 0.8, "window": 0}
            c["least"] = rng.randint(1, c["most"])
            form = rng.choice(["one", "one", "few", "chunks"])
            c["new"] = c["new_most"] = 1
            if form == "few":
                c["new"] = c["new_most"] = min(c["least"], rng.randint(2, 8))
            elif form == "chunks":
                c["new_most"] = _log_int(rng, 1, min(c["least"], 2048))
                c["new"] = rng.randint(1, c["new_most"])
            if c["causal"] and rng.random() < 0.3:
                c["window"] = _log_int(rng, 16, 4096)
            # the plain form holds every score and all keys and values of the longest sequence, for each sequence
            if (c["seqs"] * c["heads"] * c["most"] * max(c["group"] * c["new_most"], 2 * c["dim"])) > 1 << 32:
                continue
        else:
            c = {"kind": kind, "tokens": _log_int(rng, 1, 4096), "k": _log_int(rng, 512, 14336, 8),
                 "n": _log_int(rng, 512, 28672, 8), "adapters": _log_int(rng, 1, 64),
                 "rank": rng.choice([8, 16, 16, 32, 64, 128]), "dtype": dtype, "bare": rng.choice([0, 0, 1, 4])}
        w = work(c)
        if all(w[k] <= most[k] for k in most):
            return c


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly apart."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]


def _sequences(case):
    """(tokens in the cache, new tokens) of each sequence, up to their order: the longest has the fewest new ones."""
    return list(zip(_spread(case["least"], case["most"], case["seqs"]),
                    reversed(_spread(case["new"], case["new_most"], case["seqs"]))))


def _seen(case, length, new):
    """Pairs of a query and a token that it sees, and tokens that some query sees, of one sequence."""
    if not case["causal"]:
        return length * new, length
    first = length - new
    if not case["window"]:
        return new * (first + 1 + length) // 2, length
    w = case["window"]
    return sum(min(w, p + 1) for p in range(first, length)), min(length, new + w - 1)


def work(case):
    kind = case["kind"]
    if kind == "rotary":
        t, h, d = case["tokens"], case["heads"], case["dim"]
        return {"bytes": 2 * _BYTES[case["dtype"]] * t * h * d + 4 * t, "flops": 3 * t * h * case["part"]}
    if kind == "cache":
        # keys and values in; codes and scales out, and in again; values out
        n = 2 * case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * 2 * n + 2 * (n // 2 + n // 32) + 2 * 4 * case["tokens"], "flops": 0}
    if kind == "attention":
        d, hk = case["dim"], case["heads"]
        hq = hk * case["group"]
        seqs = _sequences(case)
        pairs = sum(_seen(case, *s)[0] for s in seqs)
        tokens = sum(_seen(case, *s)[1] for s in seqs)
        return {"bytes": 2 * tokens * hk * (d // 2 + d // 32) + 2 * 2 * sum(n for _, n in seqs) * hq * d,
                "flops": 4 * d * hq * pairs}
    t, k, n, r = case["tokens"], case["k"], case["n"], case["rank"]
    with_one = t - t * case["bare"] // 8
    busy = min(case["adapters"], with_one)
    return {"bytes": 2 * (with_one * k + busy * r * (k + n) + 2 * t * n), "flops": 2 * with_one * r * (k + n)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _normal(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _frequencies(case):
    """Angle by which a pair turns from one position to the next, in 64 bits on the host: bands that turn often over the
    context that they were made for keep it, slow ones are stretched, those between are mixed."""
    half = case["part"] // 2
    out = []
    for i in range(half):
        f = 10000.0 ** (-i / half)
        turns = 4096 * f / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1) / 31))
        out.append(f * keep + f / case["factor"] * (1 - keep))
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _keys_values(g, *shape, dtype):
    """Normal keys with one channel in sixteen six times larger, as keys of language models have them, and values."""
    k = torch.randn(*shape, generator=g, device="cuda")
    big = torch.rand(*shape[-2:], generator=g, device="cuda") < 0.0625
    return torch.where(big, k * 6, k).to(dtype), _normal(g, *shape, dtype=dtype)


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, dtype = case["kind"], _DTYPES[case["dtype"]]
    if kind == "rotary":
        t, h, d = case["tokens"], case["heads"], case["dim"]
        return {"x": _normal(g, t, h, d, dtype=dtype), "freqs": _frequencies(case),
                "positions": torch.randint(0, case["far"], (t,), generator=g, device="cuda", dtype=torch.int32)}
    if kind == "cache":
        t, h, d = case["tokens"], case["heads"], case["dim"]
        k, v = _keys_values(g, t, h, d, dtype=dtype)
        pages = -(-t // PAGE) + 3
        slots = torch.randperm(pages * PAGE, generator=g, device="cuda")[:t].to(torch.int32)
        return {"k": k, "v": v, "slots": slots, "pages": pages}
    if kind == "attention":
        h, d, b = case["heads"], case["dim"], case["seqs"]
        seqs = _sequences(case)
        order = torch.randperm(b, generator=g, device="cuda").tolist()
        lengths, new = [seqs[i][0] for i in order], [seqs[i][1] for i in order]
        need = [-(-n // PAGE) for n in lengths]
        pages = sum(need) + 1
        ids = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros(b, max(need), dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = ids[at:at + n]
            at += n
        slots = pages * PAGE
        cache = [torch.empty(slots, h, w, dtype=torch.uint8, device="cuda") for w in (d // 2, d // 32, d // 2, d // 32)]
        step = max(1, (1 << 26) // (h * d))
        for i in range(0, slots, step):
            k, v = _keys_values(g, min(step, slots - i), h, d, dtype=dtype)
            cache[0][i:i + step], cache[1][i:i + step] = _quantized(k.float())
            cache[2][i:i + step], cache[3][i:i + step] = _quantized(v.float())
        first = [0]
        for n in new:
            first.append(first[-1] + n)
        return {"q": _normal(g, first[-1], h * case["group"], d, scale=1.5, dtype=dtype), "cache": cache,
                "table": table, "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                "offsets": torch.tensor(first, dtype=torch.int32, device="cuda")}
    t, k, n, e, r = case["tokens"], case["k"], case["n"], case["adapters"], case["rank"]
    bare = t * case["bare"] // 8
    ids = torch.arange(t, device="cuda") * e // max(1, t - bare)
    ids = torch.where(ids < e, ids, -1)[torch.randperm(t, generator=g, device="cuda")]
    return {"x": _normal(g, t, k, dtype=dtype), "y": _normal(g, t, n, dtype=dtype), "ids": ids.to(torch.int32),
            "a": _normal(g, e, r, k, scale=k ** -0.5, dtype=dtype),
            "b": _normal(g, e, n, r, scale=0.5 * r ** -0.5, dtype=dtype),
            "scales": torch.rand(e, generator=g, device="cuda") + 0.5}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2402_10076_amd as Q
        if case["kind"] == "cache":
            s["cache"] = Q.kv4_cache(s["pages"], case["heads"], case["dim"])
        elif case["kind"] == "attention":
            # what earlier steps of the program have written
            kc, ks, vc, vs = s.pop("cache")
            cache = Q.kv4_cache(kc.shape[0] // PAGE, case["heads"], case["dim"])
            step = max(1, (1 << 26) // (case["heads"] * case["dim"]))
            for i in range(0, kc.shape[0], step):
                at = slice(i, i + step)
                k, v = (_values(c[at], x[at]).to(s["q"].dtype) for c, x in ((kc, ks), (vc, vs)))
                Q.kv4_write(cache, k, v, torch.arange(i, i + k.shape[0], dtype=torch.int32, device="cuda"))
            s["cache"] = cache
            # a program that plans its batches knows the most new tokens of a sequence; single tokens need no offsets
            if case["new_most"] == 1:
                s["offsets"] = None
        elif case["kind"] == "lora":
            # the tokens' order by adapter is the same for every projection of a step
            s["offsets"], s["rows"] = Q.lora_group(s["ids"], case["adapters"])
    return s


# ---------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------

def _run_own(s):
    import paper_2402_10076_amd as Q
    case = s["case"]
    kind = case["kind"]
    if kind == "rotary":
        return Q.rotary(s["x"], s["positions"], s["freqs"], interleaved=case["interleaved"])
    if kind == "cache":
        Q.kv4_write(s["cache"], s["k"], s["v"], s["slots"])
        return Q.kv4_read(s["cache"], s["slots"], dtype=s["k"].dtype)
    if kind == "attention":
        return Q.kv4_attention(s["q"], s["cache"], s["table"], s["lengths"], offsets=s["offsets"],
                               most=case["new_most"], causal=case["causal"], window=case["window"])
    return Q.lora_add(s["y"], s["x"], s["a"], s["b"], s["offsets"], s["rows"], scales=s["scales"])


# ---------------------------------------------------------------------------
# their plain forms
# ---------------------------------------------------------------------------

def _power(n):
    """2^n in binary32, -127 <= n <= 127, from its bits."""
    return torch.where(n > -127, (n + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _quantized(x):
    """Codes [..., d/2] and scales [..., d/32] of binary32 values [..., d]."""
    b = x.unflatten(-1, (-1, 32))
    # the exponent of the largest magnitude, less that of the largest code (4 <= 6 < 8)
    scale = ((b.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp_(min=0)
    v = b * _power(127 - scale.unsqueeze(-1))
    a = v.abs()
    # ties go to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    code = (code | (v < 0).to(torch.uint8) * 8).flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] | code[..., 1] << 4, scale.to(torch.uint8)


_pairs = {}


def _values(codes, scales):
    """Binary32 values [..., d] of codes [..., d/2] and scales [..., d/32]."""
    at = codes.device
    if at not in _pairs:
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=at)
        byte = torch.arange(256, device=at)
        _pairs[at] = torch.stack([grid[byte & 15], grid[byte >> 4]], 1)
    v = _pairs[at][codes.to(torch.int32)].view(*scales.shape, 32)
    return (v * _power(scales.to(torch.int32) - 127).unsqueeze(-1)).flatten(-2)


def _attention_plain(s):
    case = s["case"]
    b, h, g, d = case["seqs"], case["heads"], case["group"], case["dim"]
    lengths, offsets, q = s["lengths"], s["offsets"], s["q"]
    tokens = torch.arange(case["most"], device=q.device)
    slots = s["table"][:, tokens // PAGE] * PAGE + tokens % PAGE
    kc, ks, vc, vs = s["cache"]
    k = _values(kc[slots], ks[slots]).permute(0, 2, 3, 1).contiguous()       # b, h, d, tokens
    v = _values(vc[slots], vs[slots]).permute(0, 2, 1, 3).contiguous()       # b, h, tokens, d
    # each sequence's queries side by side, as many places as the one with most has
    row = torch.arange(q.shape[0], device=q.device)
    seq = (row.unsqueeze(1) >= offsets[1:]).sum(1)
    place = row - offsets[seq]
    wide = torch.zeros(b, case["new_most"], h, g, d, device=q.device)
    wide[seq, place] = q.float().view(-1, h, g, d)
    score = torch.matmul(wide.permute(0, 2, 1, 3, 4).reshape(b, h, -1, d), k) * d ** -0.5
    score = score.view(b, h, case["new_most"], g, -1)
    at = tokens.view(1, 1, 1, 1, -1)
    hidden = at >= lengths.view(-1, 1, 1, 1, 1)
    if case["causal"]:
        pos = lengths.unsqueeze(1) - (offsets[1:] - offsets[:-1]).unsqueeze(1) + torch.arange(case["new_most"], device=q.device)
        pos = pos.view(b, 1, -1, 1, 1)
        hidden = hidden | (at > pos)
        if case["window"]:
            hidden = hidden | (at <= pos - case["window"])
    score = score.masked_fill(hidden, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0))
    total = p.sum(-1)
    out = torch.matmul(p.view(b, h, -1, case["most"]), v).view(b, h, -1, g, d)
    out = out / torch.where(total > 0, total, 1).unsqueeze(-1)
    return out.permute(0, 2, 1, 3, 4)[seq, place].reshape(-1, h * g, d).to(q.dtype)


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "rotary":
        x, r = s["x"].float(), case["part"]
        # 64 bits: 32 lose the angles of far positions
        angle = s["positions"].double().unsqueeze(1) * s["freqs"]
        c, n = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
        if case["interleaved"]:
            p, q = x[..., 0:r:2], x[..., 1:r:2]
            turned = torch.stack([p * c - q * n, q * c + p * n], -1).flatten(-2)
        else:
            p, q = x[..., :r // 2], x[..., r // 2:r]
            turned = torch.cat([p * c - q * n, q * c + p * n], -1)
        return torch.cat([turned, x[..., r:]], -1).to(s["x"].dtype)
    if kind == "cache":
        return [_values(*_quantized(s[n].float())).to(s[n].dtype) for n in ("k", "v")]
    if kind == "attention":
        return _attention_plain(s)
    # each adapter's tokens side by side, as many places as the one with most has
    x, ids, e = s["x"].float(), s["ids"].long(), case["adapters"]
    to = torch.where(ids >= 0, ids, e)
    order = torch.argsort(to, stable=True)
    first = (to.unsqueeze(0) < torch.arange(e + 1, device=x.device).unsqueeze(1)).sum(1)
    place = torch.empty_like(to)
    place[order] = torch.arange(x.shape[0], device=x.device) - first[to[order]]
    wide = x.new_zeros(e + 1, _most(case), x.shape[1])
    keep = ids >= 0
    spot = torch.where(keep, place, 0)
    wide[to, spot] = torch.where(keep.unsqueeze(1), x, 0)
    low = torch.bmm(wide[:e], s["a"].float().transpose(1, 2).contiguous()) * s["scales"].view(-1, 1, 1)
    high = torch.bmm(low, s["b"].float().transpose(1, 2).contiguous())
    add = torch.where(keep.unsqueeze(1), high[torch.where(keep, ids, 0), spot], 0)
    return (s["y"].float() + add).to(s["y"].dtype)


def _most(case):
    """Most tokens that an adapter can have: as _inputs spreads them."""
    t, e = case["tokens"], case["adapters"]
    return -(-(t - t * case["bare"] // 8) // e)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def _exact_rounded(x):
    """Values that binary64 numbers [..., d] have in the microscaled format."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = torch.frexp(b.abs().amax(-1, keepdim=True))
    # amax = mantissa * 2^exponent with mantissa in [0.5, 1): its floor(log2) is exponent - 1
    unit = torch.where(top.mantissa > 0, top.exponent - 3, torch.full_like(top.exponent, -127)).clamp(min=-127)
    unit = torch.pow(2.0, unit.double())
    v = b / unit
    step = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0)).double()
    return ((v / step).round() * step).clamp(-6, 6).mul(unit).reshape(x.shape)


def _exact_values(codes, scales):
    c = torch.stack([(codes & 15).double(), (codes >> 4).double()], -1).flatten(-2)
    sign = torch.where(c >= 8, -1.0, 1.0).double()
    c = torch.where(c >= 8, c - 8, c)
    exponent = torch.div(c, 2, rounding_mode="floor")
    mantissa = c - 2 * exponent
    mag = torch.where(exponent == 0, mantissa / 2, (1 + mantissa / 2) * torch.pow(2.0, exponent - 1))
    return sign * mag * torch.pow(2.0, scales.double() - 127).repeat_interleave(32, -1)


def _exact_attention(case, s):
    g, d = case["group"], case["dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lengths, offsets = s["lengths"].tolist(), s["offsets"].tolist()
    for i, n in enumerate(lengths):
        slots = (s["table"][i].long().unsqueeze(1) * PAGE + torch.arange(PAGE, device="cuda")).flatten()[:n]
        kc, ks, vc, vs = (c[slots] for c in s["cache"])
        rows = slice(offsets[i], offsets[i + 1])
        new = offsets[i + 1] - offsets[i]
        q = s["q"][rows].double()
        pos = torch.arange(n - new, n, device="cuda").unsqueeze(1)
        at = torch.arange(n, device="cuda").unsqueeze(0)
        seen = torch.ones(new, n, dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen = at <= pos
            if case["window"]:
                seen &= at > pos - case["window"]
        for h in range(case["heads"]):
            k, v = _exact_values(kc[:, h], ks[:, h]), _exact_values(vc[:, h], vs[:, h])
            # query heads together as far as their scores stay small
            step = max(1, (1 << 27) // max(1, new * n))
            for j in range(h * g, h * g + g, step):
                heads = slice(j, min(j + step, h * g + g))
                score = q[:, heads].transpose(0, 1) @ k.t() / math.sqrt(d)
                p = torch.softmax(score.masked_fill(~seen, -math.inf), 2)
                out[rows, heads] = (p @ v).transpose(0, 1)
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        x, r = s["x"].double(), case["part"]
        angle = s["positions"].double().view(-1, 1, 1) * s["freqs"]
        turn = torch.polar(torch.ones_like(angle), angle)
        pairs = x[..., :r].unflatten(-1, (-1, 2)) if case["interleaved"] else x[..., :r].unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        x[..., :r] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        return x
    if kind == "cache":
        return [_exact_rounded(s[n].double()) for n in ("k", "v")]
    if kind == "attention":
        return _exact_attention(case, s)
    out = s["y"].double()
    for e in range(case["adapters"]):
        rows = (s["ids"] == e).nonzero().squeeze(1)
        low = s["x"][rows].double() @ s["a"][e].double().t()
        out[rows] += float(s["scales"][e]) * (low @ s["b"][e].double().t())
    return out
