"""What is measured of the mixture-of-experts and 4-bit floating-point operators.

Kinds of case, each one pass through an operator as a serving program calls it:

* ``quant``    activations or weights to microscaled 4-bit floating point (blocks of 32 channels, E2M1 codes, one
               E8M0 scale each) and back to values;
* ``linear``   a linear layer with such weights on 16-bit activations, which the call quantises: bias or gated SiLU;
* ``grouped``  the experts' product of a mixture-of-experts layer on quantised activations, rows sorted by expert;
* ``route``    router logits to each token's experts and weights, and the expert-sorted order of the routed rows;
* ``combine``  the weighted sum of every token's expert rows.

The plain forms are elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"f16": 2, "bf16": 2, "f32": 4}


def _quant(name, m, k, dtype):
    return {"name": name, "kind": "quant", "m": m, "k": k, "dtype": dtype}


def _linear(name, m, k, n, dtype="f16", bias=False, gated=False):
    return {"name": name, "kind": "linear", "m": m, "k": k, "n": n, "dtype": dtype, "bias": bias, "gated": gated}


def _grouped(name, tokens, k, n, experts, topk, gated):
    # gated: the first product of the layer (rows gathered from the tokens, gated SiLU); else the second (rows in order)
    return {"name": name, "kind": "grouped", "tokens": tokens, "k": k, "n": n, "experts": experts, "topk": topk,
            "gated": gated}


def _route(name, tokens, experts, topk, score, groups=1, topk_groups=1, group_best=1, bias=False, renorm=True,
           dtype="f32"):
    return {"name": name, "kind": "route", "tokens": tokens, "experts": experts, "topk": topk, "score": score,
            "groups": groups, "topk_groups": topk_groups, "group_best": group_best, "bias": bias, "renorm": renorm,
            "dtype": dtype}


def _combine(name, tokens, d, topk, residual, dtype="f16"):
    return {"name": name, "kind": "combine", "tokens": tokens, "d": d, "topk": topk, "residual": residual,
            "dtype": dtype}


def listed():
    return [
        # the activations of a decode batch before a 7B model's down projection: latency counts
        _quant("quant_m16_k11008", 16, 11008, "f16"),
        # a gate+up weight matrix of a 7B model, quantised when a checkpoint is loaded
        _quant("quant_weight_22016x4096", 22016, 4096, "bf16"),
        # one user's token through a 7B model's QKV projection
        _linear("linear_m1_7b_qkv", 1, 4096, 12288),
        # an odd decode batch through a 13B model's gate+up projection, activation in the epilogue
        _linear("linear_m23_13b_gate_up", 23, 5120, 27648, gated=True),
        # a prompt of no round length, bf16, with a bias
        _linear("linear_m333_13b_down_bias", 333, 13824, 5120, dtype="bf16", bias=True),
        # prefill of a large model
        _linear("linear_m2048_70b_gate_up", 2048, 8192, 57344, gated=True),
        # decode batch of a mixture of 8 experts: a few rows an expert
        _grouped("grouped_t20_gate_up", 20, 4096, 28672, 8, 2, True),
        # prefill chunk, second product: about 512 rows an expert
        _grouped("grouped_t2048_down", 2048, 14336, 4096, 8, 2, False),
        # the router of the same layer for a decode batch
        _route("route_t20_e8", 20, 8, 2, "softmax", dtype="f16"),
        # many experts in groups, sigmoid scores and a balance bias, a prefill chunk
        _route("route_t8192_e256", 8192, 256, 8, "sigmoid", groups=8, topk_groups=4, group_best=2, bias=True),
        # joining a decode batch's rows
        _combine("combine_t20_d4096", 20, 4096, 2, True),
        # joining a prefill chunk of a layer with many experts a token
        _combine("combine_t8192_d4096_k8", 8192, 4096, 8, False, dtype="bf16"),
    ]


def _log_int(rng, lo, hi, step=1):
    while True:
        v = max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step) * step))
        if v != 3072:
            return v


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        kind = rng.choice(["quant", "linear", "linear", "grouped", "grouped", "route", "combine"])
        dtype = rng.choice(["f16", "bf16"])
        if kind == "quant":
            c = {"kind": kind, "m": _log_int(rng, 1, 16384), "k": _log_int(rng, 512, 16384, 32),
                 "dtype": rng.choice(["f16", "bf16", "f32"])}
        elif kind == "linear":
            c = {"kind": kind, "m": _log_int(rng, 1, 2048), "k": _log_int(rng, 512, 28672, 32), "dtype": dtype}
            c["gated"] = rng.random() < 0.3
            # gated: gate and up columns in tiles of 16; otherwise any number of columns
            c["n"] = _log_int(rng, 512, 57344, 32 if c["gated"] else rng.choice([1, 16]))
            c["bias"] = rng.random() < 0.3
        elif kind == "grouped":
            e = rng.choice([4, 8, 16, 40, 64])
            c = {"kind": kind, "tokens": _log_int(rng, 1, 2048), "k": _log_int(rng, 512, 14336, 32),
                 "experts": e, "topk": rng.choice([1, 2, 4]), "gated": rng.random() < 0.5}
            c["n"] = _log_int(rng, 512, 28672, 32 if c["gated"] else 16)
            if c["experts"] * c["n"] * c["k"] > 8 * 28672 * 4096:
                continue
        elif kind == "route":
            groups = rng.choice([1, 1, 4, 8])
            e = groups * _log_int(rng, 8 if groups == 1 else 4, 512 // groups)
            tg = max(1, groups // 2)
            score = rng.choice(["softmax", "sigmoid"])
            # the bias only with sigmoid scores: a softmax score's last bit depends on the order of its sum, so which
            # of two nearly equal biased scores is larger is not a property of the inputs
            bias = score == "sigmoid" and rng.random() < 0.7
            c = {"kind": kind, "tokens": _log_int(rng, 1, 16384), "experts": e,
                 "topk": rng.randint(1, min(8, e // groups * tg)), "score": score, "groups": groups,
                 "topk_groups": tg, "group_best": 2 if groups > 1 and bias else 1, "bias": bias,
                 "renorm": rng.random() < 0.7, "dtype": rng.choice(["f16", "bf16", "f32"])}
        else:
            c = {"kind": kind, "tokens": _log_int(rng, 1, 8192), "d": _log_int(rng, 256, 8192, rng.choice([1, 8])),
                 "topk": rng.randint(1, 8), "residual": rng.random() < 0.5, "dtype": dtype}
        w = work(c)
        if all(w[k] <= most[k] for k in most):
            return c


def work(case):
    kind = case["kind"]
    if kind == "quant":
        # x in; codes and scales out, and in again; values out
        n = case["m"] * case["k"]
        return {"bytes": 2 * _BYTES[case["dtype"]] * n + 2 * (n // 2 + n // 32), "flops": 0}
    if kind == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        out = n // 2 if case["gated"] else n
        return {"bytes": 2 * m * k + n * k // 2 + n * k // 32 + 2 * m * out + (2 * n if case["bias"] else 0),
                "flops": 2 * m * n * k}
    if kind == "grouped":
        r, k, n = case["tokens"] * case["topk"], case["k"], case["n"]
        # experts that are expected to have rows, each token's experts being different ones
        e = case["experts"]
        busy = e * (1 - (1 - case["topk"] / e) ** case["tokens"])
        x = case["tokens"] if case["gated"] else r
        out = n // 2 if case["gated"] else n
        return {"bytes": int((n * k // 2 + n * k // 32) * busy) + x * (k // 2 + k // 32) + 2 * r * out + 8 * r,
                "flops": 2 * r * n * k}
    if kind == "route":
        t, e, k = case["tokens"], case["experts"], case["topk"]
        return {"bytes": t * e * _BYTES[case["dtype"]] + t * k * 16 + 4 * (e + 1), "flops": 4 * t * e}
    t, d, k = case["tokens"], case["d"], case["topk"]
    return {"bytes": 2 * t * d * (k + 1 + case["residual"]) + 8 * t * k, "flops": 2 * t * d * k}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _normal(g, *shape, scale=1.0, dtype=torch.float16):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _activations(g, m, k, dtype):
    # standard normal with one channel in a hundred 20 times larger, as activations of language models are
    x = torch.randn(m, k, generator=g, device="cuda")
    outlier = torch.rand(k, generator=g, device="cuda") < 0.01
    return torch.where(outlier, x * 20, x).to(dtype)


def _weights(g, n, k):
    """Codes and scales of an n x k matrix of normal weights."""
    codes = torch.empty(n, k // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(n, k // 32, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // k)
    for i in range(0, n, step):
        codes[i:i + step], scales[i:i + step] = _quantized(_normal(g, min(step, n - i), k, scale=0.02).float())
    return codes, scales


def _routing(g, tokens, experts, topk):
    """Offsets of the experts and the token of each routed row, each token at topk different experts."""
    expert = torch.rand(tokens, experts, generator=g, device="cuda").topk(topk, dim=1).indices.reshape(-1)
    order = torch.argsort(expert, stable=True)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.bincount(expert, minlength=experts).cumsum(0)
    return offsets, (order // topk).to(torch.int32), order


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, dtype = case["kind"], _DTYPES[case.get("dtype", "f16")]
    if kind == "quant":
        return {"x": _activations(g, case["m"], case["k"], dtype)}
    if kind == "linear":
        w = _weights(g, case["n"], case["k"])
        return {"x": _activations(g, case["m"], case["k"], dtype), "w": w,
                "bias": _normal(g, case["n"], dtype=dtype) if case["bias"] else None}
    if kind == "grouped":
        e, k, n = case["experts"], case["k"], case["n"]
        offsets, rows, _ = _routing(g, case["tokens"], e, case["topk"])
        codes, scales = _weights(g, e * n, k)
        x = _activations(g, case["tokens"] if case["gated"] else rows.numel(), k, torch.float16)
        return {"x": _quantized(x.float()), "w": (codes.view(e, n, k // 2), scales.view(e, n, k // 32)),
                "offsets": offsets, "rows": rows if case["gated"] else None,
                # the most rows of an expert, which a program that plans its batches knows
                "most": int((offsets[1:] - offsets[:-1]).max())}
    if kind == "route":
        return {"logits": _normal(g, case["tokens"], case["experts"], scale=1.5, dtype=dtype),
                "bias": torch.rand(case["experts"], generator=g, device="cuda") * 0.2 - 0.1 if case["bias"] else None}
    t, d, k = case["tokens"], case["d"], case["topk"]
    weights = torch.rand(t, k, generator=g, device="cuda") + 0.1
    return {"y": _normal(g, t * k, d, dtype=dtype),
            "slots": torch.randperm(t * k, generator=g, device="cuda").to(torch.int32).view(t, k),
            "weights": weights / weights.sum(1, keepdim=True),
            "residual": _normal(g, t, d, dtype=dtype) if case["residual"] else None}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own and "w" in s:
        # a serving program lays its weights out once, when it loads them, and keeps that form alone
        import paper_2402_10076_amd as Q
        s["packed"] = Q.mxfp4_pack(*s.pop("w"), gate_up=case["gated"])
    return s


# ---------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------

def _run_own(s):
    import paper_2402_10076_amd as Q
    case = s["case"]
    kind = case["kind"]
    if kind == "quant":
        return Q.mxfp4_dequantize(*Q.mxfp4_quantize(s["x"]), dtype=s["x"].dtype)
    if kind == "linear":
        return Q.mxfp4_linear(s["x"], *s["packed"], case["n"], bias=s["bias"],
                              activation=Q.ACT_SILU_GATE if case["gated"] else Q.ACT_NONE)
    if kind == "grouped":
        return Q.mxfp4_grouped_gemm(*s["x"], s["offsets"], *s["packed"], case["n"], rows=s["rows"],
                                    activation=Q.ACT_SILU_GATE if case["gated"] else Q.ACT_NONE)
    if kind == "route":
        r = Q.moe_route(s["logits"], case["topk"],
                        score=Q.SCORE_SIGMOID if case["score"] == "sigmoid" else Q.SCORE_SOFTMAX, bias=s["bias"],
                        groups=case["groups"], topk_groups=case["topk_groups"], group_best=case["group_best"],
                        renormalize=case["renorm"])
        return [r.ids, r.weights, r.offsets, r.rows, r.slots]
    return Q.moe_combine(s["y"], s["slots"], s["weights"], residual=s["residual"])


# ---------------------------------------------------------------------------
# their plain forms
# ---------------------------------------------------------------------------

def _power(n):
    """2^n in binary32, -127 <= n <= 127, from its bits."""
    return torch.where(n > -127, (n + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _quantized(x):
    """Codes [m][k/2] and scales [m][k/32] of binary32 values [m][k]."""
    m, k = x.shape
    b = x.view(m, k // 32, 32)
    # the exponent of the largest magnitude, less that of the largest code (4 <= 6 < 8)
    scale = ((b.abs().amax(2).view(torch.int32) >> 23) - 2).clamp_(min=0)
    v = b * _power(127 - scale.unsqueeze(2))
    a = v.abs()
    # ties go to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    code = (code | (v < 0).to(torch.uint8) * 8).view(m, k // 2, 2)
    return code[:, :, 0] | code[:, :, 1] << 4, scale.to(torch.uint8)


_pairs = {}


def _values(codes, scales):
    """Binary32 values of codes [..., k/2] and scales [..., k/32]."""
    at = codes.device
    if at not in _pairs:
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=at)
        byte = torch.arange(256, device=at)
        _pairs[at] = torch.stack([grid[byte & 15], grid[byte >> 4]], 1)
    v = _pairs[at][codes.to(torch.int32)].view(*scales.shape, 32)
    return (v * _power(scales.to(torch.int32) - 127).unsqueeze(-1)).flatten(-2)


def _epilogue(h, bias, gated):
    if bias is not None:
        h = h + bias.float()
    if gated:
        gate, up = h.chunk(2, dim=-1)
        h = gate / (1 + torch.exp(-gate)) * up
    return h


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "quant":
        return _values(*_quantized(s["x"].float())).to(s["x"].dtype)
    if kind == "linear":
        x = _values(*_quantized(s["x"].float()))
        return _epilogue(x @ _values(*s["w"]).t(), s["bias"], case["gated"]).to(s["x"].dtype)
    if kind == "grouped":
        # each expert's rows side by side, as many places as the fullest has
        x = _values(*s["x"])
        if s["rows"] is not None:
            x = x[s["rows"]]
        first, last = s["offsets"][:-1], s["offsets"][1:]
        r = torch.arange(x.shape[0], device=x.device, dtype=torch.int32)
        expert = (r.unsqueeze(1) >= last).sum(1)
        place = r - first[expert]
        wide = x.new_zeros(case["experts"], s["most"], case["k"])
        wide[expert, place] = x
        h = torch.bmm(wide, _values(*s["w"]).transpose(1, 2))
        return _epilogue(h[expert, place], None, case["gated"]).to(torch.float16)
    if kind == "route":
        return _route_plain(s["logits"].float(), s["bias"], case)
    y = s["y"][s["slots"]].float()
    out = (y * s["weights"].unsqueeze(2)).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return out.to(s["y"].dtype)


def _route_plain(x, bias, case):
    t, e = x.shape
    k, groups = case["topk"], case["groups"]
    if case["score"] == "sigmoid":
        score = 1 / (1 + torch.exp(-x))
        choice = score if bias is None else score + bias
    else:
        ex = torch.exp(x - x.amax(1, keepdim=True))
        score = ex / ex.sum(1, keepdim=True)
        choice = x      # softmax keeps the order of a row
    if groups > 1:
        best = choice.view(t, groups, -1).sort(dim=2, descending=True).values[:, :, :case["group_best"]].sum(2)
        chosen = best.sort(dim=1, descending=True, stable=True).indices[:, :case["topk_groups"]]
        keep = torch.zeros(t, groups, dtype=torch.bool, device=x.device).scatter_(1, chosen, True)
        choice = choice.masked_fill(~keep.repeat_interleave(e // groups, 1), -math.inf)
    ids = choice.sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = score.gather(1, ids)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True)
    flat = ids.reshape(-1)
    order = torch.argsort(flat, stable=True)
    offsets = torch.zeros(e + 1, dtype=torch.int32, device=x.device)
    offsets[1:] = (flat.unsqueeze(0) == torch.arange(e, device=x.device).unsqueeze(1)).sum(1).cumsum(0)
    slots = torch.empty(t * k, dtype=torch.int32, device=x.device)
    slots[order] = torch.arange(t * k, dtype=torch.int32, device=x.device)
    return [ids.to(torch.int32), w, offsets, (order // k).to(torch.int32), slots.view(t, k)]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def _exact_rounded(x):
    """Values that a binary64 matrix [m][k] has in the microscaled format."""
    m, k = x.shape
    b = x.reshape(m, k // 32, 32)
    top = torch.frexp(b.abs().amax(2, keepdim=True))
    # amax = mantissa * 2^exponent with mantissa in [0.5, 1): its floor(log2) is exponent - 1
    unit = torch.where(top.mantissa > 0, top.exponent - 3, torch.full_like(top.exponent, -127)).clamp(min=-127)
    unit = torch.pow(2.0, unit.double())
    v = b / unit
    step = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0)).double()
    return ((v / step).round() * step).clamp(-6, 6).mul(unit).reshape(m, k)


def _exact_values(codes, scales):
    low, high = (codes & 15).double(), (codes >> 4).double()
    c = torch.stack([low, high], -1).flatten(-2)
    sign = torch.where(c >= 8, -1.0, 1.0).double()
    c = torch.where(c >= 8, c - 8, c)
    exponent = torch.div(c, 2, rounding_mode="floor")
    mantissa = c - 2 * exponent
    mag = torch.where(exponent == 0, mantissa / 2, (1 + mantissa / 2) * torch.pow(2.0, exponent - 1))
    unit = torch.pow(2.0, scales.double() - 127).repeat_interleave(32, -1)
    return sign * mag * unit


def _exact_epilogue(h, bias, gated):
    h = h if bias is None else h + bias.double()
    if not gated:
        return h
    n = h.shape[1] // 2
    return torch.nn.functional.silu(h[:, :n]) * h[:, n:]


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "quant":
        return _exact_rounded(s["x"].double())
    if kind == "linear":
        x = _exact_rounded(s["x"].double())
        return _exact_epilogue(x @ _exact_values(*s["w"]).t(), s["bias"], case["gated"])
    if kind == "grouped":
        x = _exact_values(*s["x"])
        at = s["offsets"].tolist()
        out = []
        for e in range(case["experts"]):
            rows = slice(at[e], at[e + 1])
            xe = x[rows] if s["rows"] is None else x[s["rows"][rows].long()]
            w = _exact_values(s["w"][0][e], s["w"][1][e])
            out.append(_exact_epilogue(xe @ w.t(), None, case["gated"]))
        return torch.cat(out)
    if kind == "route":
        x = s["logits"].double()
        score = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(x, 1)
        choice = score if s["bias"] is None else score + s["bias"].double()
        if case["groups"] > 1:
            g = choice.view(case["tokens"], case["groups"], -1)
            best = g.sort(dim=2, descending=True).values[:, :, :case["group_best"]].sum(2)
            rank = best.sort(dim=1, descending=True, stable=True).indices.argsort(dim=1)
            choice = torch.where((rank < case["topk_groups"]).unsqueeze(2), g, -1e9).reshape(choice.shape)
        w = score.gather(1, choice.sort(dim=1, descending=True, stable=True).indices[:, :case["topk"]])
        return [None, w / w.sum(1, keepdim=True) if case["renorm"] else w, None, None, None]
    out = torch.zeros(case["tokens"], case["d"], dtype=torch.float64, device="cuda")
    for j in range(case["topk"]):
        out += s["y"][s["slots"][:, j].long()].double() * s["weights"][:, j:j + 1].double()
    return out if s["residual"] is None else out + s["residual"].double()
