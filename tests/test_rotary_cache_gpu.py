"""Rotary positions and the paged 4-bit cache (include/quick_attention.h) on
the GPU against binary64 forms."""
import numpy as np
import pytest
import torch

import attn_util as A
import mx_util as U
import paper_2402_10076_amd as Q
from gpu_util import say

pytestmark = pytest.mark.gpu


def _freqs(half):
    return Q.rotary_frequencies(2 * half, device="cpu")[0] if half else torch.zeros(0, dtype=torch.float64)


def _check_rotary(y, x, pos, freqs, **kw):
    ref, size = A.rotated(x.double(), pos, freqs, **kw)
    step = A.STEP[x.dtype]
    err = (y.cpu().double() - ref).abs()
    tiny = 2.0 ** -25 if x.dtype == torch.float16 else 1e-37
    assert bool((err <= ref.abs() * step * (1 + step) + size * (1 + step) + tiny).all()), float(err.max())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,H,D,R", [(1, 1, 2, 2), (1, 64, 128, 128), (3, 5, 128, 64), (7, 3, 96, 32), (17, 40, 80, 80),
                                     (2, 2, 64, 6), (5, 3, 50, 34), (300, 9, 256, 128), (33, 1, 4096, 4096),
                                     (4, 2, 1000, 16), (2, 3, 64, 0), (600, 72, 64, 64)])
def test_rotary(T, H, D, R, dtype, interleaved):
    g = A.gen(1, T, H, D, R)
    x = A.normal(g, T, H, D, dtype=A.TYPES[dtype])
    pos = torch.randint(0, 1 << 20, (T,), generator=g, dtype=torch.int32)
    freqs = _freqs(R // 2)
    say("rotary", T, H, D, R, dtype, interleaved)
    for kw in ({}, {"factor": 1.25, "inverse": True}):
        y = Q.rotary(x.cuda(), pos.cuda(), freqs.cuda(), interleaved=interleaved, **kw)
        _check_rotary(y, x, pos, freqs, interleaved=interleaved, **kw)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_strides_and_in_place(interleaved):
    """Query and key heads of a projection's output, in place; the values behind them stay; heads outermost; odd
    strides and bases (one element at a time)."""
    g = A.gen(2)
    T, D = 11, 128
    qkv = A.normal(g, T, 9 * D)
    pos = torch.randint(0, 1 << 20, (T,), generator=g, dtype=torch.int32)
    freqs = _freqs(32)
    dev = qkv.cuda()
    heads = dev.view(T, 9, D)[:, :7]
    y = Q.rotary(heads, pos.cuda(), freqs.cuda(), interleaved=interleaved, out=heads)
    assert y is heads
    _check_rotary(heads, qkv.view(T, 9, D)[:, :7], pos, freqs, interleaved=interleaved)
    assert torch.equal(dev.view(T, 9, D)[:, 7:].cpu(), qkv.view(T, 9, D)[:, 7:])
    x = A.normal(g, 5, T, D)
    y = Q.rotary(x.cuda().transpose(0, 1), pos.cuda(), freqs.cuda(), interleaved=interleaved)
    assert y.is_contiguous()
    _check_rotary(y, x.transpose(0, 1), pos, freqs, interleaved=interleaved)
    flat = A.normal(g, T * 3 * 131 + 1)
    x = flat[1:].view(T, 3, 131)[:, :, 1:129]
    full = torch.zeros((T, 3, 133), dtype=torch.float16, device="cuda")
    Q.rotary(flat.cuda()[1:].view(T, 3, 131)[:, :, 1:129], pos.cuda(), freqs.cuda(), interleaved=interleaved,
             out=full[:, :, 3:131])
    _check_rotary(full[:, :, 3:131], x, pos, freqs, interleaved=interleaved)
    assert not full[:, :, :3].any() and not full[:, :, 131:].any()


def test_rotary_far_and_negative_positions():
    """Angles of 2^31 radians keep their turn: binary32 would lose it."""
    pos = torch.tensor([0, 1, -1, 12345678, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32)
    freqs = torch.cat([_freqs(31), torch.tensor([1.0], dtype=torch.float64)])
    x = A.normal(A.gen(3), 6, 2, 64, dtype=torch.float32)
    y = Q.rotary(x.cuda(), pos.cuda(), freqs.cuda())
    # 2^31 turns / (2 pi) in binary64: 2^-53 of them, two roundings
    ref, size = A.rotated(x.double(), pos, freqs)
    err = (y.cpu().double() - ref).abs()
    assert bool((err <= ref.abs() * 2.0 ** -24 + size * (1 + 2.0 ** 31 * 3 * 2.0 ** -53 / (6 * 2.0 ** -24))).all())


def test_rotary_gradient():
    """The inverse takes the result's gradient to x's: against differences of a linear functional."""
    g = A.gen(4)
    x, w = A.normal(g, 3, 2, 32, dtype=torch.float32), A.normal(g, 3, 2, 32, dtype=torch.float32)
    pos, freqs = torch.tensor([5, 900, 70000], dtype=torch.int32), _freqs(12)
    grad = Q.rotary(w.cuda(), pos.cuda(), freqs.cuda(), factor=1.5, inverse=True).cpu().double()
    for t, h, c in ((0, 0, 0), (1, 1, 13), (2, 0, 23), (2, 1, 30)):
        d = torch.zeros_like(x)
        d[t, h, c] = 1      # the map is linear: a difference of any size is the derivative
        f = [float((Q.rotary((x + s * d).cuda(), pos.cuda(), freqs.cuda(), factor=1.5).cpu().double() * w).sum())
             for s in (1, -1)]
        # every value of both sums off by a few last places of binary32
        assert abs((f[0] - f[1]) / 2 - float(grad[t, h, c])) <= 192 * 4 * 1.5 * 2.0 ** -21


@pytest.mark.parametrize("scaling,kw", [("none", {}), ("linear", {"factor": 4.0}), ("base", {"factor": 8.0}),
                                        ("ramp", {"factor": 4.0, "original": 4096}),
                                        ("bands", {"factor": 8.0, "original": 8192, "high": 4.0})])
def test_rotary_frequencies(scaling, kw):
    dim, base = 64, 10000.0
    freqs, attention = Q.rotary_frequencies(dim, base, scaling=scaling, **kw)
    plain = base ** (-np.arange(0, dim, 2) / dim)
    got = freqs.cpu().numpy()
    f = kw.get("factor", 1.0)
    assert got.dtype == np.float64 and got.shape == (32,)
    if scaling == "none":
        assert np.allclose(got, plain, rtol=1e-14)
    elif scaling == "linear":
        assert np.allclose(got, plain / f, rtol=1e-14)
    else:
        assert np.isclose(got[0], plain[0]) and np.isclose(got[-1], plain[-1] / f)
        assert np.all(got <= plain * (1 + 1e-12)) and np.all(got >= plain / f * (1 - 1e-12))
    assert np.isclose(attention, 0.1 * np.log(f) + 1 if scaling == "ramp" else 1.0)


CACHES = [(1, 1, 64), (1, 8, 128), (20, 8, 128), (17, 3, 64), (9, 2, 256), (130, 5, 128), (70, 1, 256), (333, 2, 64)]


def _kv(g, T, H, D, dtype):
    k, v = A.normal(g, T, H, D, scale=3.0, dtype=dtype), A.normal(g, T, H, D, dtype=dtype)
    if T > 3:
        k[1] = 0                                  # a block of zeros
        v[2, :, :32] = k[2, :, :32] * 2.0 ** -13  # a small block (below f16's normal range in places)
        v[0, 0, 5] = float("nan")
        k[3, -1, D - 1] = float("-inf")
    return k, v


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,H,D", CACHES)
def test_cache_write_and_read(T, H, D, dtype):
    """Bit for bit: the layout of the pages that are written, all others as they were, and the values read back."""
    g = A.gen(5, T, H, D)
    k, v = _kv(g, T, H, D, A.TYPES[dtype])
    pages = -(-T // 64) + 2
    slots = torch.randperm(pages * 64, generator=g)[:T].to(torch.int32)
    if T > 5:
        slots[4], slots[5] = -1, pages * 64       # passed over
    say("cache", T, H, D, dtype)
    cache = Q.kv4_cache(pages, H, D)
    cache.fill_(0xA5)
    assert Q.kv4_write(cache, k.cuda(), v.cuda(), slots.cuda()) is cache
    kc, ks = U.quantize(k.double().view(-1, D).numpy())
    vc, vs = U.quantize(v.double().view(-1, D).numpy())
    got = cache.cpu().numpy()
    held = {int(s): t for t, s in enumerate(slots) if 0 <= s < pages * 64}
    for p in range(pages):
        for h in range(H):
            # which bytes belong to slots that were written, and what they are
            def rows(c, w, other):
                return [c[held[p * 64 + t] * H + h] if p * 64 + t in held else np.full(w, other, np.uint8) for t in range(64)]
            want = A.record((rows(kc, D // 2, 0xA5), rows(ks, D // 32, 0xA5)), (rows(vc, D // 2, 0xA5), rows(vs, D // 32, 0xA5)), D)
            assert np.array_equal(got[p, h], want), (p, h)
    for out in (torch.float16, torch.bfloat16, torch.float32):
        for t, codes, scales in zip(Q.kv4_read(cache, slots.cuda(), dtype=out), (kc, vc), (ks, vs)):
            with np.errstate(all="ignore"):
                ref = torch.from_numpy(U.values(codes, scales).astype(np.float32)).view(T, H, D).to(out)
            for i, s in enumerate(slots):
                if not 0 <= s < pages * 64:
                    ref[i] = 0
            assert torch.equal(t.cpu().nan_to_num(77), ref.nan_to_num(77)) and torch.equal(t.cpu().isnan(), ref.isnan())


def test_cache_of_strided_keys_and_values():
    """Slices of a projection's output, heads outermost, one token."""
    g = A.gen(6)
    T, H, D = 19, 4, 128
    qkv = A.normal(g, T, (8 + 2 * H) * D)
    dev = qkv.cuda().view(T, 8 + 2 * H, D)
    slots = torch.arange(T, dtype=torch.int32).flip(0)
    ref = Q.kv4_write(Q.kv4_cache(1, H, D), dev[:, 8:8 + H].contiguous(), dev[:, 8 + H:].contiguous(), slots.cuda())
    assert torch.equal(Q.kv4_write(Q.kv4_cache(1, H, D), dev[:, 8:8 + H], dev[:, 8 + H:], slots.cuda()), ref)
    turned = [dev[:, 8:8 + H].transpose(0, 1).contiguous().transpose(0, 1), dev[:, 8 + H:].transpose(0, 1).contiguous().transpose(0, 1)]
    assert torch.equal(Q.kv4_write(Q.kv4_cache(1, H, D), *turned, slots.cuda()), ref)
    one = Q.kv4_cache(1, H, D)
    for t in range(T):
        Q.kv4_write(one, dev[t:t + 1, 8:8 + H], dev[t:t + 1, 8 + H:], slots[t:t + 1].cuda())
    assert torch.equal(one, ref)


def test_cache_past_32_bits():
    """Pages whose bytes lie beyond 4 GiB of the cache."""
    H, D = 8, 256
    pages = (1 << 32) // (H * 68 * D) + 3
    cache = torch.empty((pages, H, 68 * D), dtype=torch.uint8, device="cuda")
    cache[0].fill_(1)
    cache[-2:].fill_(1)
    g = A.gen(7)
    k, v = A.normal(g, 6, H, D), A.normal(g, 6, H, D)
    slots = torch.tensor([0, 63, pages * 64 - 1, pages * 64 - 64, pages * 64 - 65, 5], dtype=torch.int32)
    Q.kv4_write(cache, k.cuda(), v.cuda(), slots.cuda())
    kk, vv = Q.kv4_read(cache, slots.cuda(), dtype=torch.float32)
    assert torch.equal(kk.cpu().double(), A.rounded(k)) and torch.equal(vv.cpu().double(), A.rounded(v))


def test_nothing_to_do():
    cache = Q.kv4_cache(2, 3, 64)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    x = torch.empty((0, 3, 64), dtype=torch.float16, device="cuda")
    Q.kv4_write(cache, x, x, none)
    assert Q.kv4_read(cache, none)[0].shape == (0, 3, 64)
    assert Q.rotary(x, none, _freqs(8).cuda()).shape == (0, 3, 64)


def test_rotary_angles_of_far_positions():
    """Frequency 1, positions up to 2^31: cosine and sine themselves, against those of the whole number of radians.  The
    turns are off by the roundings of 1 / (2 pi) (2^-53.8 of them) and of the product (2^-53), 2^-21.3 of a radian
    together, the rest of a turn by 2^-26 of one in binary32 (2^-23.3), and the functions by two last places (2^-23)."""
    g = A.gen(13)
    pos = torch.cat([torch.randint(1 << 30, (1 << 31) - 1, (20000,), generator=g), torch.randint(-(1 << 31), 1 << 20, (20000,), generator=g),
                     torch.tensor([(1 << 31) - 1, -(1 << 31)])])
    x = torch.tensor([1.0, 0.0]).expand(pos.shape[0], 1, 2).contiguous()
    y = Q.rotary(x.cuda(), pos.to(torch.int32).cuda(), torch.ones(1, dtype=torch.float64, device="cuda")).cpu().double()
    angle = pos.double()
    err = (y[:, 0] - torch.stack([torch.cos(angle), torch.sin(angle)], 1)).abs().max()
    assert float(err) <= 2.0 ** -21.3 + 2.0 ** -23.3 + 2.0 ** -23, float(err)
