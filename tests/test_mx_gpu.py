"""Microscaled 4-bit floating point (include/quick_mx.h) on the GPU through the
C ABI against binary64 forms of the definitions: codes, scales and packed
bytes exactly; products exactly where every sum is exact in binary32, and
otherwise within the rounding of the result and of the sums."""
import numpy as np
import pytest
import torch

import mx_util as U
import paper_2402_10076_amd as Q
from gpu_util import say

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# half a unit in the last place, relative
EPS = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def _rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _typed(v, dtype):
    """A device tensor of v in dtype and the binary64 values that it holds."""
    t = torch.from_numpy(np.asarray(v, np.float32)).to(dtype)
    return t.cuda(), t.double().numpy()


def _random_mx(seed, rows, K, spread=3):
    """Random codes and scales within 2^-spread .. 2^spread."""
    g = _rng(seed, rows, K)
    return (g.integers(0, 256, (rows, K // 2), dtype=np.uint8),
            g.integers(127 - spread, 128 + spread, (rows, K // 32), dtype=np.uint8))


# ---------------------------------------------------------------------------
# quantisation
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 32), (1, 4096), (3, 96), (7, 8224), (65, 1056), (200, 160)])
def test_quantize_is_exact(dtype, rows, K):
    g = _rng(1, rows, K)
    # magnitudes over the type's range, with zeros
    v = g.standard_normal((rows, K)) * 2.0 ** g.uniform(-12, 12, (rows, K // 32)).repeat(32, 1)
    v[g.random((rows, K)) < 0.05] = 0
    x, xv = _typed(v, TYPES[dtype])
    say("quantize %s %dx%d" % (dtype, rows, K))
    codes, scales = Q.mxfp4_quantize(x)
    rc, rs = U.quantize(xv)
    assert np.array_equal(scales.cpu().numpy(), rs)
    assert np.array_equal(codes.cpu().numpy(), rc)
    back = Q.mxfp4_dequantize(codes, scales, dtype=TYPES[dtype])
    ref = torch.from_numpy(U.values(rc, rs).astype(np.float32)).to(TYPES[dtype])
    assert torch.equal(back.cpu(), ref)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_quantize_ties_signs_and_saturation(dtype):
    """Every midpoint of the grid, its neighbours in the type, both signs, and
    magnitudes up to the next power of two (which saturate at 6)."""
    t = TYPES[dtype]
    points = [0.0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 6.5, 7, 7.75]
    vals = []
    for p in points:
        q = torch.tensor([p], dtype=t)
        vals += [float(q), float(torch.nextafter(q, torch.tensor([100.0], dtype=t))),
                 float(torch.nextafter(q, torch.tensor([-100.0], dtype=t)))]
    v = np.array(vals)
    v = np.concatenate([v[np.abs(v) < 8], -v[np.abs(v) < 8]])
    blocks = []
    for i in range(0, len(v), 31):
        b = np.zeros(32)
        b[0] = 4.0                        # fixes the scale at 2^0
        b[1:1 + len(v[i:i + 31])] = v[i:i + 31]
        blocks.append(b)
    for e in (0, -9, 9):
        x, xv = _typed(np.stack(blocks) * 2.0 ** e, t)
        say("ties", dtype, e)
        codes, scales = Q.mxfp4_quantize(x)
        rc, rs = U.quantize(xv)
        assert np.array_equal(scales.cpu().numpy(), rs) and np.array_equal(codes.cpu().numpy(), rc)


def test_quantize_special_blocks():
    """Zero blocks, -0, blocks below and at the end of the scales' range, the
    largest values, NaN and infinities."""
    b = np.zeros((9, 32), np.float32)
    b[1, ::2] = -0.0
    b[2, 3] = 2.0 ** -149
    b[3] = 2.0 ** -126 * np.linspace(-1, 1, 32)
    b[4] = np.float32(2.0 ** -125) * np.linspace(-1.9, 1.9, 32).astype(np.float32)
    b[5] = np.float32(3.4e38) * np.linspace(-1, 1, 32).astype(np.float32)
    b[6] = 1
    b[6, 31] = np.nan
    b[7] = 1
    b[7, 0] = -np.inf
    b[8] = 2.0
    codes, scales = Q.mxfp4_quantize(_dev(b.reshape(1, -1)))
    rc, rs = U.quantize(b.reshape(1, -1).astype(np.float64))
    say(scales.cpu().numpy(), rs)
    assert np.array_equal(scales.cpu().numpy(), rs) and np.array_equal(codes.cpu().numpy(), rc)
    back = Q.mxfp4_dequantize(codes, scales, dtype=torch.float32).cpu().numpy()
    assert np.array_equal(back.astype(np.float64), U.values(rc, rs), equal_nan=True)
    x16 = torch.tensor(b.reshape(1, -1)).to(torch.bfloat16)
    codes, scales = Q.mxfp4_quantize(x16.cuda())
    rc, rs = U.quantize(x16.double().numpy())
    assert np.array_equal(scales.cpu().numpy(), rs) and np.array_equal(codes.cpu().numpy(), rc)


@pytest.mark.parametrize("dtype,pad", [("f16", 8), ("bf16", 40), ("f32", 4)])
def test_quantize_rows_apart_and_given_outputs(dtype, pad):
    rows, K = 37, 2080
    wide, wv = _typed(_rng(5).standard_normal((rows, K + pad)), TYPES[dtype])
    x = wide[:, :K]
    out = (torch.full((rows, K // 2), 0xAA, dtype=torch.uint8, device="cuda"),
           torch.full((rows, K // 32), 0xAA, dtype=torch.uint8, device="cuda"))
    got = Q.mxfp4_quantize(x, *out)
    rc, rs = U.quantize(wv[:, :K])
    assert got[0].data_ptr() == out[0].data_ptr() and got[1].data_ptr() == out[1].data_ptr()
    assert np.array_equal(out[0].cpu().numpy(), rc) and np.array_equal(out[1].cpu().numpy(), rs)


def test_quantize_writes_nothing_past_its_outputs():
    for rows, K in ((1, 32), (5, 96), (3, 8224)):
        x, _ = _typed(_rng(6, rows).standard_normal((rows, K)), torch.float16)
        n, m = rows * K // 2, rows * K // 32
        codes = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        scales = torch.full((m + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        Q.mxfp4_quantize(x, codes[:n].view(rows, K // 2), scales[:m].view(rows, K // 32))
        assert bool((codes[n:] == 0x5A).all()) and bool((scales[m:] == 0x5A).all())


def test_quantize_zero_rows():
    codes, scales = Q.mxfp4_quantize(torch.zeros((0, 64), dtype=torch.float16, device="cuda"))
    assert codes.shape == (0, 32) and scales.shape == (0, 2)
    assert Q.mxfp4_dequantize(codes, scales).shape == (0, 64)


def test_dequantize_every_code_and_scale():
    """All 16 codes under all 256 scales, in every type: rounding to f16 (with
    infinities and values below its range) and to bf16 as torch's cast."""
    codes = np.tile(np.arange(16, dtype=np.uint8) | np.arange(16, dtype=np.uint8)[::-1] << 4, (256, 1))
    scales = np.arange(256, dtype=np.uint8)[:, None]
    v = torch.from_numpy(U.values(codes, scales).astype(np.float32))
    for t in TYPES.values():
        got = Q.mxfp4_dequantize(_dev(codes), _dev(scales), dtype=t).cpu()
        ref = v.to(t)
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        assert torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(ref, nan=0.0))


@pytest.mark.parametrize("E,N,K,gate_up", [(None, 16, 32, False), (None, 37, 160, False), (None, 64, 1184, True),
                                           (3, 48, 544, False), (2, 96, 512, True)])
def test_pack_layout(E, N, K, gate_up):
    codes, scales = _random_mx(7, (E or 1) * N, K)
    lead = (E,) if E else ()
    p, s = Q.mxfp4_pack(_dev(codes.reshape(*lead, N, K // 2)), _dev(scales.reshape(*lead, N, K // 32)),
                        gate_up=gate_up)
    p, s = p.cpu().numpy().reshape(E or 1, -1), s.cpu().numpy().reshape(E or 1, -1)
    assert (p.shape[1], s.shape[1]) == Q.mxfp4_packed_sizes(N, K)
    for e in range(E or 1):
        rp, rs = U.packed(codes[e * N:(e + 1) * N], scales[e * N:(e + 1) * N], gate_up)
        assert np.array_equal(p[e], rp) and np.array_equal(s[e], rs)


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------

def _check(y, ref, size, K, dtype):
    """y against binary64 ref: the rounding of the result, and of sums of K
    products in binary32 in any order (2^-23 of the products' magnitudes a
    step), size = sum of |x| |w|."""
    got = y.double().cpu().numpy()
    assert np.isfinite(got).all()
    tol = EPS[dtype] * 1.001 * np.abs(ref) + K * 2.0 ** -23 * size + 2.0 ** -24
    worst = np.max(np.abs(got - ref) / tol)
    say("  worst error %.3g of its bound" % worst)
    assert worst <= 1


SHAPES = [(1, 16, 32), (1, 512, 4096), (2, 48, 160), (5, 33, 544), (15, 272, 1024), (16, 16, 128), (17, 130, 512),
          (31, 96, 2080), (33, 256, 640), (64, 80, 1184), (65, 528, 512), (129, 144, 1152), (200, 1, 96),
          (257, 400, 768), (300, 1040, 1536)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_is_exact_where_the_sums_are(M, N, K):
    """Scales 2^0 and 2^1 on both sides: every product is a multiple of 1/4 and
    every sum under 2^24 / 4, so binary32 holds all of them and y is the
    rounded exact result."""
    g = _rng(11, M, N, K)
    xc, wc = g.integers(0, 256, (M, K // 2), dtype=np.uint8), g.integers(0, 256, (N, K // 2), dtype=np.uint8)
    xs, ws = (g.integers(127, 129, (r, K // 32), dtype=np.uint8) for r in (M, N))
    ref = U.values(xc, xs) @ U.values(wc, ws).T
    say("gemm exact", M, N, K)
    packed = Q.mxfp4_pack(_dev(wc), _dev(ws))
    for dtype in (torch.float16, torch.bfloat16):
        y = Q.mxfp4_gemm(_dev(xc), _dev(xs), *packed, N, dtype=dtype)
        assert y.shape == (M, N)
        assert torch.equal(y.cpu(), torch.from_numpy(ref).to(torch.float32).to(dtype))


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_wide_scales(M, N, K):
    xc, xs = _random_mx(12, M, K, 6)
    wc, ws = _random_mx(13, N, K, 6)
    xs[:, ::3] -= 8
    xv, wv = U.values(xc, xs), U.values(wc, ws) * 2.0 ** -6
    say("gemm", M, N, K)
    y = Q.mxfp4_gemm(_dev(xc), _dev(xs), *Q.mxfp4_pack(_dev(wc), _dev((ws - 6).astype(np.uint8))), N,
                     dtype=torch.bfloat16)
    _check(y, xv @ wv.T, np.abs(xv) @ np.abs(wv).T, K, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,Nh,K", [(1, 16, 32), (1, 256, 4096), (9, 48, 160), (33, 144, 544), (70, 112, 640),
                                    (150, 336, 1024)])
def test_gemm_bias_and_gated(M, Nh, K, dtype):
    g = _rng(14, M, Nh, K)
    N = 2 * Nh
    xc, xs = _random_mx(15, M, K, 1)
    wc, ws = _random_mx(16, N, K, 1)
    ws -= 5
    xv, wv = U.values(xc, xs), U.values(wc, ws)
    bias, bv = _typed(g.uniform(-2, 2, N), dtype)
    h, size = xv @ wv.T + bv, np.abs(xv) @ np.abs(wv).T + np.abs(bv)
    x = (_dev(xc), _dev(xs))
    plain, gated = (Q.mxfp4_pack(_dev(wc), _dev(ws), gate_up=f) for f in (False, True))
    say("bias, gated", M, N, K, dtype)
    _check(Q.mxfp4_gemm(*x, *plain, N, bias=bias, dtype=dtype), h, size, K, dtype)
    # d(silu(g) u) = silu'(g) u dg + silu(g) du with |silu'| < 1.1, |silu(g)| <= |g|
    hn, sn = h[:, :Nh], size[:, :Nh]
    gsize = 1.1 * sn * np.abs(h[:, Nh:]) + np.abs(hn) * size[:, Nh:]
    for b, hh in ((bias, h), (None, xv @ wv.T)):
        y = Q.mxfp4_gemm(*x, *gated, N, bias=b, activation=Q.ACT_SILU_GATE, dtype=dtype)
        assert y.shape == (M, Nh)
        _check(y, U.silu_gate(hh), gsize + np.abs(bv[:Nh]) * sn + np.abs(bv[Nh:]) * sn, K + 8, dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(1, 16, 32), (1, 1024, 4096), (2, 272, 11008), (3, 130, 544), (4, 528, 2080),
                                   (5, 256, 1024), (8, 64, 14336), (16, 160, 640), (23, 96, 5120), (150, 320, 1056)])
def test_linear_is_quantize_then_gemm(M, N, K, dtype):
    """The call on 16-bit activations gives the bits of the two calls, with a
    workspace of its own and with the caller's, also with outliers, zeros and
    blocks with a NaN."""
    g = _rng(17, M, N, K)
    v = g.standard_normal((M, K))
    v[:, ::97] *= 20
    v[:, 32:64] = 0
    x, xv = _typed(v, dtype)
    wc, ws = _random_mx(18, N, K, 1)
    ws -= 4
    packed = Q.mxfp4_pack(_dev(wc), _dev(ws))
    bias, bv = _typed(g.uniform(-2, 2, N), dtype)
    say("linear", M, N, K, dtype)
    need = Q.mxfp4_linear_workspace_bytes(M, N, K)
    work = torch.full((need + 16,), 0x7F, dtype=torch.uint8, device="cuda")
    for b in (None, bias):
        two = Q.mxfp4_gemm(*Q.mxfp4_quantize(x), *packed, N, bias=b, dtype=dtype)
        assert torch.equal(Q.mxfp4_linear(x, *packed, N, bias=b), two)
        assert torch.equal(Q.mxfp4_linear(x, *packed, N, bias=b, workspace=work), two)
    assert bool((work[need:] == 0x7F).all())
    qv, wv = U.values(*U.quantize(xv)), U.values(wc, ws)
    _check(two, qv @ wv.T + bv, np.abs(qv) @ np.abs(wv).T + np.abs(bv), K, dtype)
    x[M - 1, 5] = float("nan")
    y = Q.mxfp4_linear(x, *packed, N)
    assert bool(torch.isnan(y[M - 1]).all()) and not bool(torch.isnan(y[:M - 1]).any())


def test_nan_scales_reach_their_rows_and_columns_alone():
    for M, N, K in ((3, 48, 160), (40, 64, 1024), (130, 288, 512)):
        xc, xs = _random_mx(19, M, K, 1)
        wc, ws = _random_mx(20, N, K, 1)
        xs[1, 2] = 255
        ws[N - 3, K // 32 - 1] = 255
        y = Q.mxfp4_gemm(_dev(xc), _dev(xs), *Q.mxfp4_pack(_dev(wc), _dev(ws)), N).cpu()
        bad = torch.zeros((M, N), dtype=torch.bool)
        bad[1] = True
        bad[:, N - 3] = True
        say("nan", M, N, K)
        assert torch.equal(torch.isnan(y), bad)


def test_gemm_result_beyond_f16():
    xc = np.full((2, 256), 0x77, np.uint8)             # 6
    s = np.full((2, 16), 127 + 6, np.uint8)
    y = Q.mxfp4_gemm(_dev(xc), _dev(s), *Q.mxfp4_pack(_dev(xc), _dev(s)), 2)
    assert bool(torch.isinf(y).all())
    y = Q.mxfp4_gemm(_dev(xc), _dev(s), *Q.mxfp4_pack(_dev(xc), _dev(s)), 2, dtype=torch.bfloat16)
    assert torch.equal(y.float().cpu(), torch.full((2, 2), 36.0 * 512 * 4096))


def test_given_output_no_rows_and_other_streams():
    M, N, K = 20, 100, 544
    xc, xs = _random_mx(21, M, K)
    wc, ws = _random_mx(22, N, K)
    packed = Q.mxfp4_pack(_dev(wc), _dev(ws))
    x = (_dev(xc), _dev(xs))
    whole = torch.full((M + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    ref = Q.mxfp4_gemm(*x, *packed, N, dtype=torch.bfloat16)
    Q.mxfp4_gemm(*x, *packed, N, y=whole[1:M + 1])
    assert torch.equal(whole[1:M + 1], ref) and bool((whole[0] == 7).all()) and bool((whole[M + 1] == 7).all())
    assert Q.mxfp4_gemm(x[0][:0], x[1][:0], *packed, N).shape == (0, N)
    assert Q.mxfp4_linear(torch.zeros((0, K), dtype=torch.float16, device="cuda"), *packed, N).shape == (0, N)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = Q.mxfp4_gemm(*x, *packed, N, dtype=torch.bfloat16, stream=side)
    xt = Q.mxfp4_dequantize(*x, dtype=torch.bfloat16)
    side.wait_stream(torch.cuda.current_stream())
    z = Q.mxfp4_linear(xt, *packed, N, stream=side)
    side.synchronize()
    assert torch.equal(y, ref) and z.shape == ref.shape


def _experts(seed, E, N, K):
    c, s = _random_mx(seed, E * N, K, 1)
    return c.reshape(E, N, K // 2), (s - 4).reshape(E, N, K // 32).astype(np.uint8)


COUNTS = [[1], [0, 3, 0], [5, 0, 1, 2, 0, 9], [16, 17, 15, 33], [0, 0, 130, 0], [70, 1, 0, 64, 65],
          [300, 4, 257, 128, 129], [1] * 40, [0] * 63 + [5] + [0] * 448]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "E%d_R%d" % (len(c), sum(c)))
@pytest.mark.parametrize("N,K", [(96, 160), (272, 1024)])
def test_grouped(counts, N, K):
    """Uneven and empty experts, gathered rows with repeats and rows in order,
    bias, gated; against the dense product expert by expert."""
    E, R = len(counts), sum(counts)
    if E * N * K > 1 << 25:
        N = 32
    g = _rng(23, R, N)
    T = max(3, R // 2)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows = g.integers(0, T, R).astype(np.int32)
    xc, xs = _random_mx(24, T, K, 1)
    wc, ws = _experts(25, E, N, K)
    bias, bv = _typed(g.uniform(-2, 2, (E, N)), torch.float16)
    xv = U.values(xc, xs)
    packed = Q.mxfp4_pack(_dev(wc), _dev(ws))
    x, o, r = (_dev(xc), _dev(xs)), _dev(offsets), _dev(rows)
    say("grouped", counts[:8], N, K)
    y = Q.mxfp4_grouped_gemm(*x, o, *packed, N, rows=r, bias=bias)
    z = None
    if N % 32 == 0:
        z = Q.mxfp4_grouped_gemm(*x, o, *Q.mxfp4_pack(_dev(wc), _dev(ws), gate_up=True), N, rows=r,
                                 activation=Q.ACT_SILU_GATE)
        assert z.shape == (R, N // 2)
    assert y.shape == (R, N)
    xg = (x[0][r.long()].contiguous(), x[1][r.long()].contiguous())
    assert torch.equal(Q.mxfp4_grouped_gemm(*xg, o, *packed, N, bias=bias), y)
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if a == b:
            continue
        xe, we = xv[rows[a:b]], U.values(wc[e], ws[e])
        h, size = xe @ we.T, np.abs(xe) @ np.abs(we).T
        _check(y[a:b], h + bv[e], size + np.abs(bv[e]), K, torch.float16)
        if z is None:
            continue
        n = N // 2
        _check(z[a:b], U.silu_gate(h), 1.1 * size[:, :n] * np.abs(h[:, n:]) + np.abs(h[:, :n]) * size[:, n:], K + 8,
               torch.float16)


def test_grouped_leaves_other_rows_and_clamps():
    """Rows that no expert owns keep what they hold; offsets and rows beyond
    the contract stay inside the buffers, and rows within it are right."""
    E, N, K, T, R = 3, 48, 160, 10, 30
    xc, xs = _random_mx(26, T, K, 1)
    wc, ws = _experts(27, E, N, K)
    packed = Q.mxfp4_pack(_dev(wc), _dev(ws))
    x = (_dev(xc), _dev(xs))
    rows = _dev(np.arange(R, dtype=np.int32) % T)
    y = torch.full((R, N), 9.0, dtype=torch.float16, device="cuda")
    Q.mxfp4_grouped_gemm(*x, _dev(np.array([2, 5, 5, 20], np.int32)), *packed, N, rows=rows, y=y)
    assert bool((y[:2] == 9).all()) and bool((y[20:] == 9).all())
    full = Q.mxfp4_grouped_gemm(*x, _dev(np.array([0, 5, 5, 30], np.int32)), *packed, N, rows=rows)
    assert torch.equal(y[2:20], full[2:20])
    guard = torch.full((R + 4, N), 9.0, dtype=torch.float16, device="cuda")
    wild = _dev(np.array([-7, 12, 3, 1 << 30], np.int32))
    bad = rows.clone()
    bad[25:] = torch.tensor([-1, T, 1 << 30, -(1 << 31), 7], dtype=torch.int32)
    Q.mxfp4_grouped_gemm(*x, wild, *packed, N, rows=bad, y=guard[2:R + 2])
    torch.cuda.synchronize()
    assert bool((guard[:2] == 9).all()) and bool((guard[R + 2:] == 9).all())
    assert torch.equal(guard[2:14], Q.mxfp4_grouped_gemm(*x, _dev(np.array([0, 12, 12, 30], np.int32)), *packed, N,
                                                         rows=rows)[:12])


def test_grouped_no_rows():
    wc, ws = _experts(28, 2, 32, 64)
    packed = Q.mxfp4_pack(_dev(wc), _dev(ws))
    c, s = _random_mx(29, 4, 64)
    e = torch.zeros(0, dtype=torch.int32, device="cuda")
    o = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert Q.mxfp4_grouped_gemm(_dev(c), _dev(s), o, *packed, 32, rows=e).shape == (0, 32)
    y = torch.full((4, 32), 3.0, dtype=torch.float16, device="cuda")
    Q.mxfp4_grouped_gemm(_dev(c), _dev(s), o, *packed, 32, y=y)
    assert bool((y == 3).all())


def test_products_repeat_and_replay():
    """The same bits from call to call and from replays of a captured graph."""
    for M, N, K in ((1, 528, 4096), (20, 160, 1056), (260, 288, 640)):
        x, _ = _typed(_rng(30, M).standard_normal((M, K)), torch.float16)
        wc, ws = _random_mx(31, N, K, 1)
        packed = Q.mxfp4_pack(_dev(wc), _dev((ws - 4).astype(np.uint8)))
        ref = Q.mxfp4_linear(x, *packed, N)
        out = torch.empty_like(ref)
        work = torch.empty(max(16, Q.mxfp4_linear_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            Q.mxfp4_linear(x, *packed, N, y=out, workspace=work)
        for _ in range(3):
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref)
            assert torch.equal(Q.mxfp4_linear(x, *packed, N), ref)
