"""Microscaled products, bit for bit, at the sizes that the lists of
test_mx_forms_gpu.py leave out: every form of the kernels with whole, partial
and cut-off quarters of its scales (512 channels each), with weights past the
caches, dense and over experts; test_mx_coverage.py says on the CPU which."""
import numpy as np
import pytest
import torch

import mx_util as U
import paper_2402_10076_amd as Q
import test_mx_forms_gpu as F
from gpu_util import say

pytestmark = pytest.mark.gpu


def skewed(E, R):
    """Rows of E experts, R or a little fewer, from few to many; every fourth has none."""
    w = [0 if i % 4 == 3 else (i + 1) ** 2 for i in range(E)]
    return [max(R * v // sum(w), 1 if v else 0) for v in w]


# (rows, columns, channels)
DENSE = [
    (640, 5760, 2880), (884, 96, 2880), (1, 32, 128), (1171, 3520, 128), (3353, 576, 256), (1, 32, 512),
    (336, 23616, 512), (1, 32, 1280), (100, 13696, 1280), (2099, 32, 1920), (850, 9888, 2176), (2142, 19, 2688),
    (2048, 8192, 4224), (2257, 64, 8064), (333, 5120, 11008), (512, 4096, 11008)]

# weights past the caches
DENSE_ONCE = [
    (34, 49344, 8224), (1, 32704, 12320), (1, 32800, 12320), (1, 28160, 14368), (33, 32768, 14368),
    (40, 17075, 28704), (1, 49952, 8064), (1, 28128, 14336), (48, 57344, 14336), (34, 23360, 17280),
    (33, 19904, 20480), (1, 16512, 25472), (34, 16672, 25472), (48, 17600, 27648), (1, 14272, 28288)]

# (experts, rows in all, columns, channels)
GROUPED = [
    (2, 1, 32, 32), (2, 156, 10368, 32), (13, 609, 4512, 32), (2, 5, 32, 1440), (3, 47, 32, 1440),
    (2, 2490, 480, 6944), (2, 1, 32, 128), (4, 236, 11712, 128), (5, 2928, 672, 128), (2, 1955, 1088, 512),
    (13, 4388, 1600, 512), (64, 500, 2816, 640), (8, 2000, 4224, 1152), (2, 2, 32, 1280), (3, 2415, 32, 2176),
    (5, 2405, 32, 2432), (4, 2224, 32, 2560), (2, 2051, 576, 4224), (2, 2396, 64, 8064), (5, 3021, 64, 8192),
    (8, 700, 4096, 11008)]

# weights past the caches
GROUPED_ONCE = [
    (16, 19, 31488, 800), (32, 600, 5760, 2880), (2, 1, 16448, 12320), (2, 1, 7808, 25888), (3, 151, 5344, 25888),
    (40, 34, 416, 25888), (13, 11, 34624, 896), (13, 12, 30272, 1024), (3, 1, 49984, 2688), (13, 14, 1248, 25472),
    (13, 22, 1248, 25472), (64, 3541, 256, 25472), (5, 266, 3104, 27136), (13, 37, 1248, 27136), (2, 2, 7392, 27264),
    (3, 1, 4704, 28672), (40, 27, 480, 28672)]

# 16-bit activations that the launch quantises, gated: (rows, columns, channels)
ON_THE_WAY = [
    (2, 32, 32), (3, 32736, 12320), (1, 64, 128), (1, 23360, 17280)]


@pytest.mark.parametrize("M,N,K", DENSE + DENSE_ONCE)
def test_dense(M, N, K):
    F.test_dense_forms(M, N, K)


@pytest.mark.parametrize("E,R,N,K", GROUPED + GROUPED_ONCE)
def test_grouped(E, R, N, K):
    F.test_grouped_forms(skewed(E, R), N, K)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", ON_THE_WAY)
def test_gated_with_quantisation_on_the_way(M, N, K, dtype):
    """The one call and the two, which may run in forms that add in different
    orders, against the definition."""
    g = F._gen(20, M, N, K)
    x = torch.randn((M, K), device="cuda", generator=g).to(dtype)
    wc, ws = F._codes(g, N, K // 2), F._scales(g, 119, N, K // 32)
    packed = Q.mxfp4_pack(wc, ws, gate_up=True)
    say("on the way", M, N, K, dtype)
    y = Q.mxfp4_linear(x, *packed, N, activation=Q.ACT_SILU_GATE)
    codes, scales = Q.mxfp4_quantize(x)
    two = Q.mxfp4_gemm(codes, scales, *packed, N, activation=Q.ACT_SILU_GATE, dtype=dtype)
    h = F._product(F._values(codes, scales), wc, ws)
    # the rounding of y, of the sums (2^-23 of the products' magnitudes a step)
    # and of the epilogue, d(silu(g) u) = silu'(g) u dg + silu(g) du + silu'(g)
    # dg du with |silu'| < 1.1, |silu(g)| <= |g|
    size = F._product(F._values(codes, scales).abs(), wc & 0x77, ws)
    n = N // 2
    dh = K * 2.0 ** -23 * size
    ref = h[:, :n] * torch.sigmoid(h[:, :n]) * h[:, n:]
    tol = ((F.EPS[dtype] * 1.001 + 2.0 ** -19) * ref.abs() + 1.1 * dh[:, :n] * h[:, n:].abs()
           + h[:, :n].abs() * dh[:, n:] + 1.1 * dh[:, :n] * dh[:, n:] + 2.0 ** -24)
    for v in (y, two):
        assert bool(((v.double() - ref).abs() <= tol).all())


def test_rows_next_to_one_another_are_not_mixed():
    """Channels that end inside a quarter of the scales: the last row's copy is
    cut off by the end of the scales, the others' reach into the next row's,
    and a NaN scale there must stay in its row."""
    for M, N, K in ((130, 4096, 640), (512, 4096, 11008), (64, 2080, 4224), (300, 25600, 1152)):
        g = F._gen(21, M, N, K)
        xc, xs, wc, ws = F._codes(g, M, K // 2), F._scales(g, 119, M, K // 32), F._codes(g, N, K // 2), F._scales(g, 119, N, K // 32)
        xs[1::2] = 255
        say("next rows", M, N, K)
        y = Q.mxfp4_gemm(xc, xs, *Q.mxfp4_pack(wc, ws), N)
        assert bool(torch.isnan(y[1::2]).all())
        F._same(y[::2], F._product(F._values(xc[::2].contiguous(), xs[::2].contiguous()), wc, ws))


@pytest.mark.parametrize("M,N,K", [(1, 64, 160), (3, 512, 1024), (20, 160, 1056), (70, 544, 640), (200, 640, 1152)])
def test_scales_that_cancel(M, N, K):
    """Scales at both ends of their range, whose product is in the middle:
    2^-127 .. 2^-123 on one side, 2^123 .. 2^127 on the other, then the sides
    changed.  Every sum is exact in binary32."""
    g = F._gen(22, M, N, K)
    xc, wc = F._codes(g, M, K // 2), F._codes(g, N, K // 2)
    low = torch.randint(0, 5, (K // 32,), device="cuda", generator=g)
    for flip in (False, True):
        xs, ws = (v.to(torch.uint8) for v in ((low, 254 - low) if not flip else (254 - low, low)))
        xs, ws = xs.expand(M, -1).contiguous(), ws.expand(N, -1).contiguous()
        say("cancel", M, N, K, flip)
        y = Q.mxfp4_gemm(xc, xs, *Q.mxfp4_pack(wc, ws), N, dtype=torch.bfloat16)
        one = torch.full_like(xs, 127)
        F._same(y, F._product(F._values(xc, one), wc, torch.full_like(ws, 127)))
