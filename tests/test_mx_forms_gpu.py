"""Microscaled products and routing at the sizes that reach every kernel form
and tile shape, bit for bit against binary64 (the sums are exact in binary32),
and at sizes whose offsets pass 32 bits."""
import numpy as np
import pytest
import torch

import mx_util as U
import paper_2402_10076_amd as Q
from gpu_util import say

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
EPS = {F16: 2.0 ** -11, BF16: 2.0 ** -8}


def _gen(*seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(hash(seed) & 0xFFFFFFFF)
    return g


def _codes(g, *shape):
    return torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=g)


def _scales(g, low, *shape):
    return torch.randint(low, low + 2, shape, dtype=torch.uint8, device="cuda", generator=g)


def _values(codes, scales):
    """Binary64 values of codes [r][K/2] under scales [r][K/32]."""
    grid = torch.tensor(list(U.GRID) + list(-U.GRID), dtype=torch.float64, device="cuda")
    c = torch.stack((codes & 15, codes >> 4), -1).view(*scales.shape, 32).long()
    return (grid[c] * torch.exp2(scales.double() - 127)[..., None]).view(scales.shape[0], -1)


def _product(x, codes, scales, bias=None):
    """Binary64 x @ W^T, 4096 rows of W at a time."""
    h = torch.cat([x @ _values(codes[i:i + 4096], scales[i:i + 4096]).t() for i in range(0, codes.shape[0], 4096)], 1)
    return h if bias is None else h + bias.double()


def _same(y, h):
    assert torch.equal(y, h.to(y.dtype))


def _silu(y, h):
    """y against the gated h, of which binary32 holds every bit: the rounding
    of y and of an exponential, a division and a product in binary32."""
    n = h.shape[1] // 2
    ref = h[:, :n] * torch.sigmoid(h[:, :n]) * h[:, n:]
    assert bool(torch.isfinite(y).all())
    assert bool(((y.double() - ref).abs() <= (EPS[y.dtype] * 1.001 + 2.0 ** -19) * ref.abs() + 2.0 ** -24).all())


# (rows, columns, channels): a stream form of one, two and four column tiles
# (also with more runs of tiles than workgroups, and quantising on the way),
# tiles of 32x128, 64x64, 64x128 with eight and four stages, 128x128, 128x256
# and 256x256, each with whole and partial steps of channels, columns that are
# no multiple of a tile or of 8, and more row tiles than one band
DENSE = [(1, 512, 1056), (3, 520, 2048), (1, 8192, 2048), (16, 5008, 1056), (1, 12320, 2048), (5, 30020, 2048),
         (16, 57344, 1056), (64, 2080, 4128), (1, 8200, 512), (30, 2050, 160), (7, 12320, 2048), (61, 12320, 4128),
         (33, 25601, 4096), (64, 25600, 4128), (40, 25600, 512), (100, 25604, 160), (150, 12320, 512),
         (333, 5120, 2080), (150, 25600, 512), (600, 13000, 1056), (260, 25600, 512), (2310, 8200, 1024),
         (2100, 4112, 1056), (5000, 96, 288), (64, 2080, 8192), (50, 2080, 13856), (500, 2080, 4096), (200, 5120, 4128),
         (150, 12320, 160), (2, 57344, 160),
         # with a leading workgroup of each column
         (64, 1040, 2048), (512, 1056, 2080), (256, 4112, 4096), (512, 2080, 4128), (100, 10240, 2080), (512, 2080, 2048),
         (512, 4112, 2048), (1024, 2080, 2080), (448, 10240, 2080), (1024, 4112, 2048), (1536, 6144, 2048),
         (2048, 4112, 2048)]


@pytest.mark.parametrize("M,N,K", DENSE)
def test_dense_forms(M, N, K):
    g = _gen(1, M, N, K)
    xc, xs, wc, ws = _codes(g, M, K // 2), _scales(g, 127, M, K // 32), _codes(g, N, K // 2), _scales(g, 127, N, K // 32)
    bias = (torch.randint(-64, 65, (N,), device="cuda", generator=g) / 4).to(F16)
    xv = _values(xc, xs)
    h = _product(xv, wc, ws)
    packed = Q.mxfp4_pack(wc, ws)
    say("dense", M, N, K)
    guard = torch.full((M * N + 64,), 7.0, dtype=F16, device="cuda")
    _same(Q.mxfp4_gemm(xc, xs, *packed, N, bias=bias, y=guard[:M * N].view(M, N)), h + bias.double())
    assert bool((guard[M * N:] == 7).all())
    _same(Q.mxfp4_gemm(xc, xs, *packed, N, dtype=BF16), h)
    # rows of y on 8 bytes
    _same(Q.mxfp4_gemm(xc, xs, *packed, N, y=guard[4:4 + M * N].view(M, N)), h)
    assert bool((guard[:4] == (h + bias.double()).view(-1)[:4].to(F16)).all())
    # 16-bit activations that quantisation keeps: the largest of a block is 6 times its unit, so its scale is
    # the block's own
    x16 = xv.clone()
    x16[:, ::32] = 6 * torch.exp2(xs.double() - 127)
    _same(Q.mxfp4_linear(x16.to(BF16), *packed, N), _product(x16, wc, ws))
    if N % 32 == 0:
        ws = ws - 8
        packed = Q.mxfp4_pack(wc, ws, gate_up=True)
        _silu(Q.mxfp4_gemm(xc, xs, *packed, N, activation=Q.ACT_SILU_GATE, dtype=BF16), h / 256)
        bias = (bias / 64).to(F16)
        _silu(Q.mxfp4_gemm(xc, xs, *packed, N, bias=bias, activation=Q.ACT_SILU_GATE), h / 256 + bias.double())


# (rows of each expert), columns, channels: every form again, and 512 experts
GROUPED = [([0, 1, 2, 1], 512, 2048), ([1, 0, 1, 3], 520, 1056), ([1, 2, 0, 1], 12320, 2048), ([9, 7, 3, 8], 2080, 4128),
           ([1, 1, 1, 2], 520, 160), ([30, 5, 0, 40], 4096, 2048), ([20, 31, 5, 12], 4112, 4128),
           ([1, 2, 1, 0], 25600, 4096), ([60, 64, 1, 65], 25600, 1056), ([7, 30, 22, 3], 12330, 160),
           ([150, 1, 300, 129], 8192, 512), ([90, 257, 0, 210], 8200, 160), ([400, 260, 1, 300], 12320, 512),
           ([260, 333, 200, 0], 12336, 160), ([500, 1, 900, 513], 12320, 512), ([0] * 200 + [3, 0, 70] + [1] * 309, 48, 544),
           ([350, 350], 96, 2048), ([300, 410], 100, 4128), ([1100, 1000], 512, 4096), ([1500, 600], 520, 4128),
           ([600, 400], 1024, 512), ([512, 488], 2048, 512), ([700, 300], 2056, 160), ([17] * 512, 96, 288)]


@pytest.mark.parametrize("counts,N,K", GROUPED, ids=["E%d_R%d_N%d_K%d" % (len(c), sum(c), n, k) for c, n, k in GROUPED])
def test_grouped_forms(counts, N, K):
    E, R = len(counts), sum(counts)
    T = R // 2 + 3
    g = _gen(2, R, N, K)
    xc, xs = _codes(g, T, K // 2), _scales(g, 127, T, K // 32)
    wc, ws = _codes(g, E, N, K // 2), _scales(g, 127, E, N, K // 32)
    bias = (torch.randint(-64, 65, (E, N), device="cuda", generator=g) / 4).to(BF16)
    rows = torch.randint(0, T, (R,), dtype=torch.int32, device="cuda", generator=g)
    ends = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    o = torch.from_numpy(ends).cuda()
    say("grouped", counts[:6], N, K)
    y = Q.mxfp4_grouped_gemm(xc, xs, o, *Q.mxfp4_pack(wc, ws), N, rows=rows, bias=bias, dtype=BF16)
    if N % 32 == 0:
        z = Q.mxfp4_grouped_gemm(xc, xs, o, *Q.mxfp4_pack(wc, ws - 8, gate_up=True), N, rows=rows,
                                 activation=Q.ACT_SILU_GATE)
    xv = _values(xc, xs)
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        if a == b:
            continue
        h = _product(xv[rows[a:b].long()], wc[e], ws[e])
        _same(y[a:b], h + bias[e].double())
        if N % 32 == 0:
            _silu(z[a:b], h / 256)


@pytest.mark.parametrize("M,N,K", [(1, 57344, 8192), (16, 57344, 8224), (23, 57344, 8192), (64, 57344, 8224),
                                   (130, 57344, 8192)])
def test_dense_weights_past_the_caches(M, N, K):
    g = _gen(3, M, N, K)
    xc, xs, wc, ws = _codes(g, M, K // 2), _scales(g, 127, M, K // 32), _codes(g, N, K // 2), _scales(g, 119, N, K // 32)
    h = _product(_values(xc, xs), wc, ws)
    say("once", M, N, K)
    _same(Q.mxfp4_gemm(xc, xs, *Q.mxfp4_pack(wc, ws), N), h)
    _silu(Q.mxfp4_gemm(xc, xs, *Q.mxfp4_pack(wc, ws, gate_up=True), N, activation=Q.ACT_SILU_GATE), h)


@pytest.mark.parametrize("E,most,N,K", [(8, 2, 28672, 4096), (8, 40, 28672, 4096), (8, 60, 28672, 4128),
                                        (8, 120, 28672, 4096), (40, 3, 28672, 8192)])
def test_grouped_weights_past_the_caches(E, most, N, K):
    """Also with more than 2^32 bytes of weights."""
    g = _gen(4, E, most)
    counts = np.random.Generator(np.random.PCG64(most)).integers(0, most + 1, E)
    counts[-1] = most
    ends = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    R = int(ends[-1])
    xc, xs = _codes(g, R, K // 2), _scales(g, 127, R, K // 32)
    wc, ws = _codes(g, E, N, K // 2), _scales(g, 119, E, N, K // 32)
    o = torch.from_numpy(ends).cuda()
    say("once, grouped", E, R, N, K)
    y = Q.mxfp4_grouped_gemm(xc, xs, o, *Q.mxfp4_pack(wc, ws), N)
    z = Q.mxfp4_grouped_gemm(xc, xs, o, *Q.mxfp4_pack(wc, ws, gate_up=True), N, activation=Q.ACT_SILU_GATE)
    for e in [e for e in range(E) if counts[e]][-6:]:
        a, b = ends[e], ends[e + 1]
        h = _product(_values(xc[a:b], xs[a:b]), wc[e], ws[e])
        _same(y[a:b], h)
        _silu(z[a:b], h)


def _some_rows(M):
    g = np.random.Generator(np.random.PCG64(M))
    return torch.from_numpy(np.concatenate([[0, 1, M // 2, M - 2, M - 1], g.integers(0, M, 59)])).cuda()


def test_more_than_2_31_results():
    M, N, K = 70001, 32784, 64
    g = _gen(5)
    xc, xs, wc, ws = _codes(g, M, K // 2), _scales(g, 127, M, K // 32), _codes(g, N, K // 2), _scales(g, 127, N, K // 32)
    say("2^31 results")
    y = Q.mxfp4_gemm(xc, xs, *Q.mxfp4_pack(wc, ws), N)
    r = _some_rows(M)
    _same(y[r], _product(_values(xc[r], xs[r]), wc, ws))


def test_more_than_2_31_bytes_of_activations():
    M, N, K = 600011, 48, 8192
    g = _gen(6)
    xc, xs, wc, ws = _codes(g, M, K // 2), _scales(g, 127, M, K // 32), _codes(g, N, K // 2), _scales(g, 127, N, K // 32)
    packed = Q.mxfp4_pack(wc, ws)
    say("2^31 bytes of codes")
    y = Q.mxfp4_gemm(xc, xs, *packed, N)
    r = _some_rows(M)
    h = _product(_values(xc[r], xs[r]), wc, ws)
    _same(y[r], h)
    z = Q.mxfp4_grouped_gemm(xc, xs, torch.tensor([0, 64], dtype=torch.int32, device="cuda"), *packed, N,
                             rows=r.int())
    _same(z, h)


def test_quantize_more_than_2_31_values():
    M, K = 280003, 8192
    x = torch.empty((M, K), dtype=BF16, device="cuda").normal_(generator=_gen(7))
    say("quantize 2^31 values")
    codes, scales = Q.mxfp4_quantize(x)
    r = _some_rows(M)
    rc, rs = U.quantize(x[r].double().cpu().numpy())
    assert np.array_equal(codes[r].cpu().numpy(), rc) and np.array_equal(scales[r].cpu().numpy(), rs)
    back = Q.mxfp4_dequantize(codes, scales, dtype=BF16)
    assert torch.equal(back[r].double(), _values(codes[r], scales[r]))


def test_route_and_combine_past_32_bits():
    T, E, k = (1 << 22) + 1000, 512, 2
    x = torch.empty((T, E), dtype=F16, device="cuda").normal_(generator=_gen(8))
    say("route 2^31 logits")
    q = Q.moe_route(x, k)
    r = _some_rows(T)
    ids, w, _ = U.route(x[r].double().cpu().numpy(), k)
    assert np.array_equal(q.ids[r].cpu().numpy(), ids)
    assert np.abs(q.weights[r].double().cpu().numpy() - w).max() <= 530 * 2.0 ** -24
    flat = q.ids.view(-1).long()
    assert torch.equal(q.offsets[1:].long(), torch.bincount(flat, minlength=E).cumsum(0)) and int(q.offsets[0]) == 0
    order = torch.sort(flat, stable=True).indices
    assert torch.equal(q.rows.long(), order // k)
    assert torch.equal(q.slots.view(-1)[order].long(), torch.arange(T * k, device="cuda"))
    del x, q, flat, order
    T, D, k = 40009, 8192, 8
    y = torch.empty((T * k, D), dtype=BF16, device="cuda").normal_(generator=_gen(9))
    slots = torch.randperm(T * k, device="cuda", generator=_gen(10)).int().view(T, k)
    w = torch.rand((T, k), device="cuda", generator=_gen(11))
    say("combine 2^31 values")
    out = Q.moe_combine(y, slots, w)
    r = _some_rows(T)
    p = y[slots[r].long()].double() * w[r].double()[:, :, None]
    ref = p.sum(1)
    tol = EPS[BF16] * 1.001 * ref.abs() + (k + 1) * 2.0 ** -23 * p.abs().sum(1)
    assert bool(((out[r].double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [F16, BF16, torch.float32])
@pytest.mark.parametrize("E,topk,groups,topk_groups,best",
                         [(512, 16, 1, 1, 1), (512, 8, 64, 5, 2), (384, 8, 1, 1, 1), (320, 5, 4, 2, 2), (256, 8, 64, 9, 2),
                          (256, 4, 4, 1, 2), (128, 16, 1, 1, 1), (96, 3, 32, 2, 1), (12, 12, 1, 1, 1), (24, 2, 2, 1, 1)])
def test_route_widths(E, topk, groups, topk_groups, best, dtype):
    """Every width of a lane and of a token, and enough tokens for several
    workgroups of the sort; distinct logits, so that the choice is one."""
    T = 1203
    g = np.random.Generator(np.random.PCG64([E, topk, groups]))
    x = np.stack([g.permutation(E) for _ in range(T)]) / 64.0 - 2
    t = torch.from_numpy(x).to(dtype).cuda()
    assert torch.equal(t.double().cpu(), torch.from_numpy(x)) or dtype == BF16
    xv = t.double().cpu().numpy()
    kw = dict(groups=groups, topk_groups=topk_groups, group_best=best)
    say("route", E, topk, kw, dtype)
    r = Q.moe_route(t, topk, **kw)
    ids, w, c = U.route(xv, topk, **kw)
    got = r.ids.cpu().numpy()
    same = (got == ids).all(1)
    if not (groups > 1 and best > 1):
        assert same.all()                  # the logits themselves are compared, ties go by index
    else:
        # sums of two scores that binary32 may round to the same value
        a, b = np.take_along_axis(c, got.astype(np.int64), 1), np.take_along_axis(c, ids, 1)
        assert same.mean() > 0.98 and np.abs(a - b).max() <= 1 and all(len(set(v)) == topk for v in got)
    gw = r.weights.double().cpu().numpy()
    assert np.abs(gw - w)[same].max() <= 530 * 2.0 ** -24
    offsets, rows, slots = U.sort_rows(got.astype(np.int64), E)
    assert np.array_equal(r.offsets.cpu().numpy(), offsets) and np.array_equal(r.rows.cpu().numpy(), rows)
    assert np.array_equal(r.slots.cpu().numpy(), slots)
