"""Expert routing and combining (include/quick_moe.h) on the GPU through the C
ABI against binary64 forms, and the whole mixture-of-experts layer."""
import numpy as np
import pytest
import torch

import mx_util as U
import paper_2402_10076_amd as Q
from gpu_util import say

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# binary32 exponentials, sums of up to 512 and divisions: 2^-24 for each step
# of a sum, a few units in the last place for the others
W_TOL = 530 * 2.0 ** -24


def _rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _typed(v, dtype):
    t = torch.from_numpy(np.asarray(v, np.float32)).to(dtype)
    return t.cuda(), t.double().numpy()


def _check_sorted(r, ids, E):
    offsets, rows, slots = U.sort_rows(ids, E)
    assert np.array_equal(r.offsets.cpu().numpy(), offsets)
    assert np.array_equal(r.rows.cpu().numpy(), rows)
    assert np.array_equal(r.slots.cpu().numpy(), slots)


def _check(r, logits, topk, E, gap=None, **kw):
    """ids exactly, but where two choices of a row are nearer than `gap` of
    each other (scores computed in binary32): there the choice has to be as
    good, and the rest of the row is taken from it."""
    ids, w, c = U.route(logits, topk, **kw)
    got = r.ids.cpu().numpy().astype(np.int64)
    gw = r.weights.double().cpu().numpy()
    assert got.min() >= 0 and got.max() < E
    assert all(len(set(row)) == topk for row in got)
    same = (got == ids).all(1)
    if gap is None:
        assert same.all(), "%d rows differ" % int((~same).sum())
    else:
        a, b = np.take_along_axis(c, got, 1), np.take_along_axis(c, ids, 1)
        assert np.abs(a - b)[~same].max(initial=0) <= gap
        assert (~same).mean() <= 0.01
    fine = same[:, None] & np.ones_like(w, bool)
    assert np.array_equal(np.isnan(gw[fine]), np.isnan(w[fine]))
    ok = fine & ~np.isnan(w)
    assert np.all(np.abs(gw - w)[ok] <= W_TOL * np.abs(w[ok]) + 1e-37)
    _check_sorted(r, got, E)


CASES = [(1, 1, 1), (1, 8, 2), (5, 8, 8), (20, 16, 4), (67, 17, 3), (64, 32, 16), (65, 33, 2), (3, 64, 6),
         (100, 100, 8), (130, 160, 6), (16, 256, 8), (17, 256, 8), (300, 512, 10), (1000, 8, 2), (4097, 64, 4),
         (9000, 384, 8)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,E,topk", CASES)
def test_softmax(T, E, topk, dtype):
    """Logits in 16 bits have equal values in a row: ties go to the lower index."""
    x, xv = _typed(_rng(1, T, E).standard_normal((T, E)) * 2, TYPES[dtype])
    say("softmax", T, E, topk, dtype)
    for renorm in (True, False):
        _check(Q.moe_route(x, topk, renormalize=renorm, scale=1.5), xv, topk, E, renormalize=renorm, scale=1.5)


@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("T,E,topk,groups,topk_groups,best",
                         [(1, 8, 2, 1, 1, 1), (33, 16, 4, 4, 2, 1), (50, 60, 5, 6, 2, 2), (40, 64, 3, 64, 7, 2),
                          (129, 256, 8, 8, 4, 2), (700, 256, 8, 8, 3, 1), (2500, 160, 6, 8, 3, 2), (60, 512, 16, 2, 1, 2),
                          (90, 30, 4, 3, 1, 1), (11, 9, 2, 3, 2, 2)])
@pytest.mark.parametrize("sigmoid", [True, False])
def test_groups_and_bias(T, E, topk, groups, topk_groups, best, sigmoid, with_bias):
    g = _rng(2, T, E, groups)
    x, xv = _typed(g.standard_normal((T, E)) * 1.5, torch.float32)
    bias, bv = _typed(g.uniform(-0.1, 0.1, E), torch.float32)
    kw = dict(groups=groups, topk_groups=topk_groups, group_best=best)
    say("groups", T, E, topk, kw, sigmoid, with_bias)
    r = Q.moe_route(x, topk, score=Q.SCORE_SIGMOID if sigmoid else Q.SCORE_SOFTMAX, bias=bias if with_bias else None,
                    **kw)
    # scores to 2^-23 each plus the rounding of the sums
    _check(r, xv, topk, E, gap=W_TOL, sigmoid=sigmoid, bias=bv if with_bias else None, **kw)


def test_all_logits_equal_and_masked():
    """Equal logits go by index; masked experts (-inf) are chosen last and have
    weight 0, also where a row has nothing else."""
    E, k = 40, 6
    x = np.zeros((7, E), np.float32)
    x[1, :] = -np.inf
    x[2, 5:] = -np.inf                       # five experts are left for six choices
    x[3, :] = -np.inf
    x[3, 39] = -80
    x[4, ::2] = -np.inf
    x[5, 3] = np.finfo(np.float32).min       # the type's lowest value is a value
    x[6, :] = np.finfo(np.float32).min
    for sigmoid in (False, True):
        for renorm in (True, False):
            r = Q.moe_route(_dev(x), k, score=int(sigmoid), renormalize=renorm)
            _check(r, x.astype(np.float64), k, E, sigmoid=sigmoid, renormalize=renorm)
            assert bool((r.weights[1] == 0).all()) and bool(torch.isfinite(r.weights).all())


def test_nan_and_infinite_logits():
    """A NaN is chosen last, and the weights are what the formula gives: ids
    and the sorted order stay within bounds."""
    E, k = 20, 3
    x = _rng(3).standard_normal((6, E)).astype(np.float32)
    x[1, 4] = np.nan
    x[2, :] = np.nan
    x[3, 7] = np.inf
    x[4, 0] = -np.inf
    r = Q.moe_route(_dev(x), k)
    _check(r, x.astype(np.float64), k, E)
    assert bool(torch.isnan(r.weights[1]).all()) and bool(torch.isnan(r.weights[2]).all())
    assert bool(torch.isfinite(r.weights[0]).all()) and bool(torch.isfinite(r.weights[5]).all())
    r = Q.moe_route(_dev(x), k, score=Q.SCORE_SIGMOID, groups=4, topk_groups=2, group_best=2)
    _check(r, x.astype(np.float64), k, E, sigmoid=True, groups=4, topk_groups=2, group_best=2)


def test_bias_disables_an_expert():
    x, xv = _typed(_rng(4).standard_normal((50, 32)), torch.float32)
    bias = np.zeros(32, np.float32)
    bias[3] = -np.inf
    r = Q.moe_route(x, 16, bias=_dev(bias))
    assert not bool((r.ids == 3).any())


def test_every_token_at_one_expert():
    """All rows at one expert, the first and the last one."""
    for E, T in ((8, 3000), (256, 3000), (512, 40)):
        for e in (0, E - 1):
            x = torch.zeros((T, E), device="cuda")
            x[:, e] = 5
            r = Q.moe_route(x, 1)
            _check_sorted(r, np.full((T, 1), e), E)


def test_no_tokens():
    r = Q.moe_route(torch.zeros((0, 8), device="cuda"), 2)
    assert r.ids.shape == (0, 2) and r.rows.shape == (0,) and r.offsets.tolist() == [0] * 9


def test_given_outputs_workspace_and_replay():
    T, E, k = 777, 64, 4
    x, xv = _typed(_rng(5).standard_normal((T, E)), torch.float16)
    ref = Q.moe_route(x, k)
    out = Q.Routing(*(torch.full_like(t, -1) for t in ref))
    work = torch.full((Q.moe_route_workspace_bytes(T, E, k) + 16,), 0x7F, dtype=torch.uint8, device="cuda")
    assert work.numel() > 16
    Q.moe_route(x, k, out=out, workspace=work)
    assert all(torch.equal(a, b) for a, b in zip(out, ref)) and bool((work[-16:] == 0x7F).all())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        Q.moe_route(x, k, out=out, workspace=work)
    for _ in range(3):
        for t in out:
            t.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
        assert all(torch.equal(a, b) for a, b in zip(Q.moe_route(x, k), ref))


# ---------------------------------------------------------------------------
# combine
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,D,topk", [(1, 1, 1), (1, 4096, 2), (3, 7, 3), (20, 1000, 2), (33, 2056, 8), (5, 513, 16),
                                      (300, 264, 5), (70, 8192, 9)])
def test_combine(T, D, topk, dtype):
    g = _rng(6, T, D, topk)
    R = T * topk
    y, yv = _typed(g.standard_normal((R, D)), dtype)
    res, rv = _typed(g.standard_normal((T, D)), dtype)
    slots = g.permutation(R).reshape(T, topk).astype(np.int32)
    w, wv = _typed(g.uniform(-1, 1, (T, topk)), torch.float32)
    ref = (yv[slots] * wv[:, :, None]).sum(1)
    size = (np.abs(yv[slots]) * np.abs(wv)[:, :, None]).sum(1)
    eps = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8
    say("combine", T, D, topk, dtype)
    for residual, more in ((None, 0), (res, rv)):
        out = Q.moe_combine(y, _dev(slots), w, residual=residual)
        err = np.abs(out.double().cpu().numpy() - (ref + more))
        tol = eps * 1.001 * np.abs(ref + more) + (topk + 1) * 2.0 ** -23 * (size + np.abs(more)) + 2.0 ** -25
        assert np.all(err <= tol)
    # in place of the residual
    again = res.clone()
    Q.moe_combine(y, _dev(slots), w, residual=again, out=again)
    assert torch.equal(again, out)


def test_combine_leaves_out_slots_outside():
    """A slot below 0 or past y adds nothing, whatever its weight; one that is
    used passes its NaN on."""
    y, yv = _typed(_rng(7).standard_normal((6, 40)), torch.float16)
    y[5] = float("nan")
    slots = _dev(np.array([[0, -1], [6, 1], [-(1 << 31), (1 << 31) - 1], [5, 2]], np.int32))
    w = torch.tensor([[1.0, float("nan")], [float("inf"), 1.0], [2.0, 3.0], [1.0, 1.0]], device="cuda")
    out = Q.moe_combine(y, slots, w)
    assert torch.equal(out[0], y[0]) and torch.equal(out[1], y[1]) and bool((out[2] == 0).all())
    assert bool(torch.isnan(out[3]).all())


def test_combine_addresses_that_are_not_on_16_bytes():
    T, D, k = 9, 64, 2
    flat = torch.randn(T * k * D + 8, device="cuda").half()
    slots = torch.arange(T * k, dtype=torch.int32, device="cuda").view(T, k)
    w = torch.rand(T, k, device="cuda")
    y = flat[:T * k * D].view(T * k, D)
    ref = Q.moe_combine(y, slots, w)
    off = torch.empty_like(flat)
    off[1:T * k * D + 1] = y.reshape(-1)
    assert torch.equal(Q.moe_combine(off[1:T * k * D + 1].view(T * k, D), slots, w), ref)


def test_combine_empty():
    y = torch.zeros((0, 16), dtype=torch.float16, device="cuda")
    none = torch.zeros((0, 2), dtype=torch.int32, device="cuda")
    assert Q.moe_combine(y, none, none.float()).shape == (0, 16)
    # no rows at all, but tokens
    slots = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    assert bool((Q.moe_combine(y, slots, torch.ones((3, 2), device="cuda")) == 0).all())


# ---------------------------------------------------------------------------
# the layer
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("T", [1, 40, 300])
def test_layer_with_integer_weights(T):
    """Routing, the W4A16 grouped products and combining as one layer, against
    binary64 token by token."""
    import oracle
    D, F, E, k = 256, 128, 6, 2
    g = _rng(8, T)

    def mat(K, N):
        return (g.integers(0, 16, (K, N), dtype=np.uint8), g.integers(0, 16, (K // 128, N), dtype=np.uint8),
                g.uniform(0.002, 0.01, (K // 128, N)).astype(np.float16).view(np.uint16))
    w13 = [Q.interleave_gate_up(mat(D, F), mat(D, F)) for _ in range(E)]
    w2 = [mat(F, D) for _ in range(E)]
    x, xv = _typed(g.standard_normal((T, D)), torch.float16)
    logits, lv = _typed(g.standard_normal((T, E)), torch.float16)
    d13, d2 = (Q.to_device(*Q.pack_experts(w)) for w in (w13, w2))
    r = Q.moe_route(logits, k)
    h = Q.grouped_gemm_fused(x, r.offsets, *d13, 2 * F, rows=r.rows, activation=Q.ACT_SILU_GATE)
    out = Q.moe_combine(Q.grouped_gemm(h, r.offsets, *d2, D), r.slots, r.weights, residual=x)
    ids, w, _ = U.route(lv, k)
    xb = x.cpu().view(torch.int16).numpy().view(np.uint16)
    ref = xv.copy()
    for e in range(E):
        t, j = np.nonzero(ids == e)
        if len(t) == 0:
            continue
        he = oracle.epilogue(oracle.gemm(np.ascontiguousarray(xb[t]), *w13[e]), None, act=1)
        hb = he.astype(np.float16).view(np.uint16)
        np.add.at(ref, t, w[t, j][:, None] * oracle.gemm(hb, *w2[e]))
    err = np.abs(out.double().cpu().numpy() - ref).max() / np.abs(ref).max()
    say("layer T=%d err %.3g" % (T, err))
    assert err <= 5e-3


@pytest.mark.parametrize("T", [1, 40, 300])
def test_layer_with_microscaled_weights(T):
    """The same with microscaled weights and activations: the library's own
    quantised activations of the second product are the reference's input
    there, since one unit of h's last place may change a code."""
    D, F, E, k = 256, 160, 6, 2
    g = _rng(9, T)
    x, xv = _typed(g.standard_normal((T, D)), torch.bfloat16)
    logits, lv = _typed(g.standard_normal((T, E)), torch.float32)
    w13 = Q.mxfp4_quantize(_typed(g.standard_normal((E * 2 * F, D)) * 0.05, torch.bfloat16)[0])
    w2 = Q.mxfp4_quantize(_typed(g.standard_normal((E * D, F)) * 0.05, torch.bfloat16)[0])
    p13 = Q.mxfp4_pack(w13[0].view(E, 2 * F, -1), w13[1].view(E, 2 * F, -1), gate_up=True)
    p2 = Q.mxfp4_pack(w2[0].view(E, D, -1), w2[1].view(E, D, -1))
    r = Q.moe_route(logits, k, score=Q.SCORE_SIGMOID)
    h = Q.mxfp4_grouped_gemm(*Q.mxfp4_quantize(x), r.offsets, *p13, 2 * F, rows=r.rows, activation=Q.ACT_SILU_GATE,
                             dtype=torch.bfloat16)
    hq = Q.mxfp4_quantize(h)
    out = Q.moe_combine(Q.mxfp4_grouped_gemm(*hq, r.offsets, *p2, D, dtype=torch.bfloat16), r.slots, r.weights,
                        residual=x)
    ids, w, _ = U.route(lv, k, sigmoid=True)
    xq = U.values(*U.quantize(xv))
    v13 = U.values(w13[0].cpu().numpy(), w13[1].cpu().numpy()).reshape(E, 2 * F, D)
    v2 = U.values(w2[0].cpu().numpy(), w2[1].cpu().numpy()).reshape(E, D, F)
    hv, hqv = h.double().cpu().numpy(), U.values(hq[0].cpu().numpy(), hq[1].cpu().numpy())
    slots = r.slots.cpu().numpy()
    ref = xv.copy()
    for t in range(T):
        for j in range(k):
            e = ids[t, j]
            he = U.silu_gate(v13[e] @ xq[t])
            assert np.abs(hv[slots[t, j]] - he).max() <= 2.0 ** -7 * np.abs(he).max()
            ref[t] += w[t, j] * (v2[e] @ hqv[slots[t, j]])
    err = np.abs(out.double().cpu().numpy() - ref).max() / np.abs(ref).max()
    say("layer T=%d err %.3g" % (T, err))
    assert err <= 2.0 ** -7
