"""The example's layers against plain forms in binary64, and replayed."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import mx_util as U
import paper_2402_10076_amd as Q

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")
    spec = importlib.util.spec_from_file_location("moe_layer", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _kept(w):
    """Binary64 values of w after its quantisation."""
    return U.values(*U.quantize(w.double().cpu().numpy().reshape(-1, w.shape[-1]))).reshape(w.shape)


def _replays(layer, x, ref):
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):            # the integer products keep a workspace for each stream
        layer(x)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = layer(x)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(layer(x), ref)


@pytest.mark.parametrize("T", [1, 7, 50, 400])
@pytest.mark.parametrize("routing", [{}, {"score": Q.SCORE_SIGMOID, "groups": 2, "topk_groups": 1, "scale": 2.0}])
def test_microscaled_layer(T, routing):
    """Each expert's hidden values are rounded to 16 and then to 4 bits, on
    both sides; a hidden value at the edge of two codes may fall to either (a
    step of a quarter of the block's largest), which a token's sum of F = 160
    products dilutes: 5 % of the largest |out - x|."""
    D, F, E, k, S = 128, 160, 8, 2, 96
    g = torch.Generator(device="cuda")
    g.manual_seed(T)

    def mat(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(std=shape[-1] ** -0.5, generator=g)
    router, w13, w2, s13, s2 = mat(E, D), mat(E, 2 * F, D), mat(E, D, F), mat(2 * S, D), mat(D, S)
    x = mat(T, D) * 8
    layer = _example().MxMoe(router, w13, w2, k, (s13, s2), **routing)
    out = layer(x)
    xv = x.double().cpu().numpy()
    opts = dict(routing)
    ids, w, _ = U.route((x @ router.t()).double().cpu().numpy(), k, sigmoid=bool(opts.pop("score", 0)), **opts)
    xq = U.values(*U.quantize(xv))

    def expert(rows, a, b):
        h = torch.from_numpy(U.silu_gate(rows @ a.T)).to(torch.bfloat16).double().numpy()
        return U.values(*U.quantize(h)) @ b.T
    ref = expert(xq, _kept(s13), _kept(s2))
    v13, v2 = _kept(w13), _kept(w2)
    for e in range(E):
        t, j = np.nonzero(ids == e)
        if len(t):
            np.add.at(ref, t, w[t, j][:, None] * expert(xq[t], v13[e], v2[e]))
    got = out.double().cpu().numpy() - xv
    # out is rounded to bfloat16 beside x
    assert np.abs(got - ref).max() <= 0.05 * np.abs(ref).max() + 2.0 ** -7 * np.abs(xv).max()
    _replays(layer, x, out)


@pytest.mark.parametrize("T", [1, 130])
def test_integer_layer(T):
    import oracle
    D, F, E, k = 256, 128, 4, 2
    g = np.random.Generator(np.random.PCG64(T))

    def mat(K, N):
        return (g.integers(0, 16, (K, N), dtype=np.uint8), g.integers(0, 16, (K // 128, N), dtype=np.uint8),
                g.uniform(0.002, 0.01, (K // 128, N)).astype(np.float16).view(np.uint16))
    w13, w2 = [mat(D, 2 * F) for _ in range(E)], [mat(F, D) for _ in range(E)]
    router = torch.from_numpy(g.standard_normal((E, D)).astype(np.float32) / 16).half().cuda()
    x = torch.from_numpy(g.standard_normal((T, D)).astype(np.float32)).half().cuda()
    layer = _example().Int4Moe(router, w13, w2, k)
    out = layer(x)
    ids, w, _ = U.route((x @ router.t()).double().cpu().numpy(), k)
    xb = x.cpu().view(torch.int16).numpy().view(np.uint16)
    ref = x.double().cpu().numpy()
    for e in range(E):
        t, j = np.nonzero(ids == e)
        if len(t):
            h = U.silu_gate(oracle.gemm(np.ascontiguousarray(xb[t]), *w13[e])).astype(np.float16).view(np.uint16)
            np.add.at(ref, t, w[t, j][:, None] * oracle.gemm(h, *w2[e]))
    err = np.abs(out.double().cpu().numpy() - ref).max() / np.abs(ref).max()
    assert err <= 5e-3
    _replays(layer, x, out)
