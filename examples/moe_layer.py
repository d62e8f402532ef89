"""A mixture-of-experts feed-forward layer with a shared expert, from router
logits to the residual, in microscaled 4-bit floating point or in 4-bit
integers (QUICK's weights).

    python examples/moe_layer.py                      # the sizes of a Mixtral-8x7B layer, 1 to 2048 tokens
    python examples/moe_layer.py --weights int4 --tokens 1,64

Seven calls of the library do a layer's work (six with integer weights, which
take 16-bit activations as they are); nothing is copied to the host between
them, so a layer can be captured in a graph.  Weights and activations are
random.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2402_10076_amd as Q  # noqa: E402


class MxMoe:
    """out = x + shared(x) + sum over a token's topk experts of w_e expert_e(x).

    router [E][D], gate_up [E][2F][D], down [E][D][F]; shared: (gate_up [2S][D],
    down [D][S]) or None: 16-bit tensors, quantised here once."""

    def __init__(self, router, gate_up, down, topk, shared=None, **routing):
        self.router, self.topk, self.routing = router, topk, routing
        self.N1, self.D = gate_up.shape[-2], down.shape[-2]
        self.w13, self.w2 = self._pack(gate_up, True), self._pack(down, False)
        self.shared = shared and (shared[0].shape[0], self._pack(shared[0], True), self._pack(shared[1], False))

    @staticmethod
    def _pack(w, gate_up):
        codes, scales = Q.mxfp4_quantize(w.reshape(-1, w.shape[-1]))
        return Q.mxfp4_pack(codes.view(*w.shape[:-1], -1), scales.view(*w.shape[:-1], -1), gate_up=gate_up)

    def __call__(self, x):
        r = Q.moe_route(x @ self.router.t(), self.topk, **self.routing)
        h = Q.mxfp4_grouped_gemm(*Q.mxfp4_quantize(x), r.offsets, *self.w13, self.N1, rows=r.rows,
                                 activation=Q.ACT_SILU_GATE, dtype=x.dtype)
        y = Q.mxfp4_grouped_gemm(*Q.mxfp4_quantize(h), r.offsets, *self.w2, self.D, dtype=x.dtype)
        if self.shared:
            n, w13, w2 = self.shared
            x = x + Q.mxfp4_linear(Q.mxfp4_linear(x, *w13, n, activation=Q.ACT_SILU_GATE), *w2, self.D)
        return Q.moe_combine(y, r.slots, r.weights, residual=x)


class Int4Moe:
    """The same with the experts' weights (q, z, s) of [K][N] in QUICK's form:
    w13[e] columns gate then up, w2[e]; fp16 activations."""

    def __init__(self, router, w13, w2, topk, **routing):
        self.router, self.topk, self.routing = router, topk, routing
        self.N1, self.D = w13[0][0].shape[1], w2[0][0].shape[1]
        n = self.N1 // 2
        halves = [([a[:, :n] for a in w], [a[:, n:] for a in w]) for w in w13]
        self.w13 = Q.to_device(*Q.pack_experts([Q.interleave_gate_up(*h) for h in halves]))
        self.w2 = Q.to_device(*Q.pack_experts(w2))

    def __call__(self, x):
        r = Q.moe_route(x @ self.router.t(), self.topk, **self.routing)
        h = Q.grouped_gemm_fused(x, r.offsets, *self.w13, self.N1, rows=r.rows, activation=Q.ACT_SILU_GATE)
        return Q.moe_combine(Q.grouped_gemm(h, r.offsets, *self.w2, self.D), r.slots, r.weights, residual=x)


def random_mx(D, F, E, topk, shared=0, dtype=torch.bfloat16, seed=0, **routing):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def mat(*shape):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(std=shape[-1] ** -0.5, generator=g)
    return MxMoe(mat(E, D), mat(E, 2 * F, D), mat(E, D, F), topk,
                 (mat(2 * shared, D), mat(D, shared)) if shared else None, **routing)


def random_int4(D, F, E, topk, seed=0, **routing):
    import numpy as np
    g = np.random.Generator(np.random.PCG64(seed))

    def mat(K, N):
        return (g.integers(0, 16, (K, N), dtype=np.uint8), g.integers(0, 16, (K // 128, N), dtype=np.uint8),
                g.uniform(0.002, 0.004, (K // 128, N)).astype(np.float16).view(np.uint16))
    router = torch.from_numpy(g.standard_normal((E, D)).astype(np.float32) * D ** -0.5).half().cuda()
    return Int4Moe(router, [mat(D, 2 * F) for _ in range(E)], [mat(F, D) for _ in range(E)], topk, **routing)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--weights", choices=("mxfp4", "int4"), default="mxfp4")
    p.add_argument("--tokens", default="1,20,256,2048")
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--ffn", type=int, default=14336)
    p.add_argument("--experts", type=int, default=8)
    p.add_argument("--topk", type=int, default=2)
    p.add_argument("--shared", type=int, default=0, help="columns of a shared expert (mxfp4)")
    p.add_argument("--steps", type=int, default=20)
    a = p.parse_args()
    if a.weights == "mxfp4":
        layer, dtype = random_mx(a.hidden, a.ffn, a.experts, a.topk, a.shared), torch.bfloat16
    else:
        layer, dtype = random_int4(a.hidden, a.ffn, a.experts, a.topk), torch.float16
    for T in map(int, a.tokens.split(",")):
        x = torch.randn((T, a.hidden), device="cuda").to(dtype)
        layer(x)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):        # the integer products keep a workspace for each stream
            layer(x)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = layer(x)
        times = []
        for run in (lambda: layer(x), graph.replay):
            for _ in range(3):
                run()
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(a.steps):
                run()
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end) * 1e3 / a.steps)
        print("%5d tokens: %8.1f us a layer, %8.1f us replayed, largest |out| %.3g"
              % (T, *times, out.abs().max().item()), flush=True)


if __name__ == "__main__":
    main()
