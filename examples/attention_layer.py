"""An attention layer of a served model with 4-bit weights, a 4-bit cache and
the low-rank adapters of its requests: from the normed hidden states to the
output projection, prompts first, then single tokens.

    python examples/attention_layer.py                     # the sizes of a Llama-2-7B layer
    python examples/attention_layer.py --kv-heads 8 --batch 64 --context 8000

Nothing is copied to the host between the calls, so a decode step can be
captured in a graph; the table's rows are as long as the longest sequence may
get.  Weights and activations are random.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2402_10076_amd as Q  # noqa: E402


class Attention:
    """qkv and o: (q, z, s) of [K][N] in QUICK's form, the qkv columns those of
    the query heads, then of the key and of the value heads; adapters: (a
    [E][rank][D_model], b [E][(HQ + 2 H) * D][rank], scales f32 [E]) or None."""

    def __init__(self, qkv, o, heads, kv_heads, dim, pages, adapters=None, **frequencies):
        self.HQ, self.H, self.D = heads, kv_heads, dim
        self.N, self.NO = qkv[0].shape[1], o[0].shape[1]
        self.qkv, self.o = (Q.to_device(*Q.pack_weights(*w)) for w in (qkv, o))
        self.adapters = adapters
        self.freqs, self.factor = Q.rotary_frequencies(dim, **frequencies)
        self.cache = Q.kv4_cache(pages, kv_heads, dim)

    def __call__(self, x, positions, slots, table, lengths, offsets=None, most=None, group=None):
        """x [T][D_model]; positions, slots [T] of the tokens; table, lengths
        (with the new tokens), offsets and most as in kv4_attention; group: the
        tokens' adapters in order (lora_group)."""
        T, HQ, H, D = x.shape[0], self.HQ, self.H, self.D
        qkv = Q.w4a16_gemm(x, *self.qkv, self.N)
        if self.adapters and group:
            a, b, scales = self.adapters
            Q.lora_add(qkv, x, a, b, *group, scales=scales, out=qkv)
        heads = qkv.view(T, HQ + 2 * H, D)
        turned = heads[:, :HQ + H]
        Q.rotary(turned, positions, self.freqs, factor=self.factor, out=turned)
        Q.kv4_write(self.cache, heads[:, HQ:HQ + H], heads[:, HQ + H:], slots)
        y = Q.kv4_attention(heads[:, :HQ], self.cache, table, lengths, offsets=offsets, most=most)
        return Q.w4a16_gemm(y.view(T, HQ * D), *self.o, self.NO)


def random_weights(g, K, N):
    return (g.integers(0, 16, (K, N), dtype=np.uint8), g.integers(0, 16, (K // 128, N), dtype=np.uint8),
            g.uniform(0.5, 1.0, (K // 128, N)).astype(np.float16) * np.float16(0.15 * K ** -0.5))


def random_layer(hidden, heads, kv_heads, dim, pages, adapters=0, rank=16, seed=0, **frequencies):
    g = np.random.Generator(np.random.PCG64(seed))
    n = (heads + 2 * kv_heads) * dim

    def bits(w):
        return w[0], w[1], w[2].view(np.uint16)

    def mat(*shape, std):
        return torch.from_numpy((g.standard_normal(shape) * std).astype(np.float16)).cuda()
    lora = adapters and (mat(adapters, rank, hidden, std=hidden ** -0.5), mat(adapters, n, rank, std=0.3 * rank ** -0.5),
                         torch.from_numpy(g.uniform(0.5, 1.5, adapters).astype(np.float32)).cuda())
    return Attention(bits(random_weights(g, hidden, n)), bits(random_weights(g, heads * dim, hidden)), heads, kv_heads, dim,
                     pages, lora or None, **frequencies)


def batch(lengths, new, width=None, pages=None, seed=0):
    """(positions, slots, table, lengths, offsets) of sequences with so many
    tokens, the last `new` of each being the call's, on shuffled pages."""
    need = [-(-n // Q.KV4_PAGE) for n in lengths]
    ids = torch.randperm(pages or sum(need), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.zeros((len(lengths), width or max(need)), dtype=torch.int32)
    at, offsets, positions, slots = 0, [0], [], []
    for b, n in enumerate(lengths):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
        p = torch.arange(n - new[b], n)
        positions.append(p)
        slots.append(table[b, p // Q.KV4_PAGE].long() * Q.KV4_PAGE + p % Q.KV4_PAGE)
        offsets.append(offsets[-1] + new[b])

    def dev(t):
        return t.to(torch.int32).cuda()
    return dev(torch.cat(positions)), dev(torch.cat(slots)), dev(table), dev(torch.tensor(lengths)), dev(torch.tensor(offsets))


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--heads", type=int, default=32)
    p.add_argument("--kv-heads", type=int, default=32)
    p.add_argument("--dim", type=int, default=128)
    p.add_argument("--batch", type=int, default=16)
    p.add_argument("--context", type=int, default=2000)
    p.add_argument("--adapters", type=int, default=4)
    p.add_argument("--steps", type=int, default=20)
    a = p.parse_args()
    lengths = [max(1, a.context * (i + 1) // a.batch) for i in range(a.batch)]
    pages = sum(-(-(n + 1) // Q.KV4_PAGE) for n in lengths)
    layer = random_layer(a.hidden, a.heads, a.kv_heads, a.dim, pages, a.adapters)
    E = max(1, a.adapters)

    def run(name, lengths, new, capture):
        pos, slots, table, ln, off = batch(lengths, new, pages=pages)
        seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new))
        group = Q.lora_group((seq % (E + 1) - 1).to(torch.int32).cuda(), E) if a.adapters else None
        x = torch.randn((sum(new), a.hidden), device="cuda").half()
        single = max(new) == 1

        def step():
            return layer(x, pos, slots, table, ln, None if single else off, max(new), group)
        step()
        runs = [("eager", step)]
        if capture:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):        # the integer products keep a workspace for each stream
                step()
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = step()
            runs.append(("replayed", graph.replay))
        for kind, f in runs:
            for _ in range(3):
                f()
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(a.steps):
                f()
            end.record()
            end.synchronize()
            print("%-8s %6d new tokens, %8d in the cache, %-8s %9.1f us a layer"
                  % (name, sum(new), sum(lengths), kind, start.elapsed_time(end) * 1e3 / a.steps), flush=True)
        return step()

    run("prompts", lengths, lengths, False)
    out = run("decode", [n + 1 for n in lengths], [1] * a.batch, True)
    print("largest |out| %.3g" % out.abs().max().item())


if __name__ == "__main__":
    main()
