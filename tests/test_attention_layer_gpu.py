"""Rotary positions, the cache, attention and adapters together, as a program
uses them: the example's layer against a plain form in binary64, prompts, then
drafts, then single tokens on the cache they left; captured and replayed; on
streams of their own."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import attn_util as A
import paper_2402_10076_amd as Q
from gpu_util import f16_values, say

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")
    spec = importlib.util.spec_from_file_location("attention_layer", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


EX = _example()
HIDDEN, HQ, H, D, RANK, E = 256, 4, 2, 64, 16, 3


class Plain:
    """The layer in binary64, each intermediate rounded to what the layer holds it in."""

    def __init__(self, weights, adapters, freqs, factor):
        self.w = [self._matrix(*w) for w in weights]
        self.adapters = [t.double().cpu() for t in adapters]
        self.freqs, self.factor = freqs.cpu(), factor
        self.k, self.v = {}, {}       # slot: [H][D]

    @staticmethod
    def _matrix(q, z, s):
        s = f16_values(s.view(np.uint16))
        return torch.from_numpy((q.astype(np.float64) - np.repeat(z, 128, 0)) * np.repeat(s, 128, 0))

    def __call__(self, x, ids, positions, slots, table, lengths, offsets):
        a, b, scales = self.adapters
        x = x.double().cpu()
        qkv = (x @ self.w[0]).half().double()
        for t in range(x.shape[0]):
            if ids[t] >= 0:
                low = (scales[ids[t]] * (a[ids[t]] @ x[t])).half().double()
                qkv[t] = (qkv[t] + b[ids[t]] @ low).half().double()
        heads = qkv.view(-1, HQ + 2 * H, D)
        turned = A.rotated(heads[:, :HQ + H], positions.cpu(), self.freqs, factor=self.factor)[0].half().double()
        for t, s in enumerate(slots.tolist()):
            self.k[s], self.v[s] = A.rounded(turned[t, HQ:].half()), A.rounded(heads[t, HQ + H:].half())
        lengths, offsets, table = lengths.tolist(), offsets.tolist(), table.tolist()
        k = [torch.stack([self.k[table[i][j // 64] * 64 + j % 64] for j in range(n)]) for i, n in enumerate(lengths)]
        v = [torch.stack([self.v[table[i][j // 64] * 64 + j % 64] for j in range(n)]) for i, n in enumerate(lengths)]
        y, _, _ = A.attention(turned[:, :HQ], k, v, lengths, offsets, HQ // H, torch.float16)
        return (y.half().double().reshape(x.shape[0], -1) @ self.w[1])


def _weights(seed):
    g = np.random.Generator(np.random.PCG64(seed))
    return EX.random_weights(g, HIDDEN, (HQ + 2 * H) * D), EX.random_weights(g, HQ * D, HIDDEN)


def _bits(w):
    return w[0], w[1], w[2].view(np.uint16)


def _layer(pages, seed=1):
    w = _weights(seed)
    g = A.gen(seed)
    adapters = (A.normal(g, E, RANK, HIDDEN, scale=HIDDEN ** -0.5).cuda(),
                A.normal(g, E, (HQ + 2 * H) * D, RANK, scale=0.3 * RANK ** -0.5).cuda(), (torch.rand(E, generator=g) + 0.5).cuda())
    layer = EX.Attention(*map(_bits, w), HQ, H, D, pages, adapters, scaling="ramp", factor=4.0, original=128)
    return layer, Plain(w, adapters, layer.freqs, layer.factor)


def test_layer_over_prompts_drafts_and_single_tokens():
    """Each call reads what the calls before it have written.  A key or value at
    the edge of two codes may fall to either side (a step of a quarter of its
    block's largest), as its input is rounded to 16 bits after sums in another
    order; a token's scores and weights dilute it: 4 % of the largest output."""
    lengths = [70, 3, 200, 129]
    layer, plain = _layer(20)
    pages = 20
    for i, new in enumerate((lengths, [3, 1, 4, 2], [1, 1, 1, 1], [1, 1, 1, 1])):
        if i:
            lengths = [n + m for n, m in zip(lengths, new)]
        # the pages of the longest sequences that come, so that every call has the same table
        pos, slots, table, ln, off = EX.batch(lengths, new, width=5, pages=pages)
        full = EX.batch([n // 64 * 64 + 64 for n in (90, 20, 220, 140)], [1] * 4, width=5, pages=pages)[2]
        seq = torch.repeat_interleave(torch.arange(4), torch.tensor(new))
        slots = (full.cpu()[seq, pos.cpu().long() // 64].long() * 64 + pos.cpu().long() % 64).to(torch.int32).cuda()
        ids = (seq % (E + 1) - 1).to(torch.int32)
        x = A.normal(A.gen(50 + i), sum(new), HIDDEN)
        say("layer", i, lengths, new)
        out = layer(x.cuda(), pos, slots, full, ln, off, max(new), Q.lora_group(ids.cuda(), E))
        want = plain(x, ids.tolist(), pos, slots, full.cpu(), ln.cpu(), off.cpu())
        assert float((out.cpu().double() - want).abs().max() / want.abs().max()) < 0.04


def test_decode_step_is_captured_and_replayed():
    """With new inputs, slots, lengths and adapters in the same tensors at each replay, and eager steps between."""
    layer, _ = _layer(30)
    other, _ = _layer(30)
    B = 5
    lengths = torch.tensor([63, 1, 128, 300, 64])
    table = torch.randperm(30, generator=A.gen(3))[:B * 6].view(B, 6).to(torch.int32).cuda()
    x = torch.zeros((B, HIDDEN), dtype=torch.float16, device="cuda")
    pos, slots, ln, ids = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(4))
    g = A.gen(4)
    k = A.normal(g, 30 * 64, H, D).cuda()
    v = A.normal(g, 30 * 64, H, D).cuda()
    for l in (layer, other):
        Q.kv4_write(l.cache, k, v, torch.arange(30 * 64, dtype=torch.int32, device="cuda"))

    def fill(i):
        n = lengths + i
        x.copy_(A.normal(A.gen(9, i), B, HIDDEN))
        pos.copy_(n.to(torch.int32))
        slots.copy_((table.cpu()[torch.arange(B), n // 64].long() * 64 + n % 64).to(torch.int32))
        ln.copy_((n + 1).to(torch.int32))
        ids.copy_(((torch.arange(B) + i) % (E + 1) - 1).to(torch.int32))

    def step(l):
        return l(x, pos, slots, table, ln, None, 1, Q.lora_group(ids, E))
    fill(0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(layer)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step(layer)
    for i in range(4):
        fill(i)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step(other)) and torch.equal(layer.cache, other.cache)


def _calls():
    """(name, call on a stream) of every entry point that allocates."""
    g = A.gen(1)
    x = A.normal(g, 200, 4, 64).cuda()
    pos = torch.arange(200, dtype=torch.int32, device="cuda")
    freqs = Q.rotary_frequencies(64)[0]
    cache = Q.kv4_cache(60, 2, 64)
    k, v = A.normal(g, 3840, 2, 64).cuda(), A.normal(g, 3840, 2, 64).cuda()
    Q.kv4_write(cache, k, v, torch.arange(3840, dtype=torch.int32, device="cuda"))
    table = torch.arange(60, dtype=torch.int32, device="cuda").view(2, 30)
    lengths = torch.tensor([1900, 700], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 150, 200], dtype=torch.int32, device="cuda")
    ids = (torch.arange(200, device="cuda") % 4 - 1).to(torch.int32)
    lx, ly = A.normal(g, 200, 256).cuda(), A.normal(g, 200, 136).cuda()
    a, b = A.normal(g, 3, 16, 256, scale=0.1).cuda(), A.normal(g, 3, 136, 16, scale=0.1).cuda()
    order = Q.lora_group(ids, 3)
    return {
        "rotary": lambda s: Q.rotary(x, pos, freqs, stream=s),
        "read": lambda s: Q.kv4_read(cache, pos, stream=s),
        "attention, tokens": lambda s: Q.kv4_attention(x[:2], cache, table, lengths, stream=s),
        "attention, short": lambda s: Q.kv4_attention(x[:2], cache, table[:, :16].contiguous(), lengths, stream=s),
        "attention, prompts": lambda s: Q.kv4_attention(x, cache, table, lengths, offsets=off, most=150, stream=s),
        "group": lambda s: Q.lora_group(ids, 3, stream=s),
        "add": lambda s: Q.lora_add(ly, lx, a, b, *order, stream=s),
    }


CALLS = ("rotary", "read", "attention, tokens", "attention, short", "attention, prompts", "group", "add")


@pytest.fixture(scope="module")
def calls():
    return _calls()


@pytest.fixture(scope="module")
def side():
    return torch.cuda.Stream()


def _tensors(out):
    return [out] if isinstance(out, torch.Tensor) else list(out)


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_pending_work_is_left_alone(name, calls, side):
    """A block of each output's size is freed while a copy from it still waits on the current stream behind other work;
    the call on another stream gives the bits of one on the current stream, and the copy finds what it is to copy."""
    ref = _tensors(calls[name](None))
    big = torch.empty((2, 1 << 28), dtype=torch.uint8, device="cuda")
    side.synchronize()
    for n in sorted({t.nbytes for t in ref}):
        block = torch.full((n,), 0x55, dtype=torch.uint8, device="cuda")
        copy = torch.empty_like(block)
        torch.cuda.synchronize()
        say("pending", name, n)
        for _ in range(40):
            big[0].copy_(big[1])
        copy.copy_(block)
        del block
        out = _tensors(calls[name](side))
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
        torch.cuda.synchronize()
        assert bool((copy == 0x55).all())


@pytest.mark.parametrize("name", CALLS)
def test_captured_calls_replay(name, calls, side):
    """Two graphs of the same call, replayed in turn with eager calls between."""
    ref = _tensors(calls[name](None))
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = _tensors(calls[name](side))
        graphs.append((graph, out))
    for i in range(4):
        graph, out = graphs[i % 2]
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
        assert all(torch.equal(a, b) for a, b in zip(_tensors(calls[name](None)), ref))


def test_workspaces_that_are_given():
    """Filled with anything, used again, and by calls of other sizes in their order."""
    c = Q.kv4_cache(40, 2, 64)
    g = A.gen(6)
    Q.kv4_write(c, A.normal(g, 2560, 2, 64).cuda(), A.normal(g, 2560, 2, 64).cuda(),
                torch.arange(2560, dtype=torch.int32, device="cuda"))
    table = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20)
    lengths = torch.tensor([1280, 900], dtype=torch.int32, device="cuda")
    q = A.normal(g, 300, 4, 64).cuda()
    need = max(Q.kv4_attention_workspace_bytes(300, 4, 2, 64, 40, 2, 20, most=m) for m in (1, 20, 200))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        for most, off in ((1, [0, 1, 2]), (20, [0, 20, 30]), (200, [0, 200, 300])):
            o = torch.tensor(off, dtype=torch.int32, device="cuda")
            n = off[-1]
            out = Q.kv4_attention(q[:n], c, table, lengths, offsets=o, most=most, workspace=ws)
            assert torch.equal(out, Q.kv4_attention(q[:n], c, table, lengths, offsets=o, most=most))
    with pytest.raises(Q.QuickError) as e:
        Q.kv4_attention(q, c, table, lengths, offsets=o, most=200, workspace=ws[:64])
    assert e.value.status == Q.QUICK_ERR_WORKSPACE
