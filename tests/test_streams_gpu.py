"""Calls with ``stream=``: what they allocate must not be memory that work on
the current stream, behind which they are not ordered, still uses."""
import numpy as np
import pytest
import torch

import paper_2402_10076_amd as Q
from gpu_util import say

pytestmark = pytest.mark.gpu


def _calls():
    """(name, call on a stream, bytes of its workspace) of every entry point that allocates."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def codes(*shape):
        return torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=g)

    def scales(*shape):
        return torch.randint(120, 124, shape, dtype=torch.uint8, device="cuda", generator=g)
    M, N, K, E, k = 200, 1040, 2080, 16, 2
    x = torch.randn((M, K), device="cuda", generator=g).half()
    xc, xs, wc, ws = codes(M, K // 2), scales(M, K // 32), codes(N, K // 2), scales(N, K // 32)
    packed = Q.mxfp4_pack(wc, ws)
    experts = Q.mxfp4_pack(codes(2, N, K // 2), scales(2, N, K // 32))
    offsets = torch.tensor([0, 90, M], dtype=torch.int32, device="cuda")
    logits = torch.randn((3000, E), device="cuda", generator=g)
    r = Q.moe_route(logits, k)
    y = torch.randn((3000 * k, 520), device="cuda", generator=g).half()
    rng = np.random.Generator(np.random.PCG64(2))
    q, z = rng.integers(0, 16, (2048, 1024), dtype=np.uint8), rng.integers(0, 16, (16, 1024), dtype=np.uint8)
    w4 = Q.to_device(*Q.pack_weights(q, z, rng.uniform(0.002, 0.01, z.shape).astype(np.float16).view(np.uint16)))
    x4, o4 = x[:, :2048].contiguous(), torch.tensor([0, M], dtype=torch.int32, device="cuda")
    return [
        ("quantize", lambda s: Q.mxfp4_quantize(x, stream=s), 0),
        ("dequantize", lambda s: Q.mxfp4_dequantize(xc, xs, stream=s), 0),
        ("pack", lambda s: Q.mxfp4_pack(wc, ws, stream=s), 0),
        ("gemm", lambda s: Q.mxfp4_gemm(xc, xs, *packed, N, stream=s), 0),
        ("linear", lambda s: Q.mxfp4_linear(x, *packed, N, stream=s), Q.mxfp4_linear_workspace_bytes(M, N, K)),
        ("linear, one row", lambda s: Q.mxfp4_linear(x[:1], *packed, N, stream=s), 0),
        ("grouped", lambda s: Q.mxfp4_grouped_gemm(xc, xs, offsets, *experts, N, stream=s), 0),
        ("route", lambda s: Q.moe_route(logits, k, stream=s), Q.moe_route_workspace_bytes(3000, E, k)),
        ("combine", lambda s: Q.moe_combine(y, r.slots, r.weights, stream=s), 0),
        ("w4a16", lambda s: Q.w4a16_gemm(x4, *w4, 1024, stream=s), 0),
        ("w4a16 fused", lambda s: Q.gemm_fused(x4, *w4, 1024, activation=Q.ACT_SILU_GATE, stream=s), 0),
        ("w4a16 grouped", lambda s: Q.grouped_gemm(x4, o4, *w4, 1024, stream=s), 0),
        ("w4a16 grouped, fused", lambda s: Q.grouped_gemm_fused(x4, o4, *w4, 1024, stream=s), 0),
    ]


def _tensors(out):
    return [out] if isinstance(out, torch.Tensor) else list(out)


CALLS = ("quantize", "dequantize", "pack", "gemm", "linear", "linear, one row", "grouped", "route", "combine", "w4a16",
         "w4a16 fused", "w4a16 grouped", "w4a16 grouped, fused")


@pytest.fixture(scope="module")
def calls():
    return {n: (f, w) for n, f, w in _calls()}


@pytest.fixture(scope="module")
def side():
    return torch.cuda.Stream()


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_pending_work_is_left_alone(name, calls, side):
    """A block of each size that the call allocates is freed while a copy from
    it still waits on the current stream behind other work; the call on
    another stream gives the bits of one on the current stream, and the copy
    finds what it is to copy."""
    call, work = calls[name]
    ref = _tensors(call(None))
    big = torch.empty((2, 1 << 28), dtype=torch.uint8, device="cuda")
    side.synchronize()
    for n in sorted({t.nbytes for t in ref} | {work}):
        if n == 0:
            continue
        block = torch.full((n,), 0x55, dtype=torch.uint8, device="cuda")
        copy = torch.empty_like(block)
        torch.cuda.synchronize()
        say("pending", name, n)
        for _ in range(40):
            big[0].copy_(big[1])
        copy.copy_(block)
        del block
        out = _tensors(call(side))
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
        torch.cuda.synchronize()
        assert bool((copy == 0x55).all())


@pytest.mark.parametrize("name", CALLS)
def test_allocations_are_of_the_call_s_stream(name, calls, side):
    """A block that was just freed on the current stream is not what a call on
    another one gets (with nothing pending: the pools alone are looked at)."""
    call, _ = calls[name]
    ref = _tensors(call(None))
    for i in range(len(ref)):
        n = ref[i].nbytes
        torch.cuda.synchronize()
        block = torch.empty((n,), dtype=torch.uint8, device="cuda")
        at = block.data_ptr()
        del block
        assert _tensors(call(side))[i].data_ptr() != at
    torch.cuda.synchronize()


def test_results_are_kept_for_the_current_stream(calls, side):
    """A result that is read on the current stream and dropped there is not
    handed out again on its own stream before it has been read."""
    call, _ = calls["dequantize"]
    ref = call(None)
    big = torch.empty((2, 1 << 28), dtype=torch.uint8, device="cuda")
    copy = torch.empty_like(ref)
    torch.cuda.synchronize()
    y = call(side)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(40):
        big[0].copy_(big[1])
    copy.copy_(y)
    del y
    with torch.cuda.stream(side):
        torch.empty_like(ref).fill_(7)
    torch.cuda.synchronize()
    assert torch.equal(copy, ref)


@pytest.mark.parametrize("name", [n for n in CALLS if not n.startswith("w4a16")])
def test_capture_on_the_given_stream(name, calls, side):
    call, _ = calls[name]
    ref = _tensors(call(None))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = _tensors(call(side))
    for _ in range(3):
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
        assert all(torch.equal(a, b) for a, b in zip(_tensors(call(None)), ref))
