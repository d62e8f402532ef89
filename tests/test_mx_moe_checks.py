"""What the microscaled 4-bit and mixture-of-experts entry points refuse, on
the CPU: the binding's checks with the library replaced by a stub that records
calls ("meta" tensors stand in for device tensors), and the C ABI's own, which
come before any launch.  And the packed layout's sizes."""
import ctypes

import pytest
import torch

import mx_util as U
import paper_2402_10076_amd as Q

A = 0x10000          # an aligned address that is never dereferenced
OK, ARG, SHAPE, ALIGN, WORK = (Q.QUICK_OK, Q.QUICK_ERR_INVALID_ARG, Q.QUICK_ERR_SHAPE, Q.QUICK_ERR_ALIGNMENT,
                               Q.QUICK_ERR_WORKSPACE)


class _Stub:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def f(*a):
            self.calls.append(name)
            return 0
        return f


class _Stream:
    cuda_stream = 0


S = _Stream()


@pytest.fixture
def stub(monkeypatch):
    s = _Stub()
    monkeypatch.setattr(Q, "lib", lambda: s)
    monkeypatch.setattr(Q, "_DEVICE_TYPE", "meta")
    return s


def _dev(*shape, dtype=torch.uint8):
    return torch.empty(shape, dtype=dtype, device="meta")


def _rejects(stub, status, fn, *a, **kw):
    def launches():
        return [c for c in stub.calls if not c.endswith("_bytes") and c != "quick_status_string"]
    before = launches()
    with pytest.raises(Q.QuickError) as e:
        fn(*a, **kw, stream=S)
    assert e.value.status == status
    assert launches() == before


M, K, N, E = 4, 160, 32, 3
PB, SB = 2 * 2 * 1024, 2 * 256


def _x():
    return _dev(M, K // 2), _dev(M, K // 32)


def _w(e=1):
    return _dev(e * PB), _dev(e * SB)


def test_valid_calls_reach_the_library(stub):
    assert Q.mxfp4_quantize(_dev(M, K, dtype=torch.float32), stream=S)[1].shape == (M, K // 32)
    assert Q.mxfp4_dequantize(*_x(), dtype=torch.bfloat16, stream=S).shape == (M, K)
    assert Q.mxfp4_pack(_dev(E, N, K // 2), _dev(E, N, K // 32), stream=S)[0].shape == (E, PB)
    assert Q.mxfp4_gemm(*_x(), *_w(), N, stream=S).shape == (M, N)
    assert Q.mxfp4_linear(_dev(M, K, dtype=torch.float16), *_w(), N, activation=Q.ACT_SILU_GATE,
                          stream=S).shape == (M, N // 2)
    o = _dev(E + 1, dtype=torch.int32)
    assert Q.mxfp4_grouped_gemm(*_x(), o, *_w(E), N, rows=_dev(9, dtype=torch.int32), stream=S).shape == (9, N)
    r = Q.moe_route(_dev(5, 8, dtype=torch.float16), 2, stream=S)
    assert r.slots.shape == (5, 2) and r.offsets.shape == (9,)
    assert Q.moe_combine(_dev(10, 7, dtype=torch.float16), r.slots, r.weights, stream=S).shape == (5, 7)
    assert [c for c in stub.calls if not c.endswith("_bytes")] == [
        "quick_mxfp4_quantize", "quick_mxfp4_dequantize", "quick_mxfp4_pack", "quick_mxfp4_gemm", "quick_mxfp4_linear",
        "quick_mxfp4_grouped_gemm", "quick_moe_route", "quick_moe_combine"]


def test_quantize_refusals(stub):
    f = Q.mxfp4_quantize
    _rejects(stub, ARG, f, torch.zeros(M, K))
    _rejects(stub, ARG, f, _dev(M, K, dtype=torch.float64))
    _rejects(stub, ARG, f, _dev(K, M, dtype=torch.float32).t())
    _rejects(stub, ARG, f, _dev(K, dtype=torch.float32))
    _rejects(stub, SHAPE, f, _dev(M, K + 16, dtype=torch.float32))
    _rejects(stub, SHAPE, f, _dev(M, 0, dtype=torch.float32))
    _rejects(stub, SHAPE, f, _dev(1, K, dtype=torch.float32).expand(M, K))
    x = _dev(M, K, dtype=torch.float16)
    _rejects(stub, ARG, f, x, codes=_dev(M, K))
    _rejects(stub, ARG, f, x, scales=_dev(M, K // 32, dtype=torch.int32))
    _rejects(stub, ARG, f, x, codes=torch.zeros(M, K // 2, dtype=torch.uint8))
    _rejects(stub, ARG, Q.mxfp4_dequantize, _dev(M, K // 2), _dev(M, K // 32 + 1))
    _rejects(stub, ARG, Q.mxfp4_dequantize, *_x(), dtype=torch.float64)
    _rejects(stub, ARG, Q.mxfp4_dequantize, _dev(M, K // 2, dtype=torch.int8), _dev(M, K // 32))


def test_product_refusals(stub):
    o = _dev(E + 1, dtype=torch.int32)
    x16 = _dev(M, K, dtype=torch.float16)
    calls = [lambda **k: (Q.mxfp4_gemm, (*k.pop("x", _x()), *k.pop("w", _w()), k.pop("N", N)), k),
             lambda **k: (Q.mxfp4_grouped_gemm, (*k.pop("x", _x()), o, *k.pop("w", _w(E)), k.pop("N", N)), k),
             lambda **k: (Q.mxfp4_linear, (k.pop("x", (x16,))[0], *k.pop("w", _w()), k.pop("N", N)), k)]
    for i, c in enumerate(calls):
        def bad(status, **k):
            fn, a, kw = c(**k)
            _rejects(stub, status, fn, *a, **kw)
        e = E if i == 1 else 1
        pb, sb = _w(e)
        bad(SHAPE, w=(_dev(e * PB - 1), sb))
        bad(SHAPE, w=(pb, _dev(e * SB - 1)))
        bad(ARG, w=(torch.zeros(e * PB, dtype=torch.uint8), sb))
        bad(SHAPE, N=0)
        bad(SHAPE, N=-16)
        bad(SHAPE, N=40, w=(_dev(e * PB * 2), _dev(e * SB * 2)), activation=Q.ACT_SILU_GATE)
        bad(ARG, y=_dev(M, N + 1, dtype=torch.float16))
        bad(ARG, y=_dev(M, N, dtype=torch.float32))
        bad(SHAPE, bias=_dev(e * N - 1, dtype=torch.float16))
        bad(ARG, bias=_dev(e * N, dtype=torch.float32))
        if i < 2:
            bad(ARG, x=(_dev(M, K // 2), _dev(M, K // 32 + 1)))
            bad(ARG, x=(_dev(M, K // 2, dtype=torch.int8), _dev(M, K // 32)))
            bad(ARG, x=(_dev(K // 2, M).t(), _dev(M, K // 32)))
            bad(ARG, dtype=torch.float32)
        else:
            bad(ARG, x=(_dev(M, K, dtype=torch.float32),))
            bad(ARG, x=(_dev(M, 2 * K, dtype=torch.float16)[:, ::2],))
            bad(SHAPE, x=(_dev(M, K + 8, dtype=torch.float16),))
            bad(ARG, workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    g = Q.mxfp4_grouped_gemm
    _rejects(stub, ARG, g, *_x(), _dev(E + 1, dtype=torch.int64), *_w(E), N)
    _rejects(stub, ARG, g, *_x(), _dev(1, dtype=torch.int32), *_w(E), N)
    _rejects(stub, ARG, g, *_x(), o, *_w(E), N, rows=_dev(5, dtype=torch.int64))
    _rejects(stub, SHAPE, g, *_x(), o, *_w(E), N, rows=_dev(5, dtype=torch.int32), R=6)
    _rejects(stub, ARG, Q.mxfp4_pack, _dev(2, E, N, K // 2), _dev(2, E, N, K // 32))


def test_moe_refusals(stub):
    f = Q.moe_route
    x = _dev(5, 8, dtype=torch.float32)
    _rejects(stub, ARG, f, torch.zeros(5, 8), 2)
    _rejects(stub, ARG, f, _dev(5, 8, dtype=torch.int32), 2)
    _rejects(stub, ARG, f, _dev(8, 5, dtype=torch.float32).t(), 2)
    _rejects(stub, SHAPE, f, _dev(5, 513, dtype=torch.float32), 2)
    _rejects(stub, SHAPE, f, x, 0)
    _rejects(stub, SHAPE, f, x, 17)
    _rejects(stub, ARG, f, x, 2, bias=_dev(8, dtype=torch.float16))
    _rejects(stub, ARG, f, x, 2, bias=_dev(7, dtype=torch.float32))
    good = Q.moe_route(x, 2, stream=S)
    for i in range(5):
        out = list(good)
        out[i] = _dev(3, dtype=out[i].dtype)
        _rejects(stub, ARG, f, x, 2, out=Q.Routing(*out))
    _rejects(stub, ARG, f, x, 2, workspace=torch.zeros(64))
    c = Q.moe_combine
    y, s, w = _dev(10, 7, dtype=torch.float16), _dev(5, 2, dtype=torch.int32), _dev(5, 2, dtype=torch.float32)
    _rejects(stub, ARG, c, _dev(10, 7, dtype=torch.float32), s, w)
    _rejects(stub, ARG, c, _dev(7, 10, dtype=torch.float16).t(), s, w)
    _rejects(stub, ARG, c, y, _dev(5, 2, dtype=torch.int64), w)
    _rejects(stub, ARG, c, y, _dev(10, dtype=torch.int32), w)
    _rejects(stub, ARG, c, y, s, _dev(5, 3, dtype=torch.float32))
    _rejects(stub, ARG, c, y, s, w, residual=_dev(5, 7, dtype=torch.bfloat16))
    _rejects(stub, ARG, c, y, s, w, out=_dev(5, 8, dtype=torch.float16))


def test_abi_quantize_and_pack():
    L = Q.lib()

    def q(x=A, dt=0, ldx=K, rows=M, k=K, c=A, s=A):
        return L.quick_mxfp4_quantize(x, dt, ldx, rows, k, c, s, None)
    assert q(rows=0) == OK
    assert q(dt=3) == q(dt=-1) == ARG
    assert q(k=48) == q(k=0) == q(k=-32) == q(rows=-1) == q(ldx=K - 1) == q(rows=(1 << 24) + 1) == SHAPE
    assert q(k=(1 << 22) + 32, ldx=1 << 23) == SHAPE
    assert q(rows=1 << 24, k=16384, ldx=16384 + 8) == SHAPE
    assert q(x=0) == q(c=0) == q(s=0) == ARG
    assert q(x=A + 8) == q(c=A + 4) == q(ldx=K + 4) == ALIGN
    assert L.quick_mxfp4_dequantize(A, A, 0, 0, K, A, None) == OK
    assert L.quick_mxfp4_dequantize(A, A, 0, M, 33, A, None) == SHAPE
    assert L.quick_mxfp4_dequantize(A, 0, 0, M, K, A, None) == ARG
    assert L.quick_mxfp4_dequantize(A, A, 5, M, K, A, None) == ARG
    assert L.quick_mxfp4_dequantize(A, A, 0, M, K, A + 8, None) == ALIGN
    for n, k in ((1, 32), (16, 128), (17, 160), (37, 544), (64, 4096)):
        p, s = U.packed(torch.zeros((n, k // 2), dtype=torch.uint8).numpy(),
                        torch.zeros((n, k // 32), dtype=torch.uint8).numpy())
        assert Q.mxfp4_packed_sizes(n, k) == (p.nbytes, s.nbytes)
    for n, k in ((0, 32), (16, 33), (16, 0), (1 << 22, 1 << 12), ((1 << 24) + 1, 32)):
        with pytest.raises(Q.QuickError) as e:
            Q.mxfp4_packed_sizes(n, k)
        assert e.value.status == SHAPE

    def pk(c=A, s=A, e=1, n=N, k=K, g=0, p=A, t=A):
        return L.quick_mxfp4_pack(c, s, e, n, k, g, p, t, None)
    assert pk(e=0) == pk(e=513) == pk(n=48, g=1) == pk(k=31) == SHAPE
    assert pk(c=0) == pk(s=0) == pk(p=0) == pk(t=0) == ARG
    assert pk(c=A + 8) == pk(p=A + 8) == pk(t=A + 2) == ALIGN


def test_abi_products():
    L = Q.lib()

    def gemm(c=A, s=A, p=A, t=A, y=A, dt=0, m=M, n=N, k=K, b=None, act=0):
        return L.quick_mxfp4_gemm(c, s, p, t, y, dt, m, n, k, b, act, None)

    def grouped(c=A, s=A, p=A, t=A, y=A, dt=0, m=M, n=N, k=K, b=None, act=0, rows=A, offsets=A, r=9, e=E):
        return L.quick_mxfp4_grouped_gemm(c, s, rows, offsets, p, t, y, dt, m, r, e, n, k, b, act, None)

    def linear(c=A, p=A, t=A, y=A, dt=0, m=M, n=N, k=K, b=None, act=0, ws=A, wsb=1 << 20):
        return L.quick_mxfp4_linear(c, p, t, y, dt, m, n, k, b, act, ws, wsb, None)
    assert gemm(m=0) == linear(m=0) == grouped(r=0) == grouped(r=0, m=0) == OK
    for f in (gemm, grouped, linear):
        assert f(dt=2) == f(act=2) == f(c=0) == f(p=0) == f(t=0) == f(y=0) == ARG
        assert f(k=48) == f(n=0) == f(n=48, act=1) == f(m=-1) == SHAPE
        assert f(n=1 << 22, k=1 << 12) == SHAPE
        assert f(c=A + 8) == f(p=A + 8) == f(t=A + 2) == f(y=A + 4) == f(b=A + 1) == ALIGN
    assert gemm(s=0) == grouped(s=0) == ARG and gemm(s=A + 2) == grouped(s=A + 1) == ALIGN
    assert gemm(m=1 << 22, k=4096) == SHAPE                       # 2^34 activations
    assert gemm(m=(1 << 22) + 1, k=32) == SHAPE
    assert grouped(e=0) == grouped(e=513) == grouped(m=0) == grouped(rows=None, m=8, r=9) == SHAPE
    assert grouped(offsets=None) == ARG and grouped(offsets=A + 2) == grouped(rows=A + 2) == ALIGN
    m = 4096
    need = Q.mxfp4_linear_workspace_bytes(m, N, K)
    assert need >= m * K // 2 + m * K // 32
    assert linear(m=m, ws=None, wsb=0) == linear(m=m, wsb=need - 1) == WORK
    assert linear(m=m, ws=A + 8) == ALIGN
    assert Q.mxfp4_linear_workspace_bytes(0, N, K) == Q.mxfp4_linear_workspace_bytes(m, N, 33) == 0


def test_abi_moe():
    L = Q.lib()

    def route(x=A, dt=2, t=5, e=64, out=(A,) * 5, ws=A, wsb=1 << 30, **k):
        r = Q.moe.QuickRoute(k.get("score", 0), k.get("topk", 2), k.get("groups", 1), k.get("topk_groups", 1),
                             k.get("group_best", 1), 1, 1.0)
        return L.quick_moe_route(x, dt, t, e, ctypes.byref(r), k.get("bias"), *out, ws, wsb, None)
    assert route(dt=3) == route(score=2) == route(group_best=0) == route(group_best=3) == route(x=0) == ARG
    assert L.quick_moe_route(A, 2, 5, 8, None, None, A, A, A, A, A, None, 0, None) == ARG
    for i in range(5):
        out = [A] * 5
        out[i] = None
        assert route(out=out) == ARG
        out[i] = A + 2
        assert route(out=out) == ALIGN
    assert route(x=A + 2) == route(bias=A + 2) == ALIGN and route(x=A + 1, dt=0) == ALIGN
    assert route(t=-1) == route(e=0) == route(e=513) == route(topk=0) == route(topk=17) == SHAPE
    assert route(topk=2, e=1) == route(groups=7) == route(groups=0) == route(groups=65, e=130) == SHAPE
    assert route(groups=8, topk_groups=9) == route(groups=8, topk_groups=0) == SHAPE
    assert route(groups=8, topk_groups=1, topk=9) == SHAPE
    assert route(t=(1 << 30) + 1, topk=1) == route(t=1 << 28, topk=8) == SHAPE
    need = Q.moe_route_workspace_bytes(10000, 64, 2)
    assert need > 0 and route(t=10000, wsb=need - 1) == route(t=10000, ws=None) == WORK
    assert route(t=10000, ws=A + 4) == ALIGN
    assert Q.moe_route_workspace_bytes(1, 64, 2) == Q.moe_route_workspace_bytes(0, 64, 2) == 0

    def comb(y=A, dt=0, r=10, d=64, s=A, w=A, t=5, k=2, res=None, out=A):
        return L.quick_moe_combine(y, dt, r, d, s, w, t, k, res, out, None)
    assert comb(t=0) == OK
    assert comb(dt=2) == comb(y=0) == comb(s=0) == comb(w=0) == comb(out=0) == ARG
    assert comb(t=-1) == comb(r=-1) == comb(d=0) == comb(k=0) == comb(k=17) == comb(t=1 << 24) == SHAPE
    assert comb(y=A + 1) == comb(s=A + 2) == comb(w=A + 2) == comb(res=A + 1) == comb(out=A + 1) == ALIGN


def test_headers_compile_as_plain_c(tmp_path):
    import os
    import subprocess
    src = tmp_path / "t.c"
    src.write_text('#include "quick_mx.h"\n#include "quick_moe.h"\nint main(void) {\n'
                   "    size_t a, b;\n    quick_route_t r = {QUICK_SCORE_SIGMOID, 2, 1, 1, 1, 1, 1.0f};\n"
                   "    if (quick_mxfp4_packed_sizes(32, 160, &a, &b) != QUICK_OK || a != 4096 || b != 512) return 1;\n"
                   "    if (quick_moe_route(0, QUICK_F32, 4, 8, &r, 0, 0, 0, 0, 0, 0, 0, 0, 0) != QUICK_ERR_INVALID_ARG) "
                   "return 2;\n    return QUICK_MAX_TOPK == 16 && QUICK_MAX_GROUPS == 64 ? 0 : 3;\n}\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "t")
    libdir = os.path.dirname(Q.LIB_PATH)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", exe,
                    os.path.join(libdir, "libquick.so"), "-Wl,-rpath," + libdir], check=True)
    assert subprocess.run([exe]).returncode == 0
    assert (Q.MAX_TOPK, Q.MAX_GROUPS, Q.MAX_EXPERTS) == (16, 64, 512)
