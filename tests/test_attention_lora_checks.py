"""What rotary positions, the 4-bit cache, attention over it and adapters
refuse, on the CPU: the binding's checks with the library replaced by a stub
that records calls ("meta" tensors stand in for device tensors), and the C
ABI's own, which come before any launch."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2402_10076_amd as Q

A = 0x10000          # an aligned address that is never dereferenced
OK, ARG, SHAPE, UNSUP, ALIGN, WORK = (Q.QUICK_OK, Q.QUICK_ERR_INVALID_ARG, Q.QUICK_ERR_SHAPE, Q.QUICK_ERR_UNSUPPORTED,
                                      Q.QUICK_ERR_ALIGNMENT, Q.QUICK_ERR_WORKSPACE)
F16, F32, F64, I32, U8 = torch.float16, torch.float32, torch.float64, torch.int32, torch.uint8


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
    Q.attention._attention.cache_clear()
    Q.lora.lora_workspace_bytes.cache_clear()
    yield s
    Q.attention._attention.cache_clear()
    Q.lora.lora_workspace_bytes.cache_clear()


def _dev(*shape, dtype=F16):
    return torch.empty(shape, dtype=dtype, device="meta")


def _rejects(stub, status, fn, *a, **kw):
    def launches():
        return [c for c in stub.calls if not c.endswith("_bytes") and c != "quick_status_string"]
    before = launches()
    with pytest.raises(Q.QuickError) as e:
        fn(*a, **kw, stream=S)
    assert e.value.status == status, e.value
    assert launches() == before


T, H, D, B, W = 6, 2, 64, 3, 5


def _attn(**k):
    """(arguments, keywords) of an attention call, some replaced."""
    a = {"q": _dev(T, 4 * H, D), "cache": _dev(9, H, 68 * D, dtype=U8), "table": _dev(B, W, dtype=I32),
         "lengths": _dev(B, dtype=I32)}
    kw = {"offsets": _dev(B + 1, dtype=I32)}
    for n, v in k.items():
        (a if n in a else kw)[n] = v
    return tuple(a.values()), kw


def _lora(**k):
    a = {"y": _dev(T, 40), "x": _dev(T, 64), "a": _dev(3, 8, 64), "b": _dev(3, 40, 8), "offsets": _dev(4, dtype=I32),
         "rows": _dev(T, dtype=I32)}
    kw = {}
    for n, v in k.items():
        (a if n in a else kw)[n] = v
    return tuple(a.values()), kw


def test_valid_calls_reach_the_library(stub):
    x, pos, f = _dev(T, H, D, dtype=F32), _dev(T, dtype=I32), _dev(16, dtype=F64)
    assert Q.rotary(x, pos, f, stream=S).shape == (T, H, D)
    assert Q.rotary(_dev(T, 3 * H, 80)[:, H:2 * H, 8:72], pos, f, stream=S).shape == (T, H, D)
    assert Q.rotary(x, pos, f, out=x, stream=S) is x
    cache = _dev(9, H, 68 * D, dtype=U8)
    kv = _dev(T, 3 * H, D)
    assert Q.kv4_write(cache, kv[:, :H], kv[:, H:2 * H], pos, stream=S) is cache
    assert Q.kv4_read(cache, pos, dtype=torch.bfloat16, stream=S)[1].shape == (T, H, D)
    args, kw = _attn()
    assert Q.kv4_attention(*args, **kw, most=2, window=7, stream=S).shape == (T, 4 * H, D)
    args, kw = _attn(q=_dev(B, 4 * H, D), offsets=None)
    assert Q.kv4_attention(*args, **kw, lse=_dev(B, 4 * H, dtype=F32), causal=False, stream=S).shape == (B, 4 * H, D)
    o, r = Q.lora_group(pos, 3, stream=S)
    assert o.shape == (4,) and r.shape == (T,)
    args, kw = _lora()
    assert Q.lora_add(*args, scales=_dev(3, dtype=F32), stream=S).shape == (T, 40)
    wide = _dev(T, 80)
    args, kw = _lora(y=wide[:, 8:48], x=_dev(T, 72)[:, 8:])
    assert Q.lora_add(*args, out=wide[:, 8:48], stream=S).shape == (T, 40)
    assert [c for c in stub.calls if not c.endswith("_bytes")] == [
        "quick_rotary"] * 3 + ["quick_kv4_write", "quick_kv4_read"] + ["quick_kv4_attention"] * 2 + [
        "quick_lora_group"] + ["quick_lora_add"] * 2


def test_rotary_refusals(stub):
    x, pos, f = _dev(T, H, D), _dev(T, dtype=I32), _dev(16, dtype=F64)
    r = Q.rotary
    _rejects(stub, ARG, r, torch.zeros(T, H, D), pos, f)
    _rejects(stub, ARG, r, _dev(T, H, D, dtype=F64), pos, f)
    _rejects(stub, ARG, r, _dev(T, H * D), pos, f)
    _rejects(stub, ARG, r, _dev(T, D, H).transpose(1, 2), pos, f)
    _rejects(stub, ARG, r, x, _dev(T, dtype=torch.int64), f)
    _rejects(stub, ARG, r, x, _dev(T + 1, dtype=I32), f)
    _rejects(stub, ARG, r, x, torch.zeros(T, dtype=I32), f)
    _rejects(stub, ARG, r, x, pos, _dev(16, dtype=F32))
    _rejects(stub, ARG, r, x, pos, _dev(4, 4, dtype=F64))
    _rejects(stub, ARG, r, x, pos, _dev(32, dtype=F64)[::2])
    _rejects(stub, SHAPE, r, x, pos, _dev(33, dtype=F64))
    _rejects(stub, ARG, r, x, pos, f, out=_dev(T, H, D, dtype=F32))
    _rejects(stub, ARG, r, x, pos, f, out=_dev(T, H, D + 2))
    _rejects(stub, SHAPE, r, x, pos, f, out=_dev(1, H, D).expand(T, H, D))
    with pytest.raises(Q.QuickError):
        Q.rotary_frequencies(7, device="cpu")
    with pytest.raises(Q.QuickError):
        Q.rotary_frequencies(8, scaling="ramp", device="cpu")
    with pytest.raises(Q.QuickError):
        Q.rotary_frequencies(8, scaling="other", device="cpu")


def test_cache_refusals(stub):
    cache, kv, slots = _dev(9, H, 68 * D, dtype=U8), _dev(T, H, D), _dev(T, dtype=I32)
    w = Q.kv4_write
    _rejects(stub, ARG, w, cache, torch.zeros(T, H, D, dtype=F16), kv, slots)
    _rejects(stub, ARG, w, cache, _dev(T, H, D, dtype=F32), kv, slots)
    _rejects(stub, ARG, w, cache, kv, _dev(T, H, D, dtype=torch.bfloat16), slots)
    _rejects(stub, ARG, w, cache, kv, _dev(T, H + 1, D), slots)
    _rejects(stub, ARG, w, cache, _dev(T, H, 2 * D), kv, slots)
    _rejects(stub, ARG, w, cache, kv, kv, _dev(T - 1, dtype=I32))
    _rejects(stub, ARG, w, cache, kv, kv, _dev(T, dtype=torch.int64))
    _rejects(stub, ARG, w, _dev(9, H, 68 * D, dtype=torch.int8), kv, kv, slots)
    _rejects(stub, ARG, w, _dev(9, H, 68 * 96, dtype=U8), kv, kv, slots)
    _rejects(stub, ARG, w, _dev(9, H, 68 * D + 1, dtype=U8), kv, kv, slots)
    _rejects(stub, ARG, w, _dev(18, H, 68 * D, dtype=U8)[::2], kv, kv, slots)
    _rejects(stub, ARG, Q.kv4_read, cache, slots, dtype=F64)
    _rejects(stub, ARG, Q.kv4_read, cache, _dev(T, 1, dtype=I32))
    _rejects(stub, ARG, Q.kv4_read, cache, slots, k=_dev(T, H, D, dtype=F32))
    _rejects(stub, ARG, Q.kv4_read, torch.zeros(9, H, 68 * D, dtype=U8), slots)
    with pytest.raises(Q.QuickError) as e:
        Q.kv4_cache(3, 2, 96, device="meta")
    assert e.value.status == UNSUP


def test_attention_refusals(stub):
    def bad(status, **k):
        args, kw = _attn(**k)
        _rejects(stub, status, Q.kv4_attention, *args, **kw)
    bad(ARG, q=torch.zeros(T, 4 * H, D, dtype=F16))
    bad(ARG, q=_dev(T, 4 * H, D, dtype=F32))
    bad(ARG, q=_dev(T, D, 4 * H).transpose(1, 2))
    bad(SHAPE, q=_dev(T, 4 * H + 1, D))
    bad(SHAPE, q=_dev(T, 4 * H, 128))
    bad(SHAPE, q=_dev(T, 0, D))
    bad(ARG, cache=_dev(9, H, 68 * D, dtype=I32))
    bad(ARG, cache=_dev(9, H * 68 * D, dtype=U8))
    bad(ARG, table=_dev(B * W, dtype=I32))
    bad(ARG, table=_dev(B, W, dtype=torch.int64))
    bad(ARG, table=_dev(W, B, dtype=I32).t())
    bad(ARG, lengths=_dev(B + 1, dtype=I32))
    bad(ARG, lengths=torch.zeros(B, dtype=I32))
    bad(ARG, offsets=_dev(B, dtype=I32))
    bad(ARG, offsets=_dev(B + 1, dtype=torch.int64))
    bad(SHAPE, offsets=None)
    bad(ARG, out=_dev(T, 4 * H, D, dtype=torch.bfloat16))
    bad(ARG, out=_dev(T, 4 * H * D))
    bad(ARG, lse=_dev(T, 4 * H))
    bad(ARG, lse=_dev(T, H, dtype=F32))
    bad(ARG, workspace=torch.zeros(1 << 20, dtype=U8))


def test_lora_refusals(stub):
    def bad(status, **k):
        args, kw = _lora(**k)
        _rejects(stub, status, Q.lora_add, *args, **kw)
    bad(ARG, x=torch.zeros(T, 64, dtype=F16))
    bad(ARG, x=_dev(T, 64, dtype=F32))
    bad(ARG, x=_dev(64, T).t())
    bad(ARG, x=_dev(T + 1, 64))
    bad(ARG, y=_dev(T, 40, dtype=torch.bfloat16))
    bad(ARG, y=torch.zeros(T, 40, dtype=F16))
    bad(SHAPE, y=_dev(1, 40).expand(T, 40))
    bad(ARG, a=_dev(3, 64))
    bad(ARG, a=_dev(3, 8, 72))
    bad(ARG, a=_dev(3, 64, 8).transpose(1, 2))
    bad(ARG, b=_dev(3, 8, 40))
    bad(ARG, b=_dev(2, 40, 8))
    bad(ARG, scales=_dev(3))
    bad(ARG, offsets=_dev(3, dtype=I32))
    bad(ARG, rows=_dev(T + 1, dtype=I32))
    bad(ARG, rows=_dev(T, dtype=torch.int64))
    bad(ARG, out=_dev(T, 48))
    bad(SHAPE, out=_dev(1, 40).expand(T, 40))
    _rejects(stub, ARG, Q.lora_group, _dev(T, dtype=torch.int64), 3)
    _rejects(stub, ARG, Q.lora_group, _dev(T, 1, dtype=I32), 3)
    _rejects(stub, ARG, Q.lora_group, torch.zeros(T, dtype=I32), 3)
    _rejects(stub, SHAPE, Q.lora_group, _dev(T, dtype=I32), 0)
    _rejects(stub, SHAPE, Q.lora_group, _dev(T, dtype=I32), 513)


def test_abi_rotary_and_cache():
    L = Q.lib()

    def rot(x=A, dt=0, xt=512, xh=64, t=4, h=8, d=64, pos=A, f=A, r=64, out=A, ot=512, oh=64):
        return L.quick_rotary(x, dt, xt, xh, t, h, d, pos, f, r, 0, 0, 1.0, out, ot, oh, None)
    assert rot(t=0) == OK
    assert rot(dt=3) == rot(dt=-1) == rot(x=0) == rot(out=0) == rot(pos=0) == rot(f=0) == ARG
    assert rot(t=-1) == rot(t=1 << 24) == rot(h=0) == rot(h=65536) == rot(d=0) == rot(d=4097) == SHAPE
    assert rot(r=3) == rot(r=66) == rot(r=-2) == rot(xt=-8) == rot(oh=1 << 40) == SHAPE
    assert rot(x=A + 1) == rot(out=A + 1) == rot(pos=A + 2) == rot(f=A + 4) == ALIGN and rot(x=A + 2, dt=2) == ALIGN

    def write(k=A, v=A, dt=0, kt=512, kh=64, vt=512, vh=64, s=A, t=4, h=8, d=64, c=A, p=10):
        return L.quick_kv4_write(k, v, dt, kt, kh, vt, vh, s, t, h, d, c, p, None)

    def read(c=A, p=10, s=A, t=4, h=8, d=64, dt=0, k=A, v=A):
        return L.quick_kv4_read(c, p, s, t, h, d, dt, k, v, None)
    assert write(t=0) == read(t=0) == read(k=None, v=None) == OK
    assert write(dt=2) == write(k=0) == write(v=0) == write(s=0) == write(c=0) == ARG
    assert read(dt=3) == read(s=0) == read(c=0) == ARG
    for f in (write, read):
        assert f(t=-1) == f(t=1 << 24) == f(h=0) == f(h=1025) == f(p=0) == f(p=1 << 25) == SHAPE
        assert f(d=96) == f(d=0) == f(d=512) == UNSUP
        assert f(t=(1 << 24) - 1, h=1024, d=256) == SHAPE
        assert f(s=A + 2) == f(c=A + 8) == f(k=A + 8) == f(v=A + 2) == ALIGN
    assert write(kt=516) == write(kh=4) == write(vt=511) == write(vh=9) == ALIGN
    assert write(kt=-8) == write(vh=1 << 40) == SHAPE


def test_abi_attention():
    L = Q.lib()
    base = dict(T=6, q_heads=8, heads=2, D=64, pages=9, seqs=3, table_width=100, most=2, q_token=512, q_head=64, window=0,
                causal=1, scale=1.0)

    def struct(**k):
        return Q.attention.QuickAttention(*[{**base, **k}[n] for n, _ in Q.attention.QuickAttention._fields_])

    def attn(q=A, dt=0, c=A, tab=A, ln=A, off=A, out=A, lse=None, ws=A, wsb=1 << 30, **k):
        return L.quick_kv4_attention(ctypes.byref(struct(**k)), q, dt, c, tab, ln, off, out, lse, ws, wsb, None)
    assert attn(T=0) == attn(seqs=0) == OK
    assert L.quick_kv4_attention(None, A, 0, A, A, A, A, A, None, A, 1 << 30, None) == ARG
    assert attn(dt=2) == attn(q=0) == attn(c=0) == attn(tab=0) == attn(ln=0) == attn(out=0) == ARG
    for k in (dict(T=-1), dict(T=1 << 24), dict(heads=0), dict(heads=1025, q_heads=1025), dict(q_heads=1), dict(q_heads=9),
              dict(q_heads=130), dict(pages=0), dict(pages=1 << 25), dict(seqs=-1), dict(seqs=4097), dict(table_width=-1),
              dict(table_width=1 << 24), dict(most=0), dict(window=-1), dict(window=5, causal=0), dict(q_token=-8),
              dict(q_head=1 << 40), dict(T=(1 << 24) - 1, heads=1024, q_heads=1 << 16)):
        assert attn(**k) == SHAPE, k
        assert L.quick_kv4_attention_workspace_bytes(ctypes.byref(struct(**k))) == 0
    assert attn(D=96) == attn(D=0) == UNSUP
    assert attn(q=A + 8) == attn(c=A + 4) == attn(out=A + 8) == attn(tab=A + 2) == attn(ln=A + 1) == attn(off=A + 2) == ALIGN
    assert attn(lse=A + 2) == attn(q_token=516) == attn(q_head=63) == attn(ws=A + 8) == ALIGN
    for k in ({}, dict(most=20), dict(most=1 << 40), dict(T=5000, most=5000)):
        need = L.quick_kv4_attention_workspace_bytes(ctypes.byref(struct(**k)))
        assert need > 0 and attn(wsb=need - 1, **k) == attn(ws=None, **k) == WORK
    # short tables need none
    assert L.quick_kv4_attention_workspace_bytes(ctypes.byref(struct(table_width=16))) == 0
    assert L.quick_kv4_attention_workspace_bytes(None) == 0


def test_abi_lora():
    L = Q.lib()
    assert L.quick_lora_group(A, -1, 3, A, A, None) == L.quick_lora_group(A, 1 << 24, 3, A, A, None) == SHAPE
    assert L.quick_lora_group(A, 5, 0, A, A, None) == L.quick_lora_group(A, 5, 513, A, A, None) == SHAPE
    assert L.quick_lora_group(0, 5, 3, A, A, None) == L.quick_lora_group(A, 5, 3, 0, A, None) == ARG
    assert L.quick_lora_group(A, 5, 3, A, 0, None) == L.quick_lora_group(0, 0, 3, 0, 0, None) == ARG
    assert L.quick_lora_group(A + 2, 5, 3, A, A, None) == L.quick_lora_group(A, 5, 3, A, A + 1, None) == ALIGN

    def add(x=A, ldx=64, dt=0, t=6, k=64, n=40, e=3, r=8, a=A, b=A, s=None, off=A, rows=A, R=6, y=A, ldy=40, out=2 * A,
            ldo=40, ws=A, wsb=1 << 30):
        return L.quick_lora_add(x, ldx, dt, t, k, n, e, r, a, b, s, off, rows, R, y, ldy, out, ldo, ws, wsb, None)
    assert add(R=0) == add(t=0, R=0) == OK
    assert add(dt=2) == add(x=0) == add(a=0) == add(b=0) == add(off=0) == add(rows=0) == add(y=0) == add(out=0) == ARG
    assert add(out=A, ldo=48) == ARG
    assert add(t=-1) == add(t=1 << 24) == add(R=7) == add(R=-1) == add(k=4) == add(k=68) == add(k=1 << 21) == SHAPE
    assert add(n=0) == add(n=44) == add(e=0) == add(e=513) == add(r=0) == add(r=12) == add(r=136) == SHAPE
    assert add(ldx=56) == add(ldy=32) == add(ldo=1 << 40) == SHAPE
    assert add(x=A + 8) == add(a=A + 2) == add(b=A + 8) == add(y=A + 4) == add(out=A + 8) == add(s=A + 2) == ALIGN
    assert add(off=A + 2) == add(rows=A + 1) == add(ldx=68) == add(ldy=44) == add(ldo=42) == add(ws=A + 4) == ALIGN
    need = Q.lora_workspace_bytes(6, 64, 3, 8)
    assert need >= 6 * 8 * 4 and add(wsb=need - 1) == add(ws=None) == WORK
    assert Q.lora_workspace_bytes(0, 64, 3, 8) == Q.lora_workspace_bytes(6, 64, 0, 8) == 0


def test_headers_compile_as_plain_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "quick_attention.h"\n#include "quick_lora.h"\nint main(void) {\n'
                   "    quick_attention_t a = {4, 8, 2, 128, 10, 4, 3, 1, 1024, 128, 0, 1, 1.0f};\n"
                   "    if (quick_kv4_attention(&a, 0, QUICK_F16, 0, 0, 0, 0, 0, 0, 0, 0, 0) != QUICK_ERR_INVALID_ARG) return 1;\n"
                   "    if (quick_lora_workspace_bytes(4, 64, 2, 8) == 0) return 2;\n"
                   "    return QUICK_KV4_PAGE == 64 && QUICK_LORA_MAX_RANK == 128 ? 0 : 3;\n}\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "t")
    libdir = os.path.dirname(Q.LIB_PATH)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", exe,
                    os.path.join(libdir, "libquick.so"), "-Wl,-rpath," + libdir], check=True)
    assert subprocess.run([exe]).returncode == 0
    assert (Q.KV4_PAGE, Q.LORA_MAX_RANK) == (64, 128)


def test_abi_most_workgroups_of_the_cache():
    """As many tokens and heads as the header says, and no more."""
    L = Q.lib()
    for d in (64, 128, 256):
        t = (1 << 24) // 1024 * (2048 // d)        # one workgroup too many
        assert L.quick_kv4_write(A, A, 0, 0, 0, 0, 0, A, t, 1024, d, A, 10, None) == SHAPE
        assert L.quick_kv4_read(A, 10, A, t, 1024, d, 0, A, A, None) == SHAPE
        assert L.quick_kv4_write(A, A, 0, 0, 0, 0, 0, A, t - 2048 // d + 1, 1024, d, A, 10, None) == SHAPE
