"""Low-rank adapters of many requests (include/quick_lora.h) on the GPU
against the binary64 form."""
import numpy as np
import pytest
import torch

import attn_util as A
import paper_2402_10076_amd as Q
from gpu_util import say

pytestmark = pytest.mark.gpu


def _group(ids, E):
    to = np.where((ids >= 0) & (ids < E), ids, E)
    rows = np.argsort(to, kind="stable")
    return np.concatenate([[0], np.cumsum(np.bincount(to, minlength=E + 1))])[:E + 1], rows


@pytest.mark.parametrize("T,E", [(0, 3), (1, 1), (5, 1), (64, 7), (65, 512), (1000, 33), (5000, 3), (40000, 200)])
def test_group(T, E):
    ids = torch.randint(-2, E + 2, (T,), generator=A.gen(1, T, E), dtype=torch.int32)
    say("group", T, E)
    offsets, rows = Q.lora_group(ids.cuda(), E)
    want = _group(ids.numpy(), E)
    assert np.array_equal(offsets.cpu().numpy(), want[0]) and np.array_equal(rows.cpu().numpy(), want[1])


def test_group_extremes():
    for ids in ([-1] * 70, [0] * 70, [6] * 70, [-(1 << 31), (1 << 31) - 1, 2, 7, 6]):
        offsets, rows = Q.lora_group(torch.tensor(ids, dtype=torch.int32).cuda(), 7)
        want = _group(np.array(ids), 7)
        assert np.array_equal(offsets.cpu().numpy(), want[0]) and np.array_equal(rows.cpu().numpy(), want[1])


def _case(seed, T, K, N, E, r, dtype, bare=True):
    g = A.gen(seed, T, K, N, E, r)
    dt = A.TYPES[dtype]
    x, y = A.normal(g, T, K, dtype=dt), A.normal(g, T, N, dtype=dt)
    a, b = A.normal(g, E, r, K, scale=K ** -0.5, dtype=dt), A.normal(g, E, N, r, scale=0.5 * r ** -0.5, dtype=dt)
    ids = torch.randint(-1 if bare else 0, E, (T,), generator=g, dtype=torch.int32)
    return x, y, a, b, ids, torch.rand(E, generator=g) + 0.5


def _check(out, x, y, a, b, ids, scales):
    want, tol = A.adapters(y, x, a, b, ids, scales, x.dtype)
    err = (out.cpu().double() - want).abs()
    assert bool((err <= tol).all()), "err %.3g, of the bound %.3g" % (float(err.max()), float((err / tol).max()))


CASES = [(1, 64, 64, 1, 8), (1, 4096, 520, 3, 16), (27, 512, 1000, 8, 16), (5, 8, 8, 2, 24), (16, 136, 264, 1, 32),
         (33, 1032, 256, 40, 8), (100, 256, 72, 2, 40), (130, 520, 640, 2, 64), (70, 2056, 48, 1, 128),
         (300, 384, 328, 5, 16), (257, 200, 120, 3, 104), (64, 128, 16, 512, 8), (200, 320, 264, 4, 48)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,K,N,E,r", CASES)
def test_add(T, K, N, E, r, dtype):
    x, y, a, b, ids, scales = _case(2, T, K, N, E, r, dtype)
    say("lora", T, K, N, E, r, dtype)
    dev = [t.cuda() for t in (x, a, b)]
    plan = Q.lora_group(ids.cuda(), E)
    yd = y.cuda()
    out = Q.lora_add(yd, *dev, *plan, scales=scales.cuda())
    assert torch.equal(yd.cpu(), y)
    _check(out, x, y, a, b, ids, scales)
    assert torch.equal(out.cpu()[ids < 0], y[ids < 0])
    assert torch.equal(Q.lora_add(yd, *dev, *plan, scales=scales.cuda(), out=yd), out)
    _check(Q.lora_add(y.cuda(), *dev, *plan), x, y, a, b, ids, None)


@pytest.mark.parametrize("T", [9, 200])
def test_strided_rows(T):
    """Columns of a wider projection, in place, beside others that stay; x with a row stride."""
    x, y, a, b, ids, scales = _case(3, T, 256, 200, 3, 16, "f16")
    plan = Q.lora_group(ids.cuda(), 3)
    ref = Q.lora_add(y.cuda(), x.cuda(), a.cuda(), b.cuda(), *plan)
    wide = torch.full((T, 512), 9.0, dtype=torch.float16, device="cuda")
    wide[:, 8:208] = y.cuda()
    xs = torch.zeros((T, 264), dtype=torch.float16, device="cuda")
    xs[:, 8:] = x.cuda()
    part = wide[:, 8:208]
    Q.lora_add(part, xs[:, 8:], a.cuda(), b.cuda(), *plan, out=part)
    assert torch.equal(part, ref) and bool((wide[:, :8] == 9).all()) and bool((wide[:, 208:] == 9).all())


def test_one_adapter_has_all_the_rows():
    """Adapters without a row, and one with all: more rows than their mean."""
    x, y, a, b, _, scales = _case(4, 150, 192, 136, 9, 24, "bf16")
    ids = torch.full((150,), 7, dtype=torch.int32)
    out = Q.lora_add(y.cuda(), x.cuda(), a.cuda(), b.cuda(), *Q.lora_group(ids.cuda(), 9), scales=scales.cuda())
    _check(out, x, y, a, b, ids, scales)


def test_rows_that_are_not_listed_and_broken_orders():
    T, E = 40, 3
    x, y, a, b, ids, scales = _case(5, T, 128, 64, E, 8, "f16", bare=False)
    offsets, rows = Q.lora_group(ids.cuda(), E)
    out = torch.full((T, 64), 3.0, dtype=torch.float16, device="cuda")
    few = rows[:25].contiguous()
    Q.lora_add(y.cuda(), x.cuda(), a.cuda(), b.cuda(), offsets.clamp(max=25), few, out=out)
    listed = torch.zeros(T, dtype=torch.bool)
    listed[few.cpu().long()] = True
    assert bool((out.cpu()[~listed] == 3).all())
    want, tol = A.adapters(y, x, a, b, ids, None, torch.float16)
    assert bool(((out.cpu().double() - want).abs() <= tol)[listed].all())
    for o in ([-3, 50, 2, 1 << 30], [40, 30, 20, 10], [-(1 << 31)] * 4):
        Q.lora_add(y.cuda(), x.cuda(), a.cuda(), b.cuda(), torch.tensor(o, dtype=torch.int32).cuda(), rows)
    wild = rows.clone()
    wild[::3] = torch.tensor([-1, T, 1 << 30, -(1 << 31), (1 << 31) - 1] * 3, dtype=torch.int32).cuda()[:wild[::3].numel()]
    out = torch.full((T, 64), 3.0, dtype=torch.float16, device="cuda")
    Q.lora_add(y.cuda(), x.cuda(), a.cuda(), b.cuda(), offsets, wild, out=out)
    torch.cuda.synchronize()
    listed[:] = False
    listed[[int(r) for r in wild.cpu() if 0 <= r < T]] = True
    assert bool((out.cpu()[~listed] == 3).all())


def test_nan_stays_in_its_row_and_column():
    """A NaN of x makes NaN of its token alone, one of B of its column alone."""
    for r in (8, 16, 32):
        x, y, a, b, _, _ = _case(6, 20, 128, 136, 2, r, "f16")
        ids = (torch.arange(20) % 2).to(torch.int32)
        x[3, 7] = float("nan")
        b[0, 100, 5] = float("inf")
        out = Q.lora_add(y.cuda(), x.cuda(), a.cuda(), b.cuda(), *Q.lora_group(ids.cuda(), 2)).cpu()
        bad = ~out.isfinite()
        want = torch.zeros_like(bad)
        want[3] = True
        want[ids == 0, 100] = True
        assert torch.equal(bad, want)


def test_nothing_to_do():
    e = torch.empty((0, 64), dtype=torch.float16, device="cuda")
    a, b = torch.zeros((2, 8, 64), dtype=torch.float16, device="cuda"), torch.zeros((2, 64, 8), dtype=torch.float16, device="cuda")
    o, r = Q.lora_group(torch.empty(0, dtype=torch.int32, device="cuda"), 2)
    assert not o.any() and Q.lora_add(e, e, a, b, o, r).shape == (0, 64)


@pytest.mark.parametrize("T,K,N,E,r", [(400, 2600, 1096, 3, 72), (512, 5128, 328, 2, 64), (192, 9000, 72, 1, 8), (49, 9000, 136, 1, 120)])
def test_many_slices(T, K, N, E, r):
    """Many channels for few tiles: slices of them that the second product adds up, the last one short."""
    x, y, a, b, ids, scales = _case(9, T, K, N, E, r, "bf16")
    say("slices", T, K, N, E, r)
    out = Q.lora_add(y.cuda(), x.cuda(), a.cuda(), b.cuda(), *Q.lora_group(ids.cuda(), E), scales=scales.cuda())
    _check(out, x, y, a, b, ids, scales)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("few", [0, 1, 25])
@pytest.mark.parametrize("given", [False, True], ids=["current stream", "given stream"])
def test_rows_that_a_new_result_has_and_the_call_does_not_list(given, few, dtype):
    """They are y's, whatever the new tensor's memory held."""
    T, E, N = 40, 3, 64
    x, y, a, b, ids, _ = _case(10, T, 128, N, E, 8, dtype, bare=False)
    offsets, rows = Q.lora_group(ids.cuda(), E)
    dev = [t.cuda() for t in (x, a, b)]
    wide = torch.zeros((T, N + 8), dtype=x.dtype, device="cuda")
    wide[:, 8:] = y.cuda()
    stream = torch.cuda.Stream() if given else torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        left = torch.full((T, N), float("nan"), dtype=x.dtype, device="cuda")     # what the next block of this size holds
        del left
    torch.cuda.synchronize()
    out = Q.lora_add(wide[:, 8:], *dev, offsets.clamp(max=few), rows[:few].contiguous(), stream=stream if given else None)
    torch.cuda.synchronize()
    listed = torch.zeros(T, dtype=torch.bool)
    listed[rows[:few].cpu().long()] = True
    assert torch.equal(out.cpu()[~listed], y[~listed])
    _check(out, x, y, a, b, torch.where(listed, ids, -1), None)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,K,N,E,r", [(27, 512, 1000, 8, 64), (27, 520, 328, 8, 128), (20, 1032, 136, 3, 40), (30, 264, 72, 4, 104),
                                       (20, 128, 264, 2, 72), (300, 384, 328, 3, 32), (200, 520, 136, 2, 24), (500, 264, 72, 4, 48),
                                       (160, 256, 136, 2, 96), (1, 4096, 264, 16, 56), (16, 72, 4096, 1, 120)])
def test_every_rank_with_low_and_high_tiles(T, K, N, E, r, dtype):
    """A few tokens of many adapters of high ranks, many of low ones."""
    x, y, a, b, ids, scales = _case(11, T, K, N, E, r, dtype)
    say("ranks", T, K, N, E, r, dtype)
    dev = [t.cuda() for t in (x, a, b)]
    plan = Q.lora_group(ids.cuda(), E)
    yd = y.cuda()
    out = Q.lora_add(yd, *dev, *plan, scales=scales.cuda())
    _check(out, x, y, a, b, ids, scales)
    assert torch.equal(out.cpu()[ids < 0], y[ids < 0])
    assert torch.equal(Q.lora_add(yd, *dev, *plan, scales=scales.cuda(), out=yd), out)


@pytest.mark.parametrize("T", [20, 200])
@pytest.mark.parametrize("r", [24, 32, 40, 64, 72, 128])
def test_nan_stays_in_its_row_and_column_whatever_the_rank(r, T):
    """A NaN of x makes NaN of its token alone, an infinity of B of its column of its adapter alone, one of A of all of
    its adapter's tokens and columns."""
    x, y, a, b, _, _ = _case(12, T, 136, 200, 2, r, "bf16")
    ids = (torch.arange(T) % 3 - 1).to(torch.int32)
    plan = Q.lora_group(ids.cuda(), 2)

    def bad(x, a, b):
        return ~Q.lora_add(y.cuda(), x.cuda(), a.cuda(), b.cuda(), *plan).cpu().isfinite()
    row, last = 4, 199     # (of adapter 0)
    for place in ((0, 0), (135, r - 1)):
        x1, a1, b1 = x.clone(), a.clone(), b.clone()
        x1[row, place[0]] = float("nan")
        want = torch.zeros(T, 200, dtype=torch.bool)
        want[row] = True
        assert torch.equal(bad(x1, a, b), want)
        b1[0, last, place[1]] = float("inf")
        want = torch.zeros(T, 200, dtype=torch.bool)
        want[ids == 0, last] = True
        assert torch.equal(bad(x, a, b1), want)
        a1[1, place[1], place[0]] = float("nan")
        want = (ids == 1).view(-1, 1).expand(T, 200)
        assert torch.equal(bad(x, a1, b), want)
