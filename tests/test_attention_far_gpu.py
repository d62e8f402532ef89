"""Attention over the paged 4-bit cache at the ends of its numbers: scores far
from zero, against the binary64 form.  Every score is exact in binary32 (one
channel of q and k is not zero), so a row's weights are as exact as the scores'
differences are, however far the scores lie."""
import math

import pytest
import torch

import attn_util as A
import paper_2402_10076_amd as Q
from gpu_util import say

pytestmark = pytest.mark.gpu

# (D, heads, group, lengths, new, width): by a wave's pages, 16 columns and 32, whole and shared out; through LDS, 128
# columns and 256; the last ones over many workgroups
FORMS = [(64, 2, 4, [300, 70], [1, 1], None), (128, 2, 8, [300, 1, 64], [1, 1, 1], None), (256, 1, 4, [300, 9], [4, 2], None),
         (128, 1, 8, [300, 200], [4, 3], None), (64, 1, 4, [300, 200], [8, 3], 70), (128, 2, 4, [4400, 200], [2, 1], 70),
         (128, 1, 16, [2400, 200], [8, 3], 70), (256, 1, 16, [1400, 200], [2, 3], 70), (64, 1, 8, [300, 70], [100, 20], None),
         (128, 2, 8, [900, 70], [40, 20], None), (256, 1, 8, [300, 170], [40, 20], None), (64, 1, 8, [400, 70], [300, 20], None),
         (128, 1, 8, [900, 70], [300, 20], None)]


class Exact:
    """Keys of one channel that are a power of two or one and a half times it, queries of that channel that differ from
    head to head, normal values."""

    def __init__(self, D, heads, group, lengths, new, width, dtype, q_values, order, top):
        g = A.gen(51, D, heads, group, sum(lengths))
        self.dtype, self.group, self.lengths = A.TYPES[dtype], group, lengths
        need = [-(-n // 64) for n in lengths]
        ids = torch.randperm(sum(need) + 1, generator=g)
        self.table = torch.zeros((len(lengths), width or max(need)), dtype=torch.int32)
        self.cache = Q.kv4_cache(sum(need) + 1, heads, D)
        self.k, self.v = [], []
        at = 0
        for b, n in enumerate(lengths):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
            # sizes from 2^-6 to 2^top over the sequence, in runs of equal ones
            size = (torch.arange(n) * (2 * (top + 6) + 1) // max(n, 1)) - 12
            if order == "falling":
                size = size.flip(0)
            elif order == "mixed":
                size = size[torch.randperm(n, generator=g)]
            value = torch.where(size % 2 == 0, 1.0, 1.5) * 2.0 ** torch.div(size, 2, rounding_mode="floor")
            k = torch.zeros(n, heads, D)
            k[:, :, D - 3] = value.view(-1, 1)
            k, v = k.to(self.dtype), A.normal(g, n, heads, D, dtype=self.dtype)
            t = torch.arange(n)
            slots = (self.table[b, t // 64].long() * 64 + t % 64).to(torch.int32)
            Q.kv4_write(self.cache, k.cuda(), v.cuda(), slots.cuda())
            self.k.append(A.rounded(k))
            assert torch.equal(self.k[b], k.double())
            self.v.append(A.rounded(v))
        self.offsets = [0]
        for n in new:
            self.offsets.append(self.offsets[-1] + n)
        self.q = torch.zeros(self.offsets[-1], heads * group, D, dtype=self.dtype)
        pick = torch.tensor(q_values)[torch.arange(heads * group) * 7 % len(q_values)]
        self.q[:, :, D - 3] = pick.to(self.dtype)
        self.most = max(new)

    def check(self, scale, window=0):
        off = torch.tensor(self.offsets, dtype=torch.int32).cuda()
        lse = torch.zeros(self.q.shape[:2], device="cuda")
        out = Q.kv4_attention(self.q.cuda(), self.cache, self.table.cuda(), torch.tensor(self.lengths, dtype=torch.int32).cuda(),
                              offsets=off, most=self.most, scale=scale, window=window, lse=lse).cpu().double()
        args = self.lengths, self.offsets, self.group, self.dtype, scale, window
        want, want_lse, _ = A.attention(self.q.double(), self.k, self.v, *args)
        size, _, _ = A.attention(self.q.double(), self.k, [v.abs() for v in self.v], *args)
        assert out.isfinite().all(), "%d of %d rows" % ((~out.isfinite()).any(2).sum(), out.shape[0] * out.shape[1])
        # A weight's exponent, of 64 at most where it counts, is rounded once (2^-19) and its reference's changes once a
        # page; the scale's rounding counts for the score's distance from the largest (64 * 2^-23); weights and sums as
        # elsewhere (half a step of the type; 2^-23 a token), f16's below its normal range too.
        step, n = A.STEP[self.dtype], max(self.lengths)
        far = (2.0 ** -19 * (n // 64 + 8) + 2.0 ** -17) * math.log(2)
        tol = size * (step + 2 * far + n * 2.0 ** -23) + n * 2.0 ** -31 * 6 + want.abs() * step + 2.0 ** -25
        err = (out - want).abs()
        assert bool((err <= tol).all()), "err %.3g, of the bound %.3g" % (float(err.max()), float((err / tol).max()))
        err = (lse.cpu().double() - want_lse).abs()
        assert bool((err <= want_lse.abs() * 2.0 ** -21 + 2.0 ** -12).all()), float(err.max())


@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f[:3])) + "-%d-%d" % (f[3][0], f[4][0]))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_scores_far_from_zero(dtype, form, order):
    """Up to 2^30 (bfloat16: 2^72) of either sign, beside heads of ordinary ones, whose references move meanwhile."""
    say("far scores", dtype, form, order)
    q = [2.0 ** 14, 1.0, -(2.0 ** 13), 2.0 ** -3, 2.0 ** 10, -0.25, 0.0] if dtype == "f16" else \
        [2.0 ** 58, 1.0, -(2.0 ** 13), 2.0 ** -3, 2.0 ** 10, -(2.0 ** 57), 0.0]
    b = Exact(*form, dtype, q, order, 14)
    b.check(1.5)
    b.check(-1.0, window=150)


@pytest.mark.parametrize("form", FORMS[:2] + FORMS[7:10] + FORMS[-1:], ids=lambda f: "-".join(map(str, f[:3])))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_equal_scores_far_from_zero(dtype, form):
    """Every token's weight is the same, whatever the score: its product with the scale is not a binary32 number."""
    say("equal scores", dtype, form)
    b = Exact(*form, dtype, [1.5 * 2.0 ** e for e in range(-2, 14, 2)], "mixed", -6)
    for scale in (0.3, 1e3, -7e5, 3e8, 1e20):
        b.check(scale)


@pytest.mark.parametrize("exponent", [-90, 120])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f[:3])) + "-%d-%d" % (f[3][0], f[4][0]))
def test_values_far_from_one(form, exponent):
    """bfloat16 values near the ends of binary32: a row is a mean of them, and so are the sums of it that are held."""
    D, heads, group, lengths, new, width = form
    say("far values", form, exponent)
    g = A.gen(52, D, heads, sum(lengths))
    dtype, need = torch.bfloat16, [-(-n // 64) for n in lengths]
    table = torch.zeros((len(lengths), width or max(need)), dtype=torch.int32)
    cache, at, ks, vs, offsets = Q.kv4_cache(sum(need), heads, D), 0, [], [], [0]
    for b, n in enumerate(lengths):
        table[b, :need[b]] = torch.arange(at, at + need[b])
        k, v = A.normal(g, n, heads, D, dtype=dtype), (torch.randn(n, heads, D, generator=g) * 2.0 ** exponent).to(dtype)
        Q.kv4_write(cache, k.cuda(), v.cuda(), torch.arange(at * 64, at * 64 + n, dtype=torch.int32).cuda())
        at += need[b]
        ks.append(A.rounded(k))
        vs.append(A.rounded(v))
        offsets.append(offsets[-1] + new[b])
    q = A.normal(g, offsets[-1], heads * group, D, scale=1.5, dtype=dtype)
    out = Q.kv4_attention(q.cuda(), cache, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(),
                          offsets=torch.tensor(offsets, dtype=torch.int32).cuda(), most=max(new)).cpu().double()
    want, _, tol = A.attention(q.double(), ks, vs, lengths, offsets, group, dtype)
    err = (out - want).abs()
    assert bool((err <= tol).all()), "err %.3g, of the bound %.3g" % (float(err.max()), float((err / tol).max()))


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f[:3])) + "-%d-%d" % (f[3][0], f[4][0]))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_blocks_beyond_the_type(dtype, form):
    """A key or value block whose scale q's type cannot hold (of a cache that bfloat16 wrote, or of no writer) is NaN
    for the rows that see it, in its channels or in all where it is a key's, and nothing for the others."""
    D, heads, group, lengths, new, width = form
    say("beyond the type", dtype, form)
    g = A.gen(53, D, heads, sum(lengths))
    need = [-(-n // 64) for n in lengths]
    table = torch.zeros((len(lengths), width or max(need)), dtype=torch.int32)
    cache, at, offsets = Q.kv4_cache(sum(need), heads, D), 0, [0]
    for b, n in enumerate(lengths):
        table[b, :need[b]] = torch.arange(at, at + need[b])
        Q.kv4_write(cache, *(A.normal(g, n, heads, D, dtype=torch.bfloat16).cuda() for _ in "kv"),
                    torch.arange(at * 64, at * 64 + n, dtype=torch.int32).cuda())
        at += need[b]
        offsets.append(offsets[-1] + new[b])
    q = A.normal(g, offsets[-1], heads * group, D, scale=1.5, dtype=A.TYPES[dtype])
    args = q.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()

    def run(c, **kw):
        return Q.kv4_attention(args[0], c, *args[1:], offsets=torch.tensor(offsets, dtype=torch.int32).cuda(), most=max(new),
                               **kw).cpu()

    least, most = (141, 254) if dtype == "f16" else (253, 254)
    token, block = lengths[0] - 1 - new[0] // 2, D // 32 - 1       # seen by some of the first sequence's rows
    t = token % 64
    key = 32 * D + 64 * block + 4 * (t % 16) + t // 16
    value = 66 * D + 64 * block + 16 * (t % 16 // 4) + 4 * (t // 16) + t % 4
    for window in (0, 5):
        ref = run(cache, window=window)
        assert ref.isfinite().all()
        for where, scales in ((key, (least, most)), (value, (least, most))):
            for scale in scales:
                for h in (0, heads - 1):
                    bad = cache.clone()
                    bad[token // 64, h, where] = scale
                    out = run(bad, window=window)
                    for row in range(offsets[-1]):
                        pos = lengths[0] - new[0] + row
                        sees = row < new[0] and pos >= token and (not window or token > pos - window)
                        nan = torch.zeros_like(out[row], dtype=torch.bool)
                        if sees:
                            nan[h * group:(h + 1) * group, 0 if where == key else 32 * block:] = True
                        assert torch.equal(out[row].isnan(), nan), (where == key, scale, h, row, window)
                        same = torch.ones_like(nan[:, 0])
                        if sees:
                            same[h * group:(h + 1) * group] = False
                        assert torch.equal(out[row][same], ref[row][same]), (where == key, scale, h, row, window)
    # the largest scale that the type holds is one
    held = cache.clone()
    held[token // 64, 0, value] = least - 1
    assert run(held).isfinite().all()


@pytest.mark.parametrize("form", [FORMS[1], FORMS[5], FORMS[9], FORMS[12]], ids=lambda f: "-".join(map(str, f[:3])))
def test_replayed_with_near_and_far_scores(form):
    """A captured call, replayed with queries whose scores are near, far and near again: the bits of eager calls."""
    D, heads, group, lengths, new, width = form
    say("replayed", form)
    g = A.gen(54, D, heads)
    need = [-(-n // 64) for n in lengths]
    table = torch.zeros((len(lengths), width or max(need)), dtype=torch.int32)
    cache, at, offsets = Q.kv4_cache(sum(need), heads, D), 0, [0]
    for b, n in enumerate(lengths):
        table[b, :need[b]] = torch.arange(at, at + need[b])
        Q.kv4_write(cache, *(A.normal(g, n, heads, D).cuda() for _ in "kv"), torch.arange(at * 64, at * 64 + n, dtype=torch.int32).cuda())
        at += need[b]
        offsets.append(offsets[-1] + new[b])
    q = A.normal(g, offsets[-1], heads * group, D, scale=1.5).cuda()
    far = q.clone()
    far[::2, ::3] *= 8192.0
    table, ln, off = table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), torch.tensor(offsets, dtype=torch.int32).cuda()
    at = q.clone()

    def run():
        return Q.kv4_attention(at, cache, table, ln, offsets=off, most=max(new), scale=1e3)
    want = {}
    for name, x in (("near", q * 1e-3), ("far", far)):
        at.copy_(x)
        want[name] = run()
    assert want["far"].isfinite().all() and not torch.equal(want["near"], want["far"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for name, x in (("near", q * 1e-3), ("far", far), ("near", q * 1e-3), ("far", far), ("near", q * 1e-3)):
        at.copy_(x)
        out.fill_(7)
        graph.replay()
        assert torch.equal(out, want[name]), name
        assert torch.equal(run(), want[name]), name
