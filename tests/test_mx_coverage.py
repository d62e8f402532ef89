"""Which forms of the microscaled products' kernels the GPU tests run, from
the library's own choice of a form (csrc/quick_mx_forms.h): all that it
reaches over sizes of every kind."""
import numpy as np

import mx_plan
import test_mx_coverage_gpu as C
import test_mx_forms_gpu as F

# as in the tests' own parameters
FORMS_ONCE = [(1, 57344, 8192), (16, 57344, 8224), (23, 57344, 8192), (64, 57344, 8224), (130, 57344, 8192)]


def _quarter(K):
    """How the scales of 512 channels end: whole, with a part that is whole steps of 128, or inside a step."""
    return "cut off" if K % 128 else "partial" if K % 512 else "whole"


def _body(bm, rows):
    """The kernel's body for a tile of that many rows: of the full height, half, or a quarter."""
    return 4 if bm >= 256 and rows <= bm // 4 else 2 if bm >= 128 and rows <= bm // 2 else 1


def _runs(size, plan, counts):
    """What a call runs: (form, body, scales' end, weights past the caches, over experts, gated)."""
    M, N, K, E, grouped, gated, x16 = size
    if x16:
        return {("quantises", plan["form"], _quarter(K) == "cut off", plan["once"], gated)}
    bm = plan["bm"]
    rows = {r for c in counts for r in ({bm} if c >= bm else set()) | ({c % bm} if c % bm else set())}
    if plan["lead"]:
        rows.add(1)
    return {(plan["form"], _body(bm, r), _quarter(K), plan["once"], grouped, gated) for r in rows}


def _dense(M, N, K, gated):
    return (M, N, K, 1, 0, gated, 0), [M]


def _tested():
    out = []
    for M, N, K in F.DENSE + FORMS_ONCE + C.DENSE + C.DENSE_ONCE:
        out += [_dense(M, N, K, gated) for gated in ((0, 1) if N % 32 == 0 else (0,))]
        if (M, N, K) not in FORMS_ONCE and M <= 4 and M * K <= 57344:
            out.append(((M, N, K, 1, 0, 0, 1), None))
    out += [((M, N, K, 1, 0, 1, 1), None) for M, N, K in C.ON_THE_WAY]
    grouped = F.GROUPED + [(C.skewed(E, R), N, K) for E, R, N, K in C.GROUPED + C.GROUPED_ONCE]
    for counts, N, K in grouped:
        out += [((sum(counts), N, K, len(counts), 1, gated, 0), counts) for gated in ((0, 1) if N % 32 == 0 else (0,))]
    return out


def _sizes(n):
    """Sizes of every kind, spread over the logarithm of their ranges."""
    g = np.random.Generator(np.random.PCG64(5))
    u = g.random((n, 8))

    def log(v, lo, hi):
        return int(np.exp(np.log(lo) + v * np.log(hi / lo)))
    for v in u:
        grouped, gated = int(v[0] < 0.5), int(v[1] < 0.4)
        M, N, K = log(v[2], 1, 5000), log(v[3], 16, 60000), log(v[4], 1, 900) * 32
        K = -(-K // 128) * 128 if v[5] < 0.6 else K
        N = -(-N // 32) * 32 if gated else N
        E = log(v[6], 2, 64) if grouped else 1
        x16 = int(not grouped and M <= 4 and M * K <= 57344 and v[7] < 0.5)
        if E * N * K > 9e9:
            continue
        # rows of experts that make a tile's every body
        counts = [256, 128, 64] if grouped and M >= 448 else [M]
        yield (M, N, K, E, grouped, gated, x16), counts


def _all_runs(folder, calls):
    calls = list(calls)
    runs = {}
    for (size, counts), plan in zip(calls, mx_plan.plans(folder, [s for s, _ in calls])):
        for key in _runs(size, plan, counts):
            runs.setdefault(key, size)
    return runs


def test_every_form_that_is_reached_is_tested(tmp_path):
    tested, reached = _all_runs(tmp_path, _tested()), _all_runs(tmp_path, _sizes(150000))
    left = {k: v for k, v in reached.items() if k not in tested}
    assert not left, "%d of %d: %s" % (len(left), len(reached), sorted(left.items(), key=str)[:20])
    # every form, each with every end of the scales that it is built for, dense and over experts, gated or not
    for form in range(10):
        for quarter in ("whole", "partial", "cut off"):
            for grouped in (0, 1):
                for gated in (0, 1):
                    if (form, gated) != (0, 1) and (form, quarter) != (9, "cut off"):
                        assert any(k[0] == form and k[2] == quarter and k[4:] == (grouped, gated) for k in tested
                                   if k[0] != "quantises"), (form, quarter, grouped, gated)


def test_lists_of_weights_past_the_caches(tmp_path):
    sizes = [(M, N, K, 1, 0, 0, 0) for M, N, K in C.DENSE_ONCE + FORMS_ONCE[:4]]
    sizes += [(sum(C.skewed(E, R)), N, K, E, 1, 0, 0) for E, R, N, K in C.GROUPED_ONCE]
    assert all(p["once"] for p in mx_plan.plans(tmp_path, sizes))
