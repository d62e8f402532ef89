"""The choice of a microscaled product's form, on the CPU."""
import subprocess

import numpy as np

import mx_plan
import paper_2402_10076_amd as Q

# Every form in turn made the cheapest of all, and put at every place of the
# table: the choice has to be a form that is built for the call.
TABLES = mx_plan.HEAD + r"""
int main()
{
    long bad = 0, chosen = 0;
    for (int cheap = 0; cheap < kFormCount; cheap++)
        for (int first = 0; first < kFormCount; first++) {
            Form t[kFormCount];
            for (int i = 0; i < kFormCount; i++) {
                t[i] = kForms[(i + first) % kFormCount];
                if ((i + first) % kFormCount == cheap) t[i] = {t[i].bm, t[i].bn, 0, 0, 0, 0, 1e9f, 0};
            }
            for (int64_t M : {1, 4, 40, 300, 3000})
                for (int64_t K : {32, 512, 4128, 8192})
                    for (int64_t N : {32, 4096, 57344})
                        for (int how = 0; how < 6; how++) {
                            // dense, gated, grouped, grouped and gated, 16-bit activations, the same gated
                            const bool x16 = how > 3;
                            if (x16 && M > 4) continue;
                            const MxSizes s = {M, N, K, how / 2 == 1 ? 8 : 1, how / 2 == 1, how % 2 == 1, x16};
                            const Form& f = t[choose_form(t, s)];
                            bad += (K % 128 && f.bm * f.bn == 256 * 256) || (s.gated && f.bn < 32) ||
                                   (x16 && (f.bm != 16 || f.bn > 32));
                            const Form& c = kForms[cheap];
                            chosen += f.bm == c.bm && f.bn == c.bn;
                        }
        }
    const MxSizes none = {1, 32, 32, 8, true, false, true};
    std::printf("%ld wrong, %ld chosen\n", bad, chosen);
    return bad != 0 || chosen == 0 || plan_product(none).form != -1;
}
"""


def test_only_forms_that_are_built_are_chosen(tmp_path):
    r = subprocess.run([mx_plan.program(tmp_path, TABLES, "tables")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_plans_are_within_what_the_kernels_are_built_for(tmp_path):
    """Over sizes of all kinds: no form without the call's tail or epilogue, no
    weights past the caches in tall tiles, a leading workgroup in dense tiled
    forms alone, and a grid that a stream form's launch accepts."""
    g = np.random.Generator(np.random.PCG64(1))
    sizes = []
    for _ in range(20000):
        grouped, gated, x16 = int(g.integers(2)), int(g.integers(2)), 0
        M = int(np.exp(g.uniform(0, np.log(1 << 22))))
        N = int(np.exp(g.uniform(0, np.log(60000))))
        N = -(-N // 32) * 32 if gated else N
        K = int(np.exp(g.uniform(0, np.log(900)))) * 32
        if M * K >= 1 << 33:
            continue
        if not grouped and M <= 4 and M * K <= 57344:
            x16 = int(g.integers(2))
        sizes.append((M, N, K, int(np.exp(g.uniform(0, np.log(513)))) if grouped else 1, grouped, gated, x16))
    for s, p in zip(sizes, mx_plan.plans(tmp_path, sizes)):
        M, N, K, E, grouped, gated, x16 = s
        assert 0 <= p["form"] < 10 and p["tail"] == (K % 128 != 0)
        assert not (p["tail"] and p["form"] == 9) and not (gated and p["form"] == 0) and not (x16 and p["form"] > 1)
        assert not (p["once"] and p["bm"] > 64) and not (p["lead"] and (grouped or p["form"] < 3))
        assert p["form"] > 2 or p["row_tiles"] <= 65535


def _accepted(s, p):
    """As the launches check a grid."""
    if p["form"] < 3:
        return p["row_tiles"] <= 65535
    return -(-(p["row_tiles"] + p["lead"]) * p["columns"] // 8) * 8 <= 1 << 22


def test_sizes_within_the_header_s_limits_are_accepted(tmp_path):
    g = np.random.Generator(np.random.PCG64(2))
    sizes, beyond = [], []
    for u in g.random((60000, 6)):
        grouped, gated = int(u[0] < 0.5), int(u[1] < 0.3)
        M, N, K = int((1 << 22) ** u[2]), int((1 << 24) ** u[3]), int((1 << 17) ** u[4]) * 32
        E = int(512 ** u[5]) if grouped else 1
        N = -(-N // 32) * 32 if gated else N
        if max(M, N) * K >= 1 << 33:
            continue
        within = (M // 32 + E) * (N + 128) <= 1 << 28 if grouped else (M + 64) * (N + 128) <= 1 << 34
        (sizes if within else beyond).append((M, N, K, E, grouped, gated, 0))
    # on the lines themselves
    for m in range(23):
        for k in (32, 512, 2048):
            n = min((1 << 34) // ((1 << m) + 64) - 128, 1 << 24, ((1 << 33) - 1) // k)
            if n > 0 and k << m < 1 << 33:
                sizes.append((1 << m, n, k, 1, 0, 0, 0))
            for e in (2, 64, 512):
                n = min((1 << 28) // ((1 << m) // 32 + e) - 128, 1 << 24, ((1 << 33) - 1) // k)
                if n > 0 and k << m < 1 << 33:
                    sizes.append((1 << m, n, k, e, 1, 0, 0))
    assert all(_accepted(s, p) for s, p in zip(sizes, mx_plan.plans(tmp_path, sizes)))
    # ... and past them some are not
    assert not all(_accepted(s, p) for s, p in zip(beyond, mx_plan.plans(tmp_path, beyond)))


def test_limits_of_the_calls():
    """The library's own answers at the limits of rows, before anything is launched."""
    L, a = Q.lib(), 0x10000

    def grouped(t, r, n=32, k=32, y=0):
        return L.quick_mxfp4_grouped_gemm(a, a, a, a, a, a, y, 0, t, r, 2, n, k, None, 0, None)

    def gemm(m, n=32, k=32):
        return L.quick_mxfp4_gemm(a, a, a, a, 0, 0, m, n, k, None, 0, None)
    # accepted: the next thing that is found wrong is the missing y
    assert gemm(1 << 22) == grouped(1 << 24, 1 << 22) == gemm(1, 1 << 24) == Q.QUICK_ERR_INVALID_ARG
    assert gemm((1 << 22) + 1) == grouped(1 << 24, (1 << 22) + 1) == Q.QUICK_ERR_SHAPE
    assert grouped((1 << 24) + 1, 1) == gemm(1, (1 << 24) + 1) == Q.QUICK_ERR_SHAPE
