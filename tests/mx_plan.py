"""The library's choice of a form for microscaled products, on the host: its
own code (csrc/quick_mx_forms.h) compiled into a small program.  Test
infrastructure."""
from __future__ import annotations

import os
import subprocess

import paper_2402_10076_amd as Q

HEAD = r"""
#include <cstdio>
#include <initializer_list>
#include "quick_mx_forms.h"
using namespace quick;
"""

PLANS = HEAD + r"""
int main()
{
    long long M, N, K, E;
    int grouped, gated, x16;
    while (std::scanf("%lld %lld %lld %lld %d %d %d", &M, &N, &K, &E, &grouped, &gated, &x16) == 7) {
        const MxPlan p = plan_product({M, N, K, E, grouped != 0, gated != 0, x16 != 0});
        std::printf("%d %d %d %d %d %lld %lld\n", p.form, p.form < 0 ? 0 : kForms[p.form].bm, p.tail, p.once, p.lead,
                    (long long)p.row_tiles, (long long)p.columns);
    }
}
"""

FIELDS = ("form", "bm", "tail", "once", "lead", "row_tiles", "columns")


def program(folder, text, name):
    src = os.path.join(str(folder), name + ".cpp")
    with open(src, "w") as f:
        f.write(text)
    exe = src[:-4]
    csrc = os.path.join(os.path.dirname(Q.LIB_PATH), "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", csrc, src, "-o", exe], check=True)
    return exe


def plans(folder, sizes):
    """Plans of sizes (M, N, K, experts, grouped, gated, 16-bit activations)."""
    text = "".join("%d %d %d %d %d %d %d\n" % s for s in sizes)
    out = subprocess.run([program(folder, PLANS, "plans")], input=text, capture_output=True, text=True, check=True).stdout
    rows = [dict(zip(FIELDS, map(int, line.split()))) for line in out.splitlines()]
    assert len(rows) == len(sizes)
    return rows
