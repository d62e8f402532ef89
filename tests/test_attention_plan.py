"""How attention over the paged cache is shared out, on the CPU: the kernels'
own arithmetic (csrc/quick_attention_plan.h) gone through as their waves and
workgroups do, for random and for broken lengths and offsets.  Every part of
every item is taken by one worker, parts of an item follow each other from
worker to worker as the joining kernel expects, and rows, pages and tokens stay
inside."""
import os
import subprocess

import paper_2402_10076_amd as Q

SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <map>
#include <tuple>
#include <vector>
#include "quick_attention_plan.h"
using namespace quick;

static long bad = 0;
#define CHECK(x) do { if (!(x) && bad++ < 5) std::printf("line %d: %s\n", __LINE__, #x); } while (0)

struct Piece { int worker, at, take; bool first; int64_t share; };

template <int BC, bool MANY>
static void go(const AttnShape& a, int workers, int least)
{
    // find_share of one worker, lane by lane
    std::vector<int64_t> upto(64);
    int64_t run = 0;
    for (int l = 0; l < 64; l++) upto[l] = run += cost_of<BC, MANY>(a, items_of<MANY>(a, l));
    const int64_t all = run;
    std::map<std::tuple<int, int, int>, std::vector<Piece>> items;
    for (int w = 0; w < workers; w++) {
        Walk k;
        k.share = share_of(all, workers, least);
        CHECK(k.share * workers >= all);
        const int64_t u = w * k.share;
        k.b = k.j = k.h = k.at = 0;
        k.left = u >= all ? 0 : k.share < all - u ? k.share : all - u;
        if (k.left > 0) {
            int from = 0;
            while (upto[from] <= u) from++;
            find_item<BC, MANY>(a, items_of<MANY>(a, from), from ? upto[from - 1] : 0, u, k);
            begin_item(a, k);
        }
        for (bool first = true; k.left > 0 && k.b < a.seqs; first = false) {
            const Seq s = seq_of(a, k.b);
            const Tile t = tile_of<BC>(a, s, k.j);
            CHECK(s.queries > 0 && k.j < tiles_of<BC>(a, s) && k.h >= 0 && k.h < a.heads && k.at >= 0 && k.at < t.cost);
            CHECK(t.first >= 0 && t.first + s.queries <= a.T && s.queries <= a.most);
            const int take = (int)(t.cost - k.at < k.left ? t.cost - k.at : k.left);
            if (left_to_next(a, k, t, take)) break;
            int p0, p1;
            pages_of(a, t, k.at, take, p0, p1);
            if (p1 > p0) {
                CHECK(p0 >= 0 && p1 <= a.width);
                // some column sees a token of the first and of the last page
                CHECK(p0 * 64 < t.length && (p1 - 1) * 64 < t.length);
            }
            // what every column sees is seen by the first and by the last
            for (int col : {k.j * BC, (k.j + 1) * BC < t.columns ? (k.j + 1) * BC - 1 : t.columns - 1}) {
                const int pos = t.base + col / a.group;
                const int hi = a.causal ? (pos + 1 < t.length ? pos + 1 : t.length) : t.length;
                const int lo = a.window ? (pos + 1 - a.window > 0 ? pos + 1 - a.window : 0) : 0;
                CHECK(hi <= 0 || hi >= t.all_hi);
                CHECK(lo <= t.all_lo);
                if (hi > lo) CHECK(lo / 64 >= t.p0 && (hi + 63) / 64 <= t.p1);
            }
            items[{k.b, k.j, k.h}].push_back({w, k.at, take, first, k.share});
            advance<BC, MANY>(a, k, t, take);
        }
    }
    size_t n = 0;
    for (int b = 0; b < a.seqs; b++) {
        const Seq s = seq_of(a, b);
        for (int j = 0; j < tiles_of<BC>(a, s) && (MANY || j < 1); j++)
            for (int h = 0; h < a.heads; h++, n++) {
                const auto& p = items[{b, j, h}];
                const int cost = tile_of<BC>(a, s, j).cost;
                int at = 0;
                for (size_t i = 0; i < p.size(); i++) {
                    CHECK(p[i].at == at);
                    at += p[i].take;
                    if (i) CHECK(p[i].worker == p[0].worker + (int)i && p[i].first);
                }
                CHECK(at == cost);
                if (p.size() && p[0].take < cost)   // what set_join tells the joining kernel
                    CHECK(1 + (cost - p[0].take + p[0].share - 1) / p[0].share == (int64_t)p.size());
            }
    }
    CHECK(items.size() == n);
}

static int rnd(int lo, int hi) { return lo + (int)(rand() % (unsigned)(hi - lo + 1)); }

int main()
{
    srand(1);
    for (int round = 0; round < 4000; round++) {
        AttnShape a;
        const bool wild = round % 4 == 0;
        a.seqs = round % 50 == 0 ? rnd(60, 200) : rnd(1, 12);
        a.heads = rnd(1, 4);
        a.group = rnd(1, 16);
        a.width = round % 7 == 0 ? rnd(0, 2) : rnd(1, 80);
        a.start = rnd(1, 16);
        a.causal = rnd(0, 3) > 0;
        a.window = a.causal && rnd(0, 1) ? (rnd(0, 9) ? rnd(1, 2000) : 1 << 30) : 0;
        std::vector<int32_t> lengths(a.seqs), offsets(a.seqs + 1);
        a.T = 0;
        for (int b = 0; b < a.seqs; b++) {
            offsets[b] = a.T;
            a.T += round % 3 == 0 ? rnd(0, 200) : rnd(0, 2);
            lengths[b] = rnd(0, a.width * 64);
        }
        offsets[a.seqs] = a.T;
        if (wild)
            for (int i = 0; i < 3; i++) {
                lengths[rnd(0, a.seqs - 1)] = rnd(0, 1) ? rand() - (1 << 30) : INT32_MIN;
                offsets[rnd(0, a.seqs)] = rnd(0, 1) ? rand() - (1 << 30) : rnd(0, 1) ? INT32_MIN : INT32_MAX;
            }
        a.lengths = lengths.data();
        a.offsets = offsets.data();
        if (a.T == 0) continue;
        a.most = rnd(1, a.T);
        const int workers = rnd(1, 300), least = a.start + rnd(1, 8);
        go<32, true>(a, workers, least);
        go<128, true>(a, workers, least);
        go<256, true>(a, workers, least);
        // one tile a sequence
        a.most = a.most * a.group > 16 ? 16 / a.group : a.most;
        if (a.most) go<16, false>(a, workers, least);
        a.offsets = nullptr;
        a.T = a.seqs;
        a.most = 1;
        go<16, false>(a, workers, least);
    }
    std::printf("%ld wrong\n", bad);
    return bad != 0;
}
"""


def test_shares_cover_every_item_once(tmp_path):
    src = tmp_path / "t.cpp"
    src.write_text(SOURCE)
    exe = str(tmp_path / "t")
    csrc = os.path.join(os.path.dirname(Q.LIB_PATH), "csrc")
    include = os.path.join(os.path.dirname(os.path.dirname(Q.LIB_PATH)), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", csrc, "-I",
                    include, str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
