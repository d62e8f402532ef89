// How attention over the paged cache is shared out among workgroups: the parts
// that are plain arithmetic, which a host program can go through too.
//
// An item is a tile of columns (a column is a query and one of the query heads
// that share a cache head) of a sequence for one cache head, and costs the
// pages that some column of it sees and, before those, the time it takes to
// begin one, in pages.  Items lie in the order of sequence, tile and head; a
// worker takes an equal run of the cost of all, so that lengths may differ as
// they like and nothing of them is known to the host.  Items that cross from
// one worker to the next are joined afterwards; one that would not come past its
// beginning in a worker is left to the next.
#pragma once
#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#else
#define __device__
#define __host__
#define __forceinline__ inline
#endif
#include <cstdint>

#include "quick_kv4.h"

namespace quick {

struct AttnShape {
    const int32_t* lengths;
    const int32_t* offsets;   // or null: one query a sequence
    int32_t T, heads, group, seqs, width, most, window, causal;
    int32_t start;            // what an item costs beside its pages
};

// The columns of a sequence.
struct Seq {
    int first;      // row of its first query
    int queries;    // that are worked on
    int base;       // position of the first
    int length;     // tokens in the cache
};

__device__ __host__ __forceinline__ int clamped(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __host__ __forceinline__ Seq seq_of(const AttnShape& a, int b)
{
    Seq s;
    const int64_t room = (int64_t)a.width * kPage;
    s.length = clamped(a.lengths[b], 0, room > INT32_MAX ? INT32_MAX : (int)room);
    s.first = a.offsets ? clamped(a.offsets[b], 0, a.T) : clamped(b, 0, a.T);
    const int end = a.offsets ? clamped(a.offsets[b + 1], s.first, a.T) : clamped(b + 1, s.first, a.T);
    s.base = s.length - (end - s.first);
    s.queries = end - s.first < a.most ? end - s.first : a.most;
    return s;
}

struct Tile {
    int p0, p1;             // pages that some column sees (p1 <= p0: none)
    int cost;               // of the item
    int columns;            // of the sequence
    int first, base, length;
    int all_lo, all_hi;     // tokens that every column sees
};

template <int BC>
__device__ __host__ __forceinline__ int tiles_of(const AttnShape& a, const Seq& s)
{
    return (int)(((int64_t)s.queries * a.group + BC - 1) / BC);
}

template <int BC>
__device__ __host__ __forceinline__ Tile tile_of(const AttnShape& a, const Seq& s, int j)
{
    Tile t;
    t.columns = s.queries * a.group;
    t.first = s.first;
    t.base = s.base;
    t.length = s.length;
    const int last = (j + 1) * BC < t.columns ? (j + 1) * BC - 1 : t.columns - 1;
    const int lo = s.base + j * BC / a.group, hi = s.base + last / a.group;   // positions
    int begin = 0, end = s.length;
    t.all_lo = 0;
    t.all_hi = s.length;
    if (a.causal) {
        end = clamped(hi + 1, 0, s.length);
        t.all_hi = clamped(lo + 1, 0, s.length);
        if (a.window) {
            begin = lo + 1 - a.window > 0 ? lo + 1 - a.window : 0;
            t.all_lo = hi + 1 - a.window > 0 ? hi + 1 - a.window : 0;
        }
    }
    t.p0 = begin / kPage;
    t.p1 = (int)(((int64_t)end + kPage - 1) / kPage);
    t.cost = (t.p1 > t.p0 ? t.p1 - t.p0 : 0) + a.start;
    return t;
}

// The pages of tile t in a part of its cost.
__device__ __host__ __forceinline__ void pages_of(const AttnShape& a, const Tile& t, int at, int take, int& p0, int& p1)
{
    const int lo = at - a.start, hi = at + take - a.start;
    p0 = t.p0 + (lo > 0 ? lo : 0);
    p1 = t.p0 + (hi > 0 ? hi : 0);
    if (p1 > t.p1) p1 = t.p1;
}

// Where a worker stands.
struct Walk {
    int b, j, h, at;        // at: how far into the item's cost
    int64_t left;           // cost to go
    int64_t share;          // of every worker but the last
};

// Whether a worker's last item is the next one's, which then begins there.
__device__ __host__ __forceinline__ bool left_to_next(const AttnShape& a, const Walk& k, const Tile& t, int take)
{
    return k.at == 0 && take < t.cost && take <= a.start;
}
__device__ __host__ __forceinline__ void begin_item(const AttnShape& a, Walk& k)
{
    if (k.at > a.start) return;
    k.left += k.at;
    k.at = 0;
}

// On by `take` of tile t's cost.
template <int BC, bool MANY>
__device__ __host__ __forceinline__ void advance(const AttnShape& a, Walk& k, const Tile& t, int take)
{
    k.left -= take;
    k.at += take;
    if (k.at < t.cost) return;
    k.at = 0;
    if (++k.h < a.heads) return;
    k.h = 0;
    if (MANY && (int64_t)(++k.j) * BC < t.columns) return;
    k.j = 0;
    // sequences without a query have no item; there is one more item if any cost is left
    do k.b++;
    while (k.left > 0 && k.b < a.seqs && seq_of(a, k.b).queries == 0);
}

// A worker's share of a total cost: a whole number, `least` or more.
__device__ __host__ __forceinline__ int64_t share_of(int64_t all, int workers, int least)
{
    // (binary64 has the quotient to a unit, and its product is exact)
    int64_t s = (int64_t)((double)all / workers);
    while (s * workers < all) s++;
    return s < least ? least : s;
}

// Which of 64 lanes adds up what of the items: whole sequences, or (MANY tiles
// of one) with fewer of those than lanes slices of one's tiles.
struct LaneItems {
    int b0, b1, slice, slices;
};
template <bool MANY>
__device__ __host__ __forceinline__ LaneItems items_of(const AttnShape& a, int lane)
{
    LaneItems k;
    const int per = (a.seqs + 63) / 64;
    k.slices = !MANY || a.seqs > 32 ? 1 : 64 / a.seqs;
    k.b0 = k.slices > 1 ? lane / k.slices : lane * per;
    k.b1 = k.b0 + per < a.seqs ? k.b0 + per : a.seqs;
    k.slice = k.slices > 1 ? lane % k.slices : 0;
    return k;
}
// Calls f(b, j, cost) for those in their order, until it returns true.
template <int BC, bool MANY, class F>
__device__ __host__ __forceinline__ void each_item(const AttnShape& a, const LaneItems& k, F f)
{
    for (int b = k.b0; b < k.b1; b++) {
        const Seq s = seq_of(a, b);
        if constexpr (MANY) {
            const int tiles = tiles_of<BC>(a, s), run = k.slices > 1 ? (tiles + k.slices - 1) / k.slices : tiles;
            for (int j = k.slice * run; j < tiles && j < (k.slice + 1) * run; j++)
                if (f(b, j, tile_of<BC>(a, s, j).cost)) return;
        } else if (s.queries > 0 && f(b, 0, tile_of<BC>(a, s, 0).cost)) return;
    }
}
template <int BC, bool MANY>
__device__ __host__ __forceinline__ int64_t cost_of(const AttnShape& a, const LaneItems& k)
{
    int64_t sum = 0;
    each_item<BC, MANY>(a, k, [&](int, int, int cost) {
        sum += cost;
        return false;
    });
    return sum * a.heads;
}
// The item of one's lane that holds place u of the whole cost, `before` of which
// lies before the lane's.
template <int BC, bool MANY>
__device__ __host__ __forceinline__ void find_item(const AttnShape& a, const LaneItems& k, int64_t before, int64_t u, Walk& w)
{
    each_item<BC, MANY>(a, k, [&](int b, int j, int cost) {
        const int64_t all = (int64_t)cost * a.heads;
        if (u >= before + all) {
            before += all;
            return false;
        }
        // (exact: both are far below 2^53, and so the quotient is further from the next whole number than that)
        w.h = (int)((double)(u - before) / cost);
        w.at = (int)(u - before - (int64_t)w.h * cost);
        w.b = b;
        w.j = j;
        return true;
    });
}

#if defined(__HIPCC__)

template <int BC>
__device__ __forceinline__ Tile tile_of(const AttnShape& a, int b, int j)
{
    return tile_of<BC>(a, seq_of(a, b), j);
}

// v of the lane CTRL away (0 where there is none) added to v.
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t add_from(int64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, true);
    return v + (int64_t)((uint64_t)hi << 32 | lo);
}

// The run of a worker.  Every wave works it out by itself, its lanes adding up
// the items' costs, with no exchange but between them.
template <int BC, bool MANY>
__device__ __forceinline__ Walk find_share(const AttnShape& a, int workers, int worker, int least)
{
    const int lane = threadIdx.x & 63;
    const LaneItems k = items_of<MANY>(a, lane);
    const int64_t sum = cost_of<BC, MANY>(a, k);
    // sums along each row of 16 lanes, then over the rows
    int64_t upto = sum;
    upto = add_from<0x111, 0xF>(upto);
    upto = add_from<0x112, 0xF>(upto);
    upto = add_from<0x114, 0xF>(upto);
    upto = add_from<0x118, 0xF>(upto);
    upto = add_from<0x142, 0xA>(upto);
    upto = add_from<0x143, 0xC>(upto);
    auto of_lane = [](int64_t v, int lane) {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
        return (int64_t)((uint64_t)hi << 32 | lo);
    };
    const int64_t all = of_lane(upto, 63);
    Walk w;
    w.share = share_of(all, workers, least);
    const int64_t u = worker * w.share;
    w.b = w.j = w.h = w.at = 0;
    w.left = u >= all ? 0 : w.share < all - u ? w.share : all - u;
    if (w.left > 0) {
        const int from = __builtin_ctzll(__ballot(upto > u));
        if (lane == from) find_item<BC, MANY>(a, k, upto - sum, u, w);
        w.b = __builtin_amdgcn_readlane(w.b, from);
        w.j = __builtin_amdgcn_readlane(w.j, from);
        w.h = __builtin_amdgcn_readlane(w.h, from);
        w.at = __builtin_amdgcn_readlane(w.at, from);
        begin_item(a, w);
    }
    return w;
}

#endif

}  // namespace quick
