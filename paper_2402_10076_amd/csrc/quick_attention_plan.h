// How attention over the paged cache is shared out among workgroups: the parts
// that are plain arithmetic, which a host program can go through too.
//
// An item is a tile of columns (a column is a query and one of the query heads
// that share a cache head) of a sequence for one cache head, and costs the
// pages that some column of it sees and, before those, the time it takes to
// begin one, in pages.  Items lie in the order of sequence, tile and head; a
// worker takes an equal run of the cost of all, so that lengths may differ as
// they like and nothing of them is known to the host.  Items that cross from
// one worker to the next are joined afterwards.
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

#if defined(__HIPCC__)

template <int BC>
__device__ __forceinline__ Tile tile_of(const AttnShape& a, int b, int j)
{
    return tile_of<BC>(a, seq_of(a, b), j);
}

// Where a worker stands.
struct Walk {
    int b, j, h, at;        // at: how far into the item's cost
    int64_t left;           // cost to go
    int64_t share;          // of every worker but the last
};

// LDS of find_share.
struct PlanSpace {
    int64_t wave[8];
    int at[4];
};

// The run of a worker, by all its N threads.  A thread adds up the cost of some
// sequences or, with fewer sequences than threads, of some tiles of one.
template <int BC, int N>
__device__ __forceinline__ Walk find_share(const AttnShape& a, int workers, int worker, int least, PlanSpace& space)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int slices = a.seqs >= N ? 1 : N / a.seqs;            // threads of a sequence
    const int per = a.seqs >= N ? (a.seqs + N - 1) / N : 1;     // sequences of a thread
    const int b0 = a.seqs >= N ? tid * per : tid / slices;
    const int slice = a.seqs >= N ? 0 : tid % slices;
    int64_t sum = 0;
    for (int b = b0; b < min(b0 + per, a.seqs); b++) {
        const Seq s = seq_of(a, b);
        const int tiles = tiles_of<BC>(a, s), run = (tiles + slices - 1) / slices;
        for (int j = slice * run; j < min(tiles, (slice + 1) * run); j++) sum += tile_of<BC>(a, s, j).cost;
    }
    sum *= a.heads;
    int64_t upto = sum;
    for (int d = 1; d < 64; d *= 2) {
        const int64_t o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) space.wave[wave] = upto;
    __syncthreads();
    int64_t all = 0, before = upto - sum;
#pragma unroll
    for (int w = 0; w < N / 64; w++) {
        if (w < wave) before += space.wave[w];
        all += space.wave[w];
    }
    Walk k;
    k.share = (all + workers - 1) / workers;
    k.share = k.share < least ? least : k.share;
    const int64_t u0 = min(all, worker * k.share);
    k.left = min(k.share, all - u0);
    if (u0 < all && before <= u0 && u0 < before + sum) {
        int64_t at = before;
        bool found = false;
        for (int b = b0; b < min(b0 + per, a.seqs) && !found; b++) {
            const Seq s = seq_of(a, b);
            const int tiles = tiles_of<BC>(a, s), run = (tiles + slices - 1) / slices;
            for (int j = slice * run; j < min(tiles, (slice + 1) * run); j++) {
                const int cost = tile_of<BC>(a, s, j).cost;
                if (u0 < at + (int64_t)cost * a.heads) {
                    const int64_t in = u0 - at;
                    space.at[0] = b;
                    space.at[1] = j;
                    space.at[2] = (int)(in / cost);
                    space.at[3] = (int)(in % cost);
                    found = true;
                    break;
                }
                at += (int64_t)cost * a.heads;
            }
        }
    }
    __syncthreads();
    k.b = __builtin_amdgcn_readfirstlane(space.at[0]);
    k.j = __builtin_amdgcn_readfirstlane(space.at[1]);
    k.h = __builtin_amdgcn_readfirstlane(space.at[2]);
    k.at = __builtin_amdgcn_readfirstlane(space.at[3]);
    return k;
}

// The pages of tile t in a part of its cost.
__device__ __host__ __forceinline__ void pages_of(const AttnShape& a, const Tile& t, int at, int take, int& p0, int& p1)
{
    const int lo = at - a.start, hi = at + take - a.start;
    p0 = t.p0 + (lo > 0 ? lo : 0);
    p1 = t.p0 + (hi > 0 ? hi : 0);
    if (p1 > t.p1) p1 = t.p1;
}

// On by `take` of tile t's cost.
template <int BC>
__device__ __forceinline__ void advance(const AttnShape& a, Walk& k, const Tile& t, int take)
{
    k.left -= take;
    k.at += take;
    if (k.at < t.cost) return;
    k.at = 0;
    if (++k.h < a.heads) return;
    k.h = 0;
    if ((int64_t)(++k.j) * BC < t.columns) return;
    k.j = 0;
    // sequences without a query have no item; there is one more item if any page is left
    do k.b++;
    while (k.left > 0 && k.b < a.seqs && seq_of(a, k.b).queries == 0);
}

#endif

}  // namespace quick
