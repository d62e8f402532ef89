// Attention over the paged 4-bit cache.
#include <algorithm>
#include <cmath>

#include "quick_attention_parts.h"

namespace {

using namespace quick;

// Workgroups of the stream kernel that a compute unit holds at once, by the
// registers that D channels and NC times 16 columns take; the grid is that for
// all units.
constexpr int stream_resident(int64_t D, int NC) { return D == 64 ? 6 - 2 * NC : D == 128 ? 2 : 3 - NC; }
constexpr int kUnits = 256;
// What a workgroup takes at least, and what an item costs beside its pages.
constexpr int kStreamShare = 16, kStreamStart = 12;
// Most pages of an item that a workgroup takes whole: a wave's lanes hold their ids.
constexpr int kWholePages = 64;
// Most sequences that such workgroups put in order.
constexpr int kRanked = 128;

// Exchanges over the four groups of 16 lanes that share a column.
template <class F>
__device__ __forceinline__ float over_groups(float v, F f)
{
    const auto r = __builtin_amdgcn_permlane16_swap(bits_as<uint32_t>(v), bits_as<uint32_t>(v), false, false);
    v = f(bits_as<float>(r[0]), bits_as<float>(r[1]));
    const auto s = __builtin_amdgcn_permlane32_swap(bits_as<uint32_t>(v), bits_as<uint32_t>(v), false, false);
    return f(bits_as<float>(s[0]), bits_as<float>(s[1]));
}

// What a lane (group g = lane / 16, c = lane % 16) holds of a page: of the keys
// of tokens c of each 16, its quarter of the channels; of the values of tokens
// 4 g .. 4 g + 3 of each 16, channels c * w .. c * w + w - 1 of each 128.
template <int D>
struct KeyWords {
    static constexpr int KW = D / 32, HALVES = D > 128 ? 2 : 1;
    uint32_t k[4][KW], s[HALVES];
};
template <int D>
struct ValueWords {
    static constexpr int HALVES = D > 128 ? 2 : 1, VW = D < 128 ? 2 : 4;
    uint32_t v[HALVES][4][VW], s[HALVES][4];
};

template <int D>
__device__ __forceinline__ void load_keys(KeyWords<D>& w, const uint8_t* page, int lane)
{
    typedef Kv4<D> L;
    const uint32_t c = lane & 15, g = lane >> 4;
    const uint32_t key = L::kKeys + c * (D / 2) + g * (D == 64 ? 8 : 16);
    const uint32_t scale = L::kKeyScales + (D == 64 ? g >> 1 : g) * 64 + c * 4;
#pragma unroll
    for (int h = 0; h < KeyWords<D>::HALVES; h++) {
        w.s[h] = *(const uint32_t*)(page + scale + h * 256);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint8_t* k = page + key + i * (8 * D) + h * 64;
            if constexpr (D == 64) {
                const u2_t a = *(const u2_t*)k;
                w.k[i][0] = a[0];
                w.k[i][1] = a[1];
            } else {
                const u4_t a = *(const u4_t*)k;
#pragma unroll
                for (int j = 0; j < 4; j++) w.k[i][h * 4 + j] = a[j];
            }
        }
    }
}

template <int D>
__device__ __forceinline__ void load_values(ValueWords<D>& w, const uint8_t* page, int lane)
{
    typedef Kv4<D> L;
    constexpr int VW = ValueWords<D>::VW;
    const uint32_t c = lane & 15, g = lane >> 4;
    const uint32_t value = L::kValues + (g * 16 + c) * (4 * VW);
    const uint32_t scale = L::kValueScales + (D == 64 ? c >> 3 : c >> 2) * 64 + g * 16;
#pragma unroll
    for (int h = 0; h < ValueWords<D>::HALVES; h++) {
        const u4_t s = *(const u4_t*)(page + scale + h * 256);
#pragma unroll
        for (int i = 0; i < 4; i++) w.s[h][i] = s[i];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint8_t* v = page + value + h * 4096 + i * (256 * VW);
            if constexpr (D == 64) {
                const u2_t a = *(const u2_t*)v;
                w.v[h][i][0] = a[0];
                w.v[h][i][1] = a[1];
            } else {
                const u4_t a = *(const u4_t*)v;
#pragma unroll
                for (int j = 0; j < 4; j++) w.v[h][i][j] = a[j];
            }
        }
    }
}

// A column's state: reference, sum of this lane's weights, and the sums of
// values.  Of d-tile j, register i: channel 128 (j / T) + (4 g + i) T + j % T,
// T = min(D, 128) / 16.
template <int D>
struct Column {
    Reference ref;
    bool away;      // whether it is further than this form of the loop goes
    float l;
    f4_t o[D / 16];
};

// Tokens a column sees: lo <= token < hi.
struct Seen {
    int lo, hi;
};

// The blocks of values that are beyond the type make NaN of the columns that
// see them, and nothing of the others: they are taken out of the product (their
// scales become 2^-127) and the sums of those columns set.  Seldom run.  (Blocks of
// keys are NaN by themselves, and what does not see them hides their scores.)
template <int DT, int D>
__device__ __forceinline__ void take_out(ValueWords<D>& w)
{
#pragma unroll
    for (int h = 0; h < ValueWords<D>::HALVES; h++)
#pragma unroll
        for (int i = 0; i < 4; i++) w.s[h][i] &= ~whole_bytes(beyond<DT>(w.s[h][i]));
}
template <int DT, int D>
__device__ __forceinline__ void spoil(Column<D>& col, const uint8_t* page, int lo, int hi, int lane)
{
    typedef Kv4<D> L;
    constexpr int TILES = (D < 128 ? D : 128) / 16;
    const int g = lane >> 4;
#pragma unroll
    for (int h = 0; h < ValueWords<D>::HALVES; h++) {
        bool bad = false;
#pragma unroll 1
        for (int t = 0; t < kPage; t++) {
            const uint32_t s = page[L::value_scale(t, (D == 64 ? g >> 1 : g) + 4 * h)];
            bad |= beyond<DT>(s) != 0 && t >= lo && t < hi;
        }
        const float f = bad ? NAN : 0.0f;
#pragma unroll
        for (int j = 0; j < TILES; j++) col.o[h * TILES + j] += f;
    }
}

// Scores of a page's keys with the NC columns of a lane (16 tokens each 16).
template <int DT, int D, int NC>
__device__ __forceinline__ void score(const KeyWords<D>& w, const u4_t (&q)[NC][D / 32], f4_t (&s)[NC][4])
{
    // (blocks beyond the type get the scale of NaN)
    uint32_t scales[KeyWords<D>::HALVES];
#pragma unroll
    for (int h = 0; h < KeyWords<D>::HALVES; h++) scales[h] = w.s[h] | whole_bytes(beyond<DT>(w.s[h]));
#pragma unroll
    for (int i = 0; i < 4; i++) {
#pragma unroll
        for (int n = 0; n < NC; n++) s[n][i] = f4_t{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < D / 32; j++) {
            const u4_t k = code_words<DT>(w.k[i][j], scale_of(scales[j / 4], i));
#pragma unroll
            for (int n = 0; n < NC; n++) s[n][i] = mfma16<DT>(k, q[n][j], s[n][i]);
        }
    }
}

// The weights of those, as operands p[n][r] of 32 tokens each.
template <int DT, int D, int NC, bool FAR>
__device__ __forceinline__ void weigh(f4_t (&s)[NC][4], Column<D> (&col)[NC], const Seen (&seen)[NC], int token0, bool masked,
                                      bool ok, float scale, int lane, u4_t (&p)[NC][2])
{
    const int g = lane >> 4;
#pragma unroll
    for (int n = 0; n < NC; n++) {
        if (masked) {
            seldom();
            const int lo = seen[n].lo - token0 - 4 * g, hi = (ok ? seen[n].hi : token0) - token0 - 4 * g;
            const uint32_t bits[2] = {bits_between(lo, hi), bits_between(lo - 32, hi - 32)};
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int e = 0; e < 4; e++) s[n][i][e] = where_bit(s[n][i][e], bits[i / 2], 16 * (i % 2) + e);
        }
        float top = s[n][0][0];
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) top = fmaxf(top, s[n][i][e]);
        if (FAR || __ballot(fmaf(top, scale, -col[n].ref.m) > kRoom<DT>)) {
            seldom();
            top = over_groups(top, [](float a, float b) { return fmaxf(a, b); });
            const float f = col[n].ref.template raise<DT, FAR>(top, scale, col[n].away);
            col[n].l *= f;
#pragma unroll
            for (int j = 0; j < D / 16; j++) col[n].o[j] *= f;
        }
        if constexpr (FAR) {
#pragma unroll
            for (int i = 0; i < 4; i++) s[n][i] -= col[n].ref.base;
        }
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const float u = __builtin_amdgcn_exp2f(fmaf(s[n][i][e], scale, -col[n].ref.m));
                const float v = __builtin_amdgcn_exp2f(fmaf(s[n][i][e + 1], scale, -col[n].ref.m));
                col[n].l += u + v;
                p[n][i / 2][i % 2 * 2 + e / 2] = pair16<DT>(u, v);
            }
    }
}

// The values that those weigh.
template <int DT, int D, int NC>
__device__ __forceinline__ void add_values(const ValueWords<D>& w, const u4_t (&p)[NC][2], Column<D> (&col)[NC])
{
    typedef ValueWords<D> W;
    constexpr int TILES = (D < 128 ? D : 128) / 16;
#pragma unroll
    for (int r = 0; r < 2; r++) {
#pragma unroll
        for (int h = 0; h < W::HALVES; h++) {
            float sa[4], sb[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                sa[e] = scale_of(w.s[h][2 * r], e);
                sb[e] = scale_of(w.s[h][2 * r + 1], e);
            }
            u4_t lo, hi;
            auto add = [&](int j) {
#pragma unroll
                for (int n = 0; n < NC; n++) {
                    col[n].o[h * TILES + j] = mfma16<DT>(lo, p[n][r], col[n].o[h * TILES + j]);
                    col[n].o[h * TILES + j + 1] = mfma16<DT>(hi, p[n][r], col[n].o[h * TILES + j + 1]);
                }
            };
            value_words<DT, W::VW, 0>(w.v[h][2 * r], w.v[h][2 * r + 1], sa, sb, lo, hi);
            add(0);
            value_words<DT, W::VW, 1>(w.v[h][2 * r], w.v[h][2 * r + 1], sa, sb, lo, hi);
            add(2);
            if constexpr (D != 64) {
                value_words<DT, W::VW, 2>(w.v[h][2 * r], w.v[h][2 * r + 1], sa, sb, lo, hi);
                add(4);
                value_words<DT, W::VW, 3>(w.v[h][2 * r], w.v[h][2 * r + 1], sa, sb, lo, hi);
                add(6);
            }
        }
    }
}

// The sequence of rank r, those of the most pages first and equal ones in their
// order: items beyond the resident ones even out when the longest begin first.
// Every workgroup counts the sequences by their pages, 64 at most, and looks for
// its own.  32 sequences of 37 to 4096 tokens, 32 heads: 54.9 us, 62.1 in the order
// they come in; 128 equal ones of 4000, 8 heads: 106 and 103; many sequences, whose
// items are short, lose more (1000 of 50 to 500: 104 and 80) and are left alone.
template <int THREADS>
__device__ __forceinline__ int of_rank(const AttnShape& s, int r)
{
    __shared__ uint32_t count[64];
    __shared__ uint8_t of[kRanked];
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < 64) count[threadIdx.x] = 0;
    __syncthreads();
    for (int b = threadIdx.x; b < s.seqs; b += THREADS) {
        const int from_most = kWholePages - clamped((seq_of(s, b).length + kPage - 1) / kPage, 1, kWholePages);
        of[b] = (uint8_t)from_most;
        atomicAdd(&count[from_most], 1u);
    }
    __syncthreads();
    const int n = (int)count[lane];
    int64_t upto = n;
    upto = add_from<0x111, 0xF>(upto);
    upto = add_from<0x112, 0xF>(upto);
    upto = add_from<0x114, 0xF>(upto);
    upto = add_from<0x118, 0xF>(upto);
    upto = add_from<0x142, 0xA>(upto);
    upto = add_from<0x143, 0xC>(upto);
    const int at = __builtin_ctzll(__ballot(upto > r));     // (r is less than their sum)
    int k = r - __builtin_amdgcn_readlane((int)upto - n, at);
    for (int b0 = 0; b0 < s.seqs; b0 += 64) {
        const uint64_t m = __ballot(b0 + lane < s.seqs && of[min(b0 + lane, s.seqs - 1)] == at);
        const int c = __popcll(m);
        if (k < c) return b0 + __builtin_ctzll(__ballot((m >> lane & 1) && __popcll(m & ((1ull << lane) - 1)) == k));
        k -= c;
    }
    return 0;
}

// A few queries of each sequence (tiles of 16 NC columns, a column being a query
// and one of the heads that share keys and values; NC = 1: one tile each).  A wave takes every WAVES'th page
// of its workgroup's share: scores transposed, keys . queries^T, so that a
// column's scores are in the lanes that need its weights as the operand of
// values^T . weights, with no exchange between lanes and nothing in LDS; the
// waves' sums meet in LDS once an item.
// Long sequences are bound by HBM: 64 of 512 to 32768 tokens, 8 heads of 128 read
// by 8 each, 207 us, 5.6 TB/s; 32 of 37 to 4096, 32 heads, 55 us, 5.2 TB/s.  Short
// shares are bound by the chain of plan, table, page and the sums' meeting, some 15
// thousand cycles an item: 8 of 2000 to 9000, 5 queries, 21 us, 2.3 TB/s; 1 of
// 1000, whole, 7 us.
template <int DT, int D, int NC, int WAVES, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES, stream_resident(D, NC)) void attn_stream_kernel(AttnArgs a)
{
    typedef Kv4<D> L;
    constexpr int BC = 16 * NC, KW = D / 32, TILES = (D < 128 ? D : 128) / 16, ROW = D + 4;
    // where registers are short the last step's addresses are not kept over the loop (64 channels: 67.8 us for 64.8 with
    // four of them in scratch; with 128, which have registers left, drafts take 26.2 for 25.3 so)
    constexpr bool LATE = !WHOLE && ((D == 64 && NC == 1) || D > 128);
    __shared__ float sums[WAVES][16][ROW];
    __shared__ float refs[WAVES][16][3];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int worker = blockIdx.x;
    Walk walk;
    int32_t ids = 0;
    if constexpr (WHOLE) {
        // an item each: no joining, and no place for it; all of a sequence's pages come while its length does
        walk.b = worker / a.s.heads;
        const int rank = walk.b;
        if constexpr (WAVES == 4) {
            if (a.ranked) walk.b = of_rank<64 * WAVES>(a.s, rank);
        }
        walk.h = worker - rank * a.s.heads;
        walk.j = walk.at = 0;
        walk.left = walk.share = INT32_MAX;
        if (a.s.width) ids = a.table[(int64_t)walk.b * a.s.width + min(lane, a.s.width - 1)];
    } else walk = find_share<BC, NC == 2>(a.s, a.workers, worker, kStreamShare);
    int join[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (bool first = true; walk.left > 0 && walk.b < a.s.seqs; first = false) {
        const Seq seq = seq_of(a.s, walk.b);
        const int columns = seq.queries * a.s.group;
        if (WHOLE && columns == 0) return;
        // (columns behind the last are that one again, and go nowhere)
        u4_t q[NC][KW];
        int of[NC];
        auto load_queries = [&] {
#pragma unroll
            for (int n = 0; n < NC; n++) {
                const int cc = min(walk.j * BC + n * 16 + c, columns - 1);
                of[n] = cc * a.group_inv >> 16;
                const uint8_t* from = a.q + 2 * ((int64_t)(seq.first + of[n]) * a.q_token +
                                                 (int64_t)(walk.h * a.s.group + cc - of[n] * a.s.group) * a.q_head);
#pragma unroll
                for (int j = 0; j < KW; j++)
                    q[n][j] = *(const u4_t*)(from + (D == 64 ? 2 * g + j : 16 * (j / 4) + 4 * g + j % 4) * 16);
            }
        };
        if (WHOLE) load_queries();      // (they need no length)
        const Tile t = tile_of<BC>(a.s, seq, walk.j);
        const int take = (int)min((int64_t)(t.cost - walk.at), walk.left);
        if (!WHOLE && left_to_next(a.s, walk, t, take)) break;
        int p0, p1;
        pages_of(a.s, t, walk.at, take, p0, p1);
        const int32_t* table = a.table + (int64_t)walk.b * a.s.width;
        const int count = p1 > p0 + wave ? (p1 - p0 - wave + WAVES - 1) / WAVES : 0;
        if (!WHOLE) {
            // the first pages' ids ahead of the queries, for which nothing waits yet
            if (count) ids = table[min(p0 + wave + WAVES * lane, p1 - 1)];
            load_queries();
        }
        Column<D> col[NC];
        Seen seen[NC];
#pragma unroll
        for (int n = 0; n < NC; n++) {
            const int pos = t.base + of[n];
            seen[n].hi = a.s.causal ? min(pos + 1, t.length) : t.length;
            seen[n].lo = a.s.window ? max(0, pos + 1 - a.s.window) : 0;
        }
        const uint8_t* head = a.cache + walk.h * L::kBytes;
        const uint32_t stride = a.s.heads * L::kBytes;
        auto page_of = [&](int n, bool& inside) {    // page n of this wave
            if (!WHOLE && n && (n & 63) == 0) ids = table[min(p0 + wave + WAVES * (n + lane), p1 - 1)];
            const int x = __builtin_amdgcn_readlane(ids, WHOLE ? p0 + wave + WAVES * n : n & 63);
            inside = x >= 0 && x < a.pages;
            return head + (int64_t)(inside ? x : 0) * stride;
        };
        auto all_pages = [&](auto form) {
            constexpr bool FAR = decltype(form)::far;
#pragma unroll
            for (int n = 0; n < NC; n++) {
                col[n].ref = kNoReference;
                col[n].away = false;
                col[n].l = 0;
#pragma unroll
                for (int j = 0; j < D / 16; j++) col[n].o[j] = f4_t{0, 0, 0, 0};
            }
            KeyWords<D> keys;
            ValueWords<D> values;
            bool ok = false;
            const uint8_t* page = a.cache;
            if (!FAR && count) {
                page = page_of(0, ok);
                load_keys<D>(keys, page, lane);
                load_values<D>(values, page, lane);
            }
            if (!FAR && a.q_sign) {
                seldom();
#pragma unroll
                for (int n = 0; n < NC; n++)
#pragma unroll
                    for (int j = 0; j < KW; j++) q[n][j] ^= a.q_sign;
            }
            for (int n = 0; n < count; n++) {
                if (FAR) {
                    page = page_of(n, ok);
                    load_keys<D>(keys, page, lane);
                }
                const int token0 = (p0 + wave + WAVES * n) * kPage;
                const bool masked = token0 + kPage > t.all_hi || token0 < t.all_lo || !ok;
                f4_t s[NC][4];
                u4_t p[NC][2];
                score<DT, D, NC>(keys, q, s);
                // the next page's keys and values take the place of this one's as those are done with (the last one's again)
                bool next_ok = false;
                const uint8_t* next = page;
                if (!FAR) {
                    next = page_of(min(n + 1, count - 1), next_ok);
                    load_keys<D>(keys, next, lane);
                }
                weigh<DT, D, NC, FAR>(s, col, seen, token0, masked, ok, a.scale, lane, p);
                if (FAR) {
                    seldom();
                    load_values<D>(values, page, lane);
                }
                uint32_t mark = 0;
#pragma unroll
                for (int h = 0; h < ValueWords<D>::HALVES; h++)
#pragma unroll
                    for (int i = 0; i < 4; i++) mark |= beyond<DT>(values.s[h][i]);
                if (__ballot(mark != 0)) {
                    seldom();
#pragma unroll
                    for (int x = 0; x < NC; x++)
                        spoil<DT, D>(col[x], page, seen[x].lo - token0, ok ? seen[x].hi - token0 : 0, lane);
                    take_out<DT, D>(values);
                }
                add_values<DT, D, NC>(values, p, col);
                if (!FAR) {
                    load_values<D>(values, next, lane);
                    page = next;
                    ok = next_ok;
                }
            }
        };
        all_pages(Near{});
        // far scores: this wave's pages again, one after the other
        bool away = false;
#pragma unroll
        for (int n = 0; n < NC; n++) away |= col[n].away;
        if (__builtin_expect(__ballot(away) != 0, 0)) {
            seldom();
            if (!WHOLE) ids = table[min(p0 + wave + WAVES * lane, p1 - 1)];
            all_pages(Far{});
        }
        const bool whole = walk.at == 0 && take == t.cost;
        const int64_t slot = 2 * worker + (first ? 0 : 1);
        if (walk.at == 0 && !whole) {
            set_join(join, walk, t, BC, take, (int)slot);
        }
#pragma unroll
        for (int n = 0; n < NC; n++) {
            if (n || !first) __syncthreads();
            const float l = over_groups(col[n].l, [](float x, float y) { return x + y; });
            if (g == 0) {
                refs[wave][c][0] = col[n].ref.m;
                refs[wave][c][1] = col[n].ref.base;
                refs[wave][c][2] = l;
            }
#pragma unroll
            for (int h = 0; h < ValueWords<D>::HALVES; h++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    float* to = &sums[wave][c][h * 128 + (4 * g + i) * TILES];
#pragma unroll
                    for (int j = 0; j < TILES; j += 4)
                        *(f4_t*)(to + j) = f4_t{col[n].o[h * TILES + j][i], col[n].o[h * TILES + j + 1][i],
                                                col[n].o[h * TILES + j + 2][i], col[n].o[h * TILES + j + 3][i]};
                }
            __syncthreads();
            constexpr int PIECES = D / 8;
            for (int at = LATE ? late(threadIdx.x) : threadIdx.x; at < 16 * PIECES; at += 64 * WAVES) {
                const int x = at / PIECES, d = at % PIECES * 8, cc = walk.j * BC + n * 16 + x;
                if (cc >= t.columns) continue;
                auto of_wave = [&](int w) { return Reference{refs[w][x][0], refs[w][x][1]}; };
                Reference most = of_wave(0);
#pragma unroll
                for (int w = 1; w < WAVES; w++)
                    if (of_wave(w).above(most, a.scale) > 0) most = of_wave(w);
                float v[8] = {0, 0, 0, 0, 0, 0, 0, 0}, sum = 0;
#pragma unroll
                for (int w = 0; w < WAVES; w++) {
                    const float f = __builtin_amdgcn_exp2f(of_wave(w).above(most, a.scale));
                    sum += refs[w][x][2] * f;
#pragma unroll
                    for (int j = 0; j < 8; j++) v[j] += sums[w][x][d + j] * f;
                }
                if (whole) {
                    const int i = cc * a.group_inv >> 16;
                    const int64_t row = (int64_t)(t.first + i) * (a.s.heads * a.s.group) + walk.h * a.s.group + cc - i * a.s.group;
                    *(u4_t*)(a.out + 2 * (row * D + d)) = rounded8<DT>(v, sum == 0 ? 0.0f : 1.0f / sum);
                    if (a.lse && d == 0) a.lse[row] = most.log_sum(sum, a.scale);
                } else {
                    float* to = a.part + (slot * BC + n * 16 + x) * D + d;
                    *(f4_t*)to = f4_t{v[0], v[1], v[2], v[3]};
                    *(f4_t*)(to + 4) = f4_t{v[4], v[5], v[6], v[7]};
                    if (d == 0) a.part_ref[slot * BC + n * 16 + x] = f4_t{most.m, most.base, sum, 0};
                }
            }
        }
        if (WHOLE) return;
        advance<BC, NC == 2>(a.s, walk, t, take);
    }
    if (threadIdx.x < 8) {
        int v = join[0];
#pragma unroll
        for (int i = 1; i < 8; i++) v = threadIdx.x == i ? join[i] : v;
        a.joins[worker * 8 + threadIdx.x] = v;
    }
}

// Joins the parts of the item that a worker left unfinished: its own, and the
// first ones of the workers after it.  A thread has eight channels of a column.
// A launch and a chain of two loads, further parts coming while these are added:
// 4.3 us (drafts), 13 (8192 queries of 64 heads, 29 MB), 11 (64 parts of 200000
// tokens; 15 with each step's loads when it begins).
template <int DT, int D, int BC>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a)
{
    const int worker = blockIdx.x;
    const int32_t* join = a.joins + worker * 8;
    const int parts = join[0], slot0 = join[1], col0 = join[2], columns = join[3], first = join[4], h = join[5];
    if (parts == 0) return;
    constexpr int PIECES = D / 8;
    const int at = threadIdx.x + 256 * blockIdx.y, x = at / PIECES, d = at % PIECES * 8, cc = col0 + x;
    if (x >= BC || cc >= columns) return;
    auto place = [&](int i) { return (int64_t)(i == 0 ? slot0 : 2 * (worker + i)) * BC + x; };
    // some parts at a time (behind the last one that again, which adds nothing): with few columns a long sequence has many
    constexpr int STEP = BC == 16 ? 4 : 2;
    Reference most = kNoReference;
    float sum = 0, v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    f4_t next[STEP][3];
    auto load = [&](int i) {
#pragma unroll
        for (int j = 0; j < STEP; j++) {
            const int64_t p = place(min(i + j, parts - 1));
            const f4_t* from = (const f4_t*)(a.part + p * D + d);
            next[j][0] = a.part_ref[p];
            next[j][1] = from[0];
            next[j][2] = from[1];
        }
    };
    load(0);
    for (int i = 0; i < parts; i += STEP) {
        f4_t r[STEP], u[STEP], w[STEP];
#pragma unroll
        for (int j = 0; j < STEP; j++) {
            r[j] = next[j][0];
            u[j] = next[j][1];
            w[j] = next[j][2];
        }
        if (i + STEP < parts) load(i + STEP);
        const Reference before = most;
#pragma unroll
        for (int j = 0; j < STEP; j++) {
            const Reference x{r[j][0], r[j][1]};
            if (x.above(most, a.scale) > 0) most = x;
        }
        const float g = __builtin_amdgcn_exp2f(before.above(most, a.scale));
        sum *= g;
#pragma unroll
        for (int k = 0; k < 8; k++) v[k] *= g;
#pragma unroll
        for (int j = 0; j < STEP; j++) {
            const float f = i + j < parts ? __builtin_amdgcn_exp2f(Reference{r[j][0], r[j][1]}.above(most, a.scale)) : 0.0f;
            sum += r[j][2] * f;
#pragma unroll
            for (int k = 0; k < 4; k++) {
                v[k] += u[j][k] * f;
                v[4 + k] += w[j][k] * f;
            }
        }
    }
    const int i = cc / a.s.group;
    const int64_t row = (int64_t)(first + i) * (a.s.heads * a.s.group) + h * a.s.group + cc - i * a.s.group;
    *(u4_t*)(a.out + 2 * (row * D + d)) = rounded8<DT>(v, sum == 0 ? 0.0f : 1.0f / sum);
    if (a.lse && d == 0) a.lse[row] = most.log_sum(sum, a.scale);
}

// Most columns of a sequence.
int64_t columns_most(const quick_attention_t& a) { return std::min(a.most, a.T) * (a.q_heads / a.heads); }

// Columns of a workgroup's tile, by the most columns n of a sequence (queries
// and the heads that share keys and values).
// Up to 128 the stream kernel, in tiles of 32 (16 sequences of 2000 to 8000
// tokens, 8 cache heads of 128: n = 40 43 us, 64 44, 96 57, 128 71; the tiled
// one, half of whose waves the first of these leave idle, 57, 60, 65, 72; of 256
// channels n = 80 124 and 162).  Of the tiled forms 256 columns with many queries
// of 128 channels: 8 sequences of 4000, 8 cache heads, n = 2056 311 us, 323 with
// 128; 4096 531 and 570; 16384 (two sequences) 429 and 461.  With fewer the columns
// that its last tile has not cost as much as that gains: n = 1296 216 and 215, 1040
// 178 and 181, 520 115 and 110; 1 to 256 queries, n = 1024 at most, 112 and 108.  Of
// 64 channels, where the vector instructions bound both, 128 is the faster one
// throughout (n = 2048 200 and 193 us, 16384 304 and 299), and of 256 the
// registers do not suffice.
int columns_of(const quick_attention_t& a)
{
    const int64_t n = columns_most(a);
    if (n <= 128) return n <= 16 ? 16 : 32;
    return n >= 2048 && a.D == 128 ? 256 : 128;
}

// Whether a workgroup takes an item each: one tile of a sequence, of so few pages
// that a second launch, and the plan before the first page, cost more than unequal
// lengths do.  Of 8 cache heads of 128 read by 4 each, against shared out: 1
// sequence of 1000 tokens 9.8 us and 13.9, of 3000 12.7 and 13.9, of 4000 15.9 and
// 14.1; 64 of 1500 21.6 and 23.3.  Items that do not all begin at once even out
// when the longest begin first: of 49 to 64 pages 560 items 34.7 and 37.9 (lengths
// of 37 to 4096) or 60.9 and 61.2 (of 3200 to 4096), 960 of them 53.3 and 61.9, or
// 95.9 and 96.4 (700 of 140 sequences, more than are put in order, 51.2 and 48.9,
// or 68.4 and 75.2); 64 of them 17.6 and 13.7, or 17.6 and 17.2; 384 28.7 and 26.9,
// or 43.3 and 44.9 (of 256 channels 58.2 and 53.5, or 82.1 and 81.3).  32 columns
// of 256 channels leave a unit four waves: 16 of 100 to 3000 38 and 34.
bool whole_items(const quick_attention_t& a)
{
    const int64_t n = columns_most(a), items = a.seqs * a.heads;
    if (n > 32) return false;
    return a.table_width <= (n > 16 && a.D > 128 ? 16 : items <= 2 * kUnits ? 48 : kWholePages);
}

int workers_of(const quick_attention_t& a)
{
    // no more than there can be pages of items
    const int64_t group = a.q_heads / a.heads, bc = columns_of(a);
    if (whole_items(a)) return (int)(a.seqs * a.heads);
    const int64_t rows = std::min(a.T, a.seqs * std::min(a.most, a.T));
    const int64_t items = (std::min(a.seqs, a.T) + rows * group / bc + 1) * a.heads;
    const int64_t least = bc > 32 ? kTiledShare : kStreamShare;
    const int64_t most = bc > 32 ? tiled_workers(a.D, bc) : kUnits * stream_resident(a.D, (int)bc / 16);
    const int64_t shares = std::max<int64_t>(1, (a.table_width + least - 1) / least);
    return (int)(items > most / shares ? most : items * shares);
}

template <int DT, int D, int NC>
void launch_stream(const AttnArgs& a, hipStream_t hs)
{
    if (a.whole) {
        // few items: more waves each (whose registers do not suffice for 32 columns of 256 channels)
        if constexpr (D * NC < 512) {
            if (a.workers <= 2 * kUnits) return attn_stream_kernel<DT, D, NC, 8, true><<<a.workers, 512, 0, hs>>>(a);
        }
        return attn_stream_kernel<DT, D, NC, 4, true><<<a.workers, 256, 0, hs>>>(a);
    }
    attn_stream_kernel<DT, D, NC, 4, false><<<a.workers, 256, 0, hs>>>(a);
    attn_join_kernel<DT, D, 16 * NC><<<dim3(a.workers, (2 * NC * D + 255) / 256), 256, 0, hs>>>(a);
}
template <int DT, int D>
void launch_attention(const AttnArgs& a, int columns, hipStream_t hs)
{
    if (columns == 16) launch_stream<DT, D, 1>(a, hs);
    else if (columns == 32) launch_stream<DT, D, 2>(a, hs);
    else {
        launch_tiled_attention(a, DT, D, columns, hs);
        const dim3 grid(a.workers, columns * D / 2048);
        if constexpr (D == 128) {
            if (columns == 256) return attn_join_kernel<DT, D, 256><<<grid, 256, 0, hs>>>(a);
        }
        attn_join_kernel<DT, D, 128><<<grid, 256, 0, hs>>>(a);
    }
}
template <int DT>
void launch_attention(const AttnArgs& a, int64_t D, int columns, hipStream_t hs)
{
    if (D == 64) launch_attention<DT, 64>(a, columns, hs);
    else if (D == 128) launch_attention<DT, 128>(a, columns, hs);
    else launch_attention<DT, 256>(a, columns, hs);
}

int check_attention(const quick_attention_t& a)
{
    if (a.T < 0 || a.T >= (1 << 24) || a.heads < 1 || a.heads > QUICK_KV4_MAX_HEADS || a.q_heads < a.heads ||
        a.q_heads % a.heads != 0 || a.q_heads / a.heads > 64 || a.pages < 1 || a.pages >= (1 << 25) || a.seqs < 0 ||
        a.seqs > QUICK_KV4_MAX_SEQS || a.table_width < 0 || a.table_width >= (1 << 24) || a.most < 1 || a.window < 0 ||
        (a.window && !a.causal) || a.q_token < 0 || a.q_head < 0 || a.q_token >= ((int64_t)1 << 40) ||
        a.q_head >= ((int64_t)1 << 40))
        return QUICK_ERR_SHAPE;
    if (a.D != 64 && a.D != 128 && a.D != 256) return QUICK_ERR_UNSUPPORTED;
    if (a.T * a.q_heads * a.D >= ((int64_t)1 << 40)) return QUICK_ERR_SHAPE;
    return QUICK_OK;
}

}  // namespace

extern "C" size_t quick_kv4_attention_workspace_bytes(const quick_attention_t* p)
{
    if (!p || check_attention(*p) || p->T == 0 || p->seqs == 0 || whole_items(*p)) return 0;
    const size_t w = (size_t)workers_of(*p), c = (size_t)columns_of(*p);
    return w * 32 + 2 * w * c * ((size_t)p->D + 4) * sizeof(float);
}

extern "C" int quick_kv4_attention(const quick_attention_t* p, const void* q, int dtype, const void* cache, const int32_t* table,
                                   const int32_t* lengths, const int32_t* offsets, void* out, float* lse, void* workspace,
                                   size_t workspace_bytes, void* stream)
{
    if (!p || (dtype != QUICK_F16 && dtype != QUICK_BF16)) return QUICK_ERR_INVALID_ARG;
    const int st = check_attention(*p);
    if (st) return st;
    if (p->T == 0 || p->seqs == 0) return QUICK_OK;
    if (!q || !cache || !lengths || !out || (p->table_width && !table)) return QUICK_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(cache, 16) || !aligned(out, 16) || !aligned(table, 4) || !aligned(lengths, 4) ||
        !aligned(offsets, 4) || !aligned(lse, 4) || p->q_token % 8 || p->q_head % 8)
        return QUICK_ERR_ALIGNMENT;
    const size_t need = quick_kv4_attention_workspace_bytes(p);
    if (need && (!workspace || workspace_bytes < need)) return QUICK_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return QUICK_ERR_ALIGNMENT;
    AttnArgs a{};
    a.workers = workers_of(*p);
    a.whole = whole_items(*p);
    // (fewer items begin at once; more sequences than that even out)
    a.ranked = a.whole && a.workers > 2 * kUnits && p->seqs > 1 && p->seqs <= kRanked;
    const int columns = columns_of(*p);
    a.s.lengths = lengths;
    a.s.offsets = offsets;
    a.s.T = (int32_t)p->T;
    a.s.heads = (int32_t)p->heads;
    a.s.group = (int32_t)(p->q_heads / p->heads);
    a.group_inv = (65535 + a.s.group) / a.s.group;
    a.s.seqs = (int32_t)p->seqs;
    a.s.width = (int32_t)p->table_width;
    a.s.most = (int32_t)std::min<int64_t>(p->most, p->T);
    a.s.window = (int32_t)std::min<int64_t>(p->window, 1 << 30);   // (tokens are fewer)
    a.s.causal = p->causal != 0;
    a.s.start = columns > 32 ? kTiledStart : kStreamStart;
    a.q = (const uint8_t*)q;
    a.cache = (const uint8_t*)cache;
    a.table = table;
    a.out = (uint8_t*)out;
    a.lse = lse;
    if (need) {
        a.joins = (int32_t*)workspace;
        a.part = (float*)((uint8_t*)workspace + (size_t)a.workers * 32);
        a.part_ref = (f4_t*)(a.part + 2 * (size_t)a.workers * columns * p->D);
    }
    a.q_token = p->q_token;
    a.q_head = p->q_head;
    a.pages = (int32_t)p->pages;
    // (never zero: a hidden score is -infinity times it)
    a.scale = std::max(std::fabs(p->scale) * 1.44269504088896341f, 1e-30f);
    a.q_sign = p->scale < 0 ? 0x80008000u : 0;
    (void)hipGetLastError();
    if (dtype == QUICK_F16) launch_attention<QUICK_F16>(a, p->D, columns, (hipStream_t)stream);
    else launch_attention<QUICK_BF16>(a, p->D, columns, (hipStream_t)stream);
    return launched();
}
