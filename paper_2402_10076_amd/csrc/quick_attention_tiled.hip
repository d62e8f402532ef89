// Attention over the paged 4-bit cache: many queries of a sequence.
#include "quick_attention_parts.h"

namespace quick {
namespace {

template <int DT>
__device__ __forceinline__ f16_t mfma32(u4_t a, u4_t b, f16_t c)
{
    if constexpr (DT == QUICK_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(bits_as<h8_t>(a), bits_as<h8_t>(b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(bits_as<b8_t>(a), bits_as<b8_t>(b), c, 0, 0, 0);
}

__device__ __forceinline__ float swapped_halves(float v, int lane)
{
    const auto r = __builtin_amdgcn_permlane32_swap(bits_as<uint32_t>(v), bits_as<uint32_t>(v), false, false);
    return bits_as<float>(lane < 32 ? r[1] : r[0]);
}

// What a thread holds of a page on its way to LDS.  NW / 4 waves have tokens 16
// w .. 16 w + 15: of the keys lane (c, g) the words of token c as in the stream
// kernel, or half of them; of the values lane (c, x, y) those of token groups x
// and x + 2, of which it converts half y of each word, or half of that.
template <int D, int NW>
struct Staged {
    static constexpr int SHARE = NW / 4, HALVES = D > 128 ? 2 : 1, VW = D < 128 ? 2 : 4;
    static constexpr int KW = D / 32 / HALVES / SHARE;     // words of keys of each half
    uint32_t k[HALVES][KW], ks[HALVES];
    uint32_t v[HALVES][2][VW], vs[HALVES][2];
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&to)[N], const uint8_t* from)
{
    if constexpr (N == 1) to[0] = *(const uint32_t*)from;
    else if constexpr (N == 2) {
        const u2_t a = *(const u2_t*)from;
        to[0] = a[0];
        to[1] = a[1];
    } else {
        const u4_t a = *(const u4_t*)from;
#pragma unroll
        for (int j = 0; j < 4; j++) to[j] = a[j];
    }
}

template <int D, int NW>
__device__ __forceinline__ void stage(Staged<D, NW>& s, const uint8_t* page, int wave, int lane)
{
    typedef Kv4<D> L;
    typedef Staged<D, NW> S;
    const int c = lane & 15, g = lane >> 4, x = g & 1, w = wave / S::SHARE, part = wave % S::SHARE;
    const uint32_t key = L::kKeys + (w * 16 + c) * (D / 2) + g * (D == 64 ? 8 : 16) + part * 4 * S::KW;
    const uint32_t key_scale = L::kKeyScales + (D == 64 ? g >> 1 : g) * 64 + c * 4;
    const uint32_t value = L::kValues + ((w * 4 + x) * 16 + c) * (4 * S::VW);
    const uint32_t value_scale = L::kValueScales + (D == 64 ? c >> 3 : c >> 2) * 64 + x * 16 + w * 4;
#pragma unroll
    for (int h = 0; h < S::HALVES; h++) {
        load_words(s.k[h], page + key + h * 64);
        s.ks[h] = *(const uint32_t*)(page + key_scale + h * 256);
#pragma unroll
        for (int i = 0; i < 2; i++) {
            load_words(s.v[h][i], page + value + h * 4096 + i * (128 * S::VW));
            s.vs[h][i] = *(const uint32_t*)(page + value_scale + h * 256 + i * 32);
        }
    }
}

// A page in LDS, as operands of the 32 x 32 x 16 instruction, 1 KiB each:
// keys [32 tokens][16 channels], values [16 tokens][32 channels]; lane 32 h + r
// holds its row r's eight of half h.  Row r of value tile i is channel
// 128 (i / 4) + (r % 16) w + 2 (i % 4) + r / 16, w = min(D, 128) / 16; its
// eight tokens are 16 s + 4 h + (0 .. 3) and 8 further on, which are those whose
// scores the lane's column has.
template <int D>
struct Tiles {
    u4_t k[2][D / 16][64];
    u4_t v[4][D / 32][64];
    uint32_t bad[4];       // whether a wave's values have blocks that the type cannot hold
};

// In four steps, so that a caller can put them between other instructions.
template <int DT, int D, int NW>
struct Unstage {
    typedef Staged<D, NW> S;
    float sa[S::HALVES][4], sb[S::HALVES][4];
    uint32_t a[S::HALVES][S::VW], b[S::HALVES][S::VW], mark;

    template <int STEP>
    __device__ __forceinline__ void step(Staged<D, NW>& s, Tiles<D>& to, int wave, int lane)
    {
        const int c = lane & 15, g = lane >> 4, x = g & 1, y = g >> 1, w = wave / S::SHARE, part = wave % S::SHARE;
        if constexpr (STEP == 0) {
            // blocks beyond the type: of keys they get the scale of NaN, of values they leave the product
            mark = 0;
            uint32_t any = 0;
#pragma unroll
            for (int h = 0; h < S::HALVES; h++) any |= beyond<DT>(s.ks[h]) | beyond<DT>(s.vs[h][0]) | beyond<DT>(s.vs[h][1]);
            if (__ballot(any != 0)) {
                seldom();
#pragma unroll
                for (int h = 0; h < S::HALVES; h++) {
                    s.ks[h] |= whole_bytes(beyond<DT>(s.ks[h]));
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const uint32_t bits = beyond<DT>(s.vs[h][i]);
                        mark |= bits;
                        s.vs[h][i] &= ~whole_bytes(bits);
                    }
                }
            }
        }
        if constexpr (STEP == 3) {
            const uint64_t any = __ballot(mark != 0);
            to.bad[w] = any != 0;     // (every lane the same)
        }
#pragma unroll
        for (int h = 0; h < S::HALVES; h++) {
            if constexpr (STEP == 0) {
                const float scale = bits_as<float>(__builtin_amdgcn_alignbit(s.ks[h], s.ks[h], 8 * w + 9));     // (byte w)
#pragma unroll
                for (int j = 0; j < S::KW; j++) {
                    // word n of a lane: channels 8 n .. of its 32 (D == 64: 16)
                    const int n = part * S::KW + j, step = D == 64 ? g : 8 * h + 2 * g + n / 2;
                    to.k[w / 2][step][n % 2 * 32 + w % 2 * 16 + c] = code_words<DT>(s.k[h][j], scale);
                }
            }
            if constexpr (STEP == 1) {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    sa[h][e] = scale_of(s.vs[h][0], e);
                    sb[h][e] = scale_of(s.vs[h][1], e);
                }
#pragma unroll
                for (int j = 0; j < S::VW; j++) {
                    // this lane's bytes of each token to the front
                    const int by = D == 64 ? 8 * y : 16 * y + 8 * part;
                    a[h][j] = s.v[h][0][j] >> by;
                    b[h][j] = s.v[h][1][j] >> by;
                }
            }
            if constexpr (STEP >= 2) {
                u4_t lo, hi;
                const int tile = D == 64 ? y : 4 * h + (S::SHARE == 1 ? 2 * y + STEP - 2 : 2 * y + part);
                if constexpr (STEP == 2 || (D > 64 && S::SHARE == 1)) {
                    value_words<DT, S::VW, STEP - 2>(a[h], b[h], sa[h], sb[h], lo, hi);
                    to.v[w][tile][x * 32 + c] = lo;
                    to.v[w][tile][x * 32 + 16 + c] = hi;
                }
            }
        }
    }
};

// Blocks of values that the type cannot hold make NaN of the columns that see
// them (they are zero in the tiles).  Seldom run.
template <int DT, int D>
__device__ void spoil(f16_t (&o)[D / 32], const uint8_t* page, int lo, int hi, int lane)
{
    typedef Kv4<D> L;
    for (int block = 0; block < D / 32; block++) {
        bool any = false;
        for (int t = 0; t < kPage; t++) {
            const uint32_t s = page[L::value_scale(t, block)];
            any |= beyond<DT>(s) != 0 && t >= lo && t < hi;
        }
        if (!any) continue;
        // a lane's rows 8 b + 4 h + i of tile j are of block 2 (b % 2) + h of their 128 channels (D == 64: b % 2)
#pragma unroll
        for (int j = 0; j < D / 32; j++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int b = i / 4 % 2, mine = D == 64 ? b : 4 * (j / 4) + 2 * b + (lane >> 5);
                if (mine == block) o[j][i] = NAN;
            }
    }
}

// Many queries of a sequence: 32 NW columns (a column being a query and one of
// the heads that share keys and values), 32 a wave.  The workgroup converts a
// page to 16-bit operands in LDS, the next one while it multiplies; a wave has
// its queries, its sums of values and the scores in registers.  Scores are
// transposed, keys . queries^T, so that a lane's weights of a column are its
// operand of values^T . weights as they stand.  Half a page at a time, and the
// scores of the next half beside the weights of this one, so that the matrix
// instructions of the one run under the vector instructions of the other.
// Bound by both: of 128 channels a page is 1024 cycles of matrix instructions for
// a wave and some 1250 of vector ones (32 exponentials a lane among them), which overlap
// in part: 8192 queries of 64 heads 1110 us, 990 TFLOP/s, matrix instructions
// busy 45 % of the cycles.  Of 64 channels it is 512 and 1100: the vector ones.  Of
// 256 a wave's sums and queries fill one register file, and moves between the two
// are a third to a half of the vector instructions: 2 sequences of 4096 tokens,
// the last 2048 as queries, 32 heads on 8, 662 us, 620 TFLOP/s.
template <int DT, int D, int NW, int NB>
__global__ __launch_bounds__(64 * NW, D > 128 ? 1 : 2) void attn_tiled_kernel(AttnArgs a)
{
    typedef Kv4<D> L;
    constexpr int BC = 32 * NW, KS = D / 16, VT = D / 32, T = (D < 128 ? D : 128) / 16;
    // the last step's addresses are not kept over the loop, which leaves them no registers (with 64 channels it does, and
    // a window's many items take 78.5 us for 76.5 so)
    constexpr bool LATE = D > 64;
    __shared__ Tiles<D> tiles[NB];
    __shared__ uint32_t aways[2][NW];   // whether a wave of this item (of the next one) has met far scores
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5;
    const int worker = blockIdx.x;
    Walk walk = find_share<BC, true>(a.s, a.workers, worker, kTiledShare);
    int join[8] = {0, 0, 0, 0, 0, 0, 0, 0}, odd = 0;
    for (bool first = true; walk.left > 0 && walk.b < a.s.seqs; first = false) {
        const Tile t = tile_of<BC>(a.s, walk.b, walk.j);
        const int take = (int)min((int64_t)(t.cost - walk.at), walk.left);
        if (left_to_next(a.s, walk, t, take)) break;
        int p0, p1;
        pages_of(a.s, t, walk.at, take, p0, p1);
        // (columns behind the last are that one again, and go nowhere)
        const int place = walk.j * BC + wave * 32 + (lane & 31), cc = min(place, t.columns - 1), i = cc / a.s.group;
        const bool live = place < t.columns, work = walk.j * BC + wave * 32 < t.columns;
        const int pos = t.base + i;
        const int hi = a.s.causal ? min(pos + 1, t.length) : t.length;
        const int lo = a.s.window ? max(0, pos + 1 - a.s.window) : 0;
        const int64_t head = (int64_t)walk.h * a.s.group + cc - i * a.s.group;
        u4_t q[KS];
        {
            const uint8_t* from = a.q + 2 * ((int64_t)(t.first + i) * a.q_token + head * a.q_head) + half * 16;
#pragma unroll
            for (int s = 0; s < KS; s++) q[s] = *(const u4_t*)(from + s * 32);
        }
        Reference ref;
        bool away = false;
        float l;
        f16_t o[VT];
        const int32_t* table = a.table + (int64_t)walk.b * a.s.width;
        const uint8_t* head_of_cache = a.cache + walk.h * L::kBytes;
        const uint32_t stride = a.s.heads * L::kBytes;
        const int count = max(0, p1 - p0);
        Staged<D, NW> next;
        const uint8_t* next_page = a.cache;
        bool next_ok = false;
        int id = 0;
        // page n to registers (the id of the one after it, too); behind the last one that again
        auto fetch = [&](int n) {
            const int x = (int)uniform((uint32_t)id);
            id = table[min(p0 + n + 1, p1 - 1)];
            next_ok = x >= 0 && x < a.pages;
            next_page = head_of_cache + (int64_t)(next_ok ? x : 0) * stride;
            stage<D, NW>(next, next_page, wave, lane);
        };
        // scores of half x of a page
        auto scores = [&](const Tiles<D>& w, int x, f16_t& s) {
#pragma unroll
            for (int r = 0; r < 16; r++) s[r] = 0;
#pragma unroll
            for (int k = 0; k < KS; k++) s = mfma32<DT>(w.k[x][k][lane], q[k], s);
        };
        // hides what a column does not see of those, and sets its reference
        auto refer = [&](auto form, f16_t& s, int token0, bool ok) {
            constexpr bool FAR = decltype(form)::far;
            if (token0 + 32 > t.all_hi || token0 < t.all_lo || !ok) {
                seldom();
                const int from = token0 + 4 * half;
                const uint32_t bits = bits_between(lo - from, (ok ? hi : from) - from);
#pragma unroll
                for (int r = 0; r < 16; r++) s[r] = where_bit(s[r], bits, r / 4 * 8 + r % 4);
            }
            float top = s[0];
#pragma unroll
            for (int r = 0; r < 16; r++) top = fmaxf(top, s[r]);
            if (FAR || __ballot(fmaf(top, a.scale, -ref.m) > kRoom<DT>)) {
                seldom();
                const float f = ref.raise<DT, FAR>(fmaxf(top, swapped_halves(top, lane)), a.scale, away);
                l *= f;
#pragma unroll
                for (int j = 0; j < VT; j++)
#pragma unroll
                    for (int r = 0; r < 16; r++) o[j][r] *= f;
            }
            if constexpr (FAR) {
#pragma unroll
                for (int r = 0; r < 16; r++) s[r] -= ref.base;
            }
        };
        // Half x of page w: s's weights and the values they weigh; beside them the scores s1 of half x1 of page w1.
        // Each step of those has a matrix instruction, a load of an operand four steps ahead and a share of the
        // weights, and the compiler is kept from gathering them.
        constexpr int AHEAD = 4, PV = 2 * VT;
        u4_t f[AHEAD];
        auto first_operands = [&](const Tiles<D>& w1, int x1) {
#pragma unroll
            for (int k = 0; k < AHEAD; k++) f[k] = w1.k[x1][k][lane];
        };
        auto half_page = [&](const Tiles<D>& w, int x, const f16_t& s, const Tiles<D>& w1, int x1, f16_t& s1, auto beside) {
            u4_t p[2];
#pragma unroll
            for (int r = 0; r < 16; r++) s1[r] = 0;
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int k = 0; k < KS; k++) {
                __builtin_amdgcn_sched_barrier(0);
                s1 = mfma32<DT>(f[k % AHEAD], q[k], s1);
                if (k + AHEAD < KS) f[k % AHEAD] = w1.k[x1][k + AHEAD][lane];
                else f[k % AHEAD] = w.v[2 * x + (k + AHEAD - KS) / VT][(k + AHEAD - KS) % VT][lane];
#pragma unroll
                for (int r = 16 * k / KS / 2 * 2; r < 16 * (k + 1) / KS / 2 * 2; r += 2) {
                    const float u = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale, -ref.m));
                    const float v = __builtin_amdgcn_exp2f(fmaf(s[r + 1], a.scale, -ref.m));
                    l += u + v;
                    p[r / 8][r % 8 / 2] = pair16<DT>(u, v);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int k = 0; k < PV; k++) {
                o[k % VT] = mfma32<DT>(f[k % AHEAD], p[k / VT], o[k % VT]);
                if (k + AHEAD < PV) f[k % AHEAD] = w.v[2 * x + (k + AHEAD) / VT][(k + AHEAD) % VT][lane];
                beside(k);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto begin = [&] {
            ref = kNoReference;
            l = 0;
#pragma unroll
            for (int j = 0; j < VT; j++)
#pragma unroll
                for (int r = 0; r < 16; r++) o[j][r] = 0;
        };
        // blocks of a page that the type cannot hold
        auto see_bad = [&](const Tiles<D>& w, const uint8_t* page, int token0, bool ok) {
            const u4_t bad = *(const u4_t*)w.bad;
            if (uniform(bad[0] | bad[1] | bad[2] | bad[3])) spoil<DT, D>(o, page, lo - token0, (ok ? hi : 0) - token0, lane);
        };
        begin();
        const uint8_t *page = a.cache, *page1 = a.cache;
        bool ok = false;
        f16_t s;
        int at = 0;
        if (count) {
            id = table[p0];
            fetch(0);
            if (a.q_sign) {
                seldom();
#pragma unroll
                for (int s = 0; s < KS; s++) q[s] ^= a.q_sign;
            }
            Unstage<DT, D, NW> un;
            un.template step<0>(next, tiles[0], wave, lane);
            un.template step<1>(next, tiles[0], wave, lane);
            un.template step<2>(next, tiles[0], wave, lane);
            un.template step<3>(next, tiles[0], wave, lane);
            ok = next_ok;
            page = next_page;
            fetch(1);
            __syncthreads();
            if (work) scores(tiles[0], 0, s);
        }
        for (int n = 0; n < count; n++) {
            const Tiles<D>& w = tiles[at];
            const int to = at + 1 == NB ? 0 : at + 1;
            const int token0 = (p0 + n) * kPage;
            f16_t s1;
            bool ok1 = false;
            Unstage<DT, D, NW> un;
            // (behind the last page that one again, which nothing reads)
            auto on = [&](int k) {
                if (k == 0) un.template step<0>(next, tiles[to], wave, lane);
                if (k == PV / 4) un.template step<1>(next, tiles[to], wave, lane);
                if (k == PV / 2) un.template step<2>(next, tiles[to], wave, lane);
                if (k == 3 * PV / 4) {
                    un.template step<3>(next, tiles[to], wave, lane);
                    ok1 = next_ok;
                    page1 = next_page;
                    fetch(n + 2);
                }
            };
            auto all_on = [&] {
                on(0);
                on(PV / 4);
                on(PV / 2);
                on(3 * PV / 4);
            };
            if (work) {
                first_operands(w, 1);
                refer(Near{}, s, token0, ok);
                if constexpr (NB > 2) half_page(w, 0, s, w, 1, s1, on);
                else half_page(w, 0, s, w, 1, s1, [](int) {});
            } else if (NB > 2) all_on();
            if constexpr (NB == 2) {
                // the tile that is overwritten now has been read
                __syncthreads();
                all_on();
            }
            __syncthreads();
            if (work) {
                first_operands(tiles[to], 0);
                refer(Near{}, s1, token0 + 32, ok);
                half_page(w, 1, s1, tiles[to], 0, s, [](int) {});
                see_bad(w, page, token0, ok);
            }
            ok = ok1;
            page = page1;
            at = to;
        }
        // the next item's first page goes where the last one's lies
        const uint32_t gone = __ballot(away) != 0;
        aways[odd][wave] = gone;     // (every lane the same)
        __syncthreads();
        uint32_t any = 0;
#pragma unroll
        for (int w = 0; w < NW; w++) any |= aways[odd][w];
        odd ^= 1;
        if (__builtin_expect(uniform(any) != 0, 0)) {
            // far scores: the pages again, one after the other
            seldom();
            begin();
            for (int n = 0; n < count; n++) {
                const Tiles<D>& w = tiles[0];
                const int token0 = (p0 + n) * kPage;
                id = table[p0 + n];
                fetch(n);
                Unstage<DT, D, NW> un;
                un.template step<0>(next, tiles[0], wave, lane);
                un.template step<1>(next, tiles[0], wave, lane);
                un.template step<2>(next, tiles[0], wave, lane);
                un.template step<3>(next, tiles[0], wave, lane);
                __syncthreads();
                if (work) {
#pragma unroll 1
                    for (int x = 0; x < 2; x++) {
                        // (the scores beside the weights are these again)
                        scores(w, x, s);
                        first_operands(w, x);
                        refer(Far{}, s, token0 + 32 * x, next_ok);
                        f16_t again;
                        half_page(w, x, s, w, x, again, [](int) {});
                    }
                    see_bad(w, next_page, token0, next_ok);
                }
                __syncthreads();
            }
        }
        const bool whole = walk.at == 0 && take == t.cost;
        const int64_t slot = 2 * worker + (first ? 0 : 1);
        if (walk.at == 0 && !whole) {
            set_join(join, walk, t, BC, take, (int)slot);
        }
        if (live) {
            const int lane = LATE ? late(threadIdx.x & 63) : threadIdx.x & 63, half = lane >> 5;
            l += swapped_halves(l, lane);
            const int64_t row = (int64_t)(t.first + i) * (a.s.heads * a.s.group) + head;
            const float f = !whole ? 1.0f : l == 0 ? 0.0f : 1.0f / l;
            float* part = a.part + (slot * BC + wave * 32 + (lane & 31)) * D;
#pragma unroll
            for (int h = 0; h < (D > 128 ? 2 : 1); h++)
#pragma unroll
                for (int b = 0; b < 2; b++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        const int channel = h * 128 + (8 * b + 4 * half + r) * T;
                        float v[T];
#pragma unroll
                        for (int j = 0; j < T; j++) v[j] = o[h * 4 + j / 2][(b + 2 * (j % 2)) * 4 + r];
                        if (whole) {
                            uint8_t* to = a.out + 2 * (row * D + channel);
                            if constexpr (T == 8) *(u4_t*)to = rounded8<DT>(v, f);
                            else *(u2_t*)to = u2_t{pair16<DT>(v[0] * f, v[1] * f), pair16<DT>(v[2] * f, v[3] * f)};
                        } else {
#pragma unroll
                            for (int j = 0; j < T; j += 4) *(f4_t*)(part + channel + j) = f4_t{v[j], v[j + 1], v[j + 2], v[j + 3]};
                        }
                    }
            if (half == 0) {
                if (!whole) a.part_ref[slot * BC + wave * 32 + lane] = f4_t{ref.m, ref.base, l, 0};
                else if (a.lse) a.lse[row] = ref.log_sum(l, a.scale);
            }
        }
        advance<BC, true>(a.s, walk, t, take);
    }
    if (threadIdx.x < 8) {
        int v = join[0];
#pragma unroll
        for (int x = 1; x < 8; x++) v = threadIdx.x == x ? join[x] : v;
        a.joins[worker * 8 + threadIdx.x] = v;
    }
}

template <int DT, int D>
void launch(const AttnArgs& a, int columns, hipStream_t hs)
{
    if constexpr (D == 128) {
        if (columns == 256) return attn_tiled_kernel<DT, D, 8, 3><<<a.workers, 512, 0, hs>>>(a);
    }
    attn_tiled_kernel<DT, D, 4, D == 64 ? 3 : 2><<<a.workers, 256, 0, hs>>>(a);
}
template <int DT>
void launch(const AttnArgs& a, int64_t D, int columns, hipStream_t hs)
{
    if (D == 64) launch<DT, 64>(a, columns, hs);
    else if (D == 128) launch<DT, 128>(a, columns, hs);
    else launch<DT, 256>(a, columns, hs);
}

}  // namespace

void launch_tiled_attention(const AttnArgs& a, int dtype, int64_t D, int columns, hipStream_t hs)
{
    if (dtype == QUICK_F16) launch<QUICK_F16>(a, D, columns, hs);
    else launch<QUICK_BF16>(a, D, columns, hs);
}

}  // namespace quick
