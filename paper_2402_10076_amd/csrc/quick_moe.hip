// Around the grouped products of a mixture-of-experts layer: the router's
// choice and the expert-sorted order of the routed rows, and the weighted sum
// that joins a token's expert rows.
#include <algorithm>

#include "quick_device.h"
#include "quick_moe.h"

namespace {

using namespace quick;

constexpr int kMaxE = QUICK_MAX_EXPERTS;
constexpr int kWaves = 16;              // of a routing workgroup
constexpr int kThreads = 64 * kWaves;
constexpr int kWgs = 512;               // routing workgroups of many tokens: two for each compute unit
constexpr int kMaxTokens = 65535;       // of a routing workgroup: its counts have 16 bits
constexpr int kSortEntries = 1024;      // (token, choice) of a sorting workgroup, about

struct RouteArgs {
    const void* logits;
    const float* bias;
    int32_t* ids;
    float* weights;
    int32_t* offsets;
    int32_t* rows;
    int32_t* slots;
    uint16_t* counts;      // [workgroups][E, rounded up to 2] rows of a workgroup's tokens at each expert
    int32_t T, E, topk, groups, topk_groups, group_best, group_size;
    int32_t group_lanes;   // lanes of a group, where it is a power of two of whole ones (else 0)
    uint32_t group_inv;    // e / group_size == e * group_inv >> 20 for e < 512
    int32_t tokens_per_wg, wgs, wgs_per_sort;
    int32_t sigmoid, renorm, by_score;   // by_score: the choice goes by s (+ bias), not by the logits
    float scale;
};

// Reduction over groups of W lanes that leaves every lane with the result:
// exchanges with lane ^ 1, lane ^ 2, 7 - lane of each eight, 15 - lane of each
// sixteen (the halves are uniform by then), then rows of 16 lanes and halves of
// the wave change places.
template <int CTRL, class T>
__device__ __forceinline__ T swapped(T v)
{
    return bits_as<T>(__builtin_amdgcn_mov_dpp(bits_as<int>(v), CTRL, 0xF, 0xF, true));
}
template <int W, class T, class F>
__device__ __forceinline__ T reduce(T v, F f)
{
    v = f(v, swapped<0xB1>(v));
    v = f(v, swapped<0x4E>(v));
    v = f(v, swapped<0x141>(v));
    v = f(v, swapped<0x140>(v));
    if constexpr (W >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(bits_as<uint32_t>(v), bits_as<uint32_t>(v), false, false);
        v = f(bits_as<T>(r[0]), bits_as<T>(r[1]));
    }
    if constexpr (W >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(bits_as<uint32_t>(v), bits_as<uint32_t>(v), false, false);
        v = f(bits_as<T>(r[0]), bits_as<T>(r[1]));
    }
    return v;
}

template <int DT>
__device__ __forceinline__ float logit(const void* p, int64_t i)
{
    if constexpr (DT == QUICK_F32) return ((const float*)p)[i];
    else return from16<DT>(((const uint16_t*)p)[i]);
}

// An integer that orders as the float does, NaN as -inf and -0 as 0; and back.
// 0 is below every float's key: what a lane exchange without a source reads.
typedef uint32_t key_t;
__device__ __forceinline__ key_t order_key(float v)
{
    const int i = bits_as<int>(v != v ? -INFINITY : v + 0.0f);
    return (key_t)(i ^ ((i >> 31) | (int)0x80000000));
}
__device__ __forceinline__ float key_value(key_t k)
{
    return bits_as<float>(k ^ ((key_t)((int)~k >> 31) | 0x80000000u));
}
constexpr key_t kExcluded = 0;

// Orders this wave's LDS accesses before those that follow.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Ints of LDS that one token's choice among groups takes.
__device__ __host__ __forceinline__ int group_ints(int E, int groups) { return E + 2 * groups; }

// Largest key of the wave, in a scalar register: running maxima along each row
// of 16 lanes (1, 2, 4 and 8 lanes up), then over the rows, end in lane 63.
template <int CTRL>
__device__ __forceinline__ key_t max_from(key_t v)
{
    return max(v, (key_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ key_t max_of_wave(key_t v)
{
    v = max_from<0x111>(v);
    v = max_from<0x112>(v);
    v = max_from<0x114>(v);
    v = max_from<0x118>(v);
    v = max_from<0x142>(v);
    v = max_from<0x143>(v);
    return (key_t)__builtin_amdgcn_readlane((int)v, 63);
}

// The two largest keys of 2^n lanes, n = log2 of `lanes`, in all of them.
__device__ __forceinline__ void best_two(int lanes, key_t& k1, key_t& k2)
{
    auto merge = [&](key_t o1, key_t o2) {
        k2 = max(min(k1, o1), max(k2, o2));
        k1 = max(k1, o1);
    };
    if (lanes >= 2) merge(swapped<0xB1>(k1), swapped<0xB1>(k2));
    if (lanes >= 4) merge(swapped<0x4E>(k1), swapped<0x4E>(k2));
    if (lanes >= 8) merge(swapped<0x141>(k1), swapped<0x141>(k2));
    if (lanes >= 16) merge(swapped<0x140>(k1), swapped<0x140>(k2));
    if (lanes >= 32) merge((key_t)__shfl_xor((int)k1, 16), (key_t)__shfl_xor((int)k2, 16));
}

// Keys of all experts outside the groups that stay become kExcluded.  Place i
// of a lane's V is expert lane * V + i.
template <int W, int V>
__device__ __forceinline__ void keep_groups(const RouteArgs& a, int lane, int* lds, key_t (&key)[V])
{
    if (a.group_lanes) {
        // a group is that many whole lanes (W == 64): all in registers
        key_t k1 = kExcluded, k2 = kExcluded;
#pragma unroll
        for (int i = 0; i < V; i++) {
            k2 = max(k2, min(k1, key[i]));
            k1 = max(k1, key[i]);
        }
        best_two(a.group_lanes, k1, k2);
        const key_t mine = order_key(a.group_best == 1 || a.group_size == 1 ? key_value(k1) : key_value(k1) + key_value(k2));
        const int g = lane / a.group_lanes;
        int before = 0;
        for (int h = 0; h < a.groups; h++) {
            const key_t other = (key_t)__builtin_amdgcn_readlane((int)mine, h * a.group_lanes);
            before += other > mine || (other == mine && h < g);
        }
#pragma unroll
        for (int i = 0; i < V; i++) key[i] = before < a.topk_groups ? key[i] : kExcluded;
        return;
    }
    key_t* keys = (key_t*)lds;
    key_t* sum = keys + a.E;
    int* keep = (int*)(sum + a.groups);
#pragma unroll
    for (int i = 0; i < V; i++)
        if (lane * V + i < a.E) keys[lane * V + i] = key[i];
    wave_fence();
    // a lane per group: its one or two best
    for (int g = lane; g < a.groups; g += W) {
        key_t k1 = kExcluded, k2 = kExcluded;
        int at = g % a.group_size;    // lanes start at different banks
#pragma unroll 8
        for (int j = 0; j < a.group_size; j++) {
            const key_t k = keys[g * a.group_size + at];
            at = at + 1 == a.group_size ? 0 : at + 1;
            k2 = max(k2, min(k1, k));
            k1 = max(k1, k);
        }
        sum[g] = order_key(a.group_best == 1 || a.group_size == 1 ? key_value(k1) : key_value(k1) + key_value(k2));
    }
    wave_fence();
    // ... and how many groups come before it
    for (int g = lane; g < a.groups; g += W) {
        const key_t mine = sum[g];
        int before = 0;
        for (int h = 0; h < a.groups; h++) before += sum[h] > mine || (sum[h] == mine && h < g);
        keep[g] = before < a.topk_groups;
    }
    wave_fence();
#pragma unroll
    for (int i = 0; i < V; i++) {
        const uint32_t e = lane * V + i;
        if (e < (uint32_t)a.E && !keep[e * a.group_inv >> 20]) key[i] = kExcluded;
    }
    wave_fence();
}

// The choice for one token by W >= topk lanes, V experts each (V == 1 unless
// W == 64), all in registers.  A lane sorts its own; then topk times the
// largest first key of all lanes is taken from the lowest lane that has it,
// which is the lowest expert.  Returns to lane j its j-th expert and weight.
// Every sum is taken over a lane's places, then across the lanes: one order.
// A token is some 600 vector instructions of its wave (256 experts in groups,
// 8 choices), and that is the bound of many: 8192 such tokens 14.0 us (with a
// maximum over all places in each of the topk turns and the groups through LDS
// 17.3).
template <int DT, int W, int V>
__device__ __forceinline__ void choose(const RouteArgs& a, int t, int lane, int* lds, int* my_id, float* my_weight)
{
    static_assert(V == 1 || W == 64, "several experts a lane in whole waves only");
    float x[V], s[V];
    key_t key[V];
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int e = lane * V + i;
        x[i] = e < a.E ? logit<DT>(a.logits, (int64_t)t * a.E + e) : -INFINITY;
    }
    if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < V; i++) s[i] = 1.0f / (1.0f + expf(-x[i]));
    } else {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < V; i++) m = fmaxf(m, x[i]);
        m = reduce<W>(m, [](float p, float q) { return fmaxf(p, q); });
        float sum = 0;
#pragma unroll
        for (int i = 0; i < V; i++) {
            s[i] = x[i] == -INFINITY ? 0.0f : expf(x[i] - m);
            sum += s[i];
        }
        sum = reduce<W>(sum, [](float p, float q) { return p + q; });
        const bool empty = sum == 0.0f;    // a row of -inf alone
#pragma unroll
        for (int i = 0; i < V; i++) s[i] = empty ? 0.0f : s[i] / sum;
    }
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int e = lane * V + i;
        float c = a.by_score ? s[i] : x[i];
        if (a.bias) c = c + a.bias[min(e, a.E - 1)];
        key[i] = e < a.E ? order_key(c) : kExcluded;
    }
    if (a.groups > 1) keep_groups<W, V>(a, lane, lds, key);
    float sum = 0, w = 0;
    int id = 0;
    if constexpr (W == 64) {
        // descending, equal keys in the order of the experts
        int expert[V];
#pragma unroll
        for (int i = 0; i < V; i++) expert[i] = lane * V + i;
#pragma unroll
        for (int n = V - 1; n > 0; n--)
#pragma unroll
            for (int i = 0; i < n; i++) {
                const bool turn = key[i + 1] > key[i];
                const key_t k = key[i];
                const int e = expert[i];
                key[i] = turn ? key[i + 1] : k;
                key[i + 1] = turn ? k : key[i + 1];
                expert[i] = turn ? expert[i + 1] : e;
                expert[i + 1] = turn ? e : expert[i + 1];
            }
        for (int j = 0; j < a.topk; j++) {
            const int from = __builtin_ctzll(__ballot(key[0] == max_of_wave(key[0])));
            const int e = __builtin_amdgcn_readlane(expert[0], from);
            if (lane == j) id = e;
            if (lane == from) {
#pragma unroll
                for (int i = 0; i + 1 < V; i++) {
                    key[i] = key[i + 1];
                    expert[i] = expert[i + 1];
                }
                key[V - 1] = kExcluded;
            }
        }
#pragma unroll
        for (int i = 0; i < V; i++) {
            const float v = __shfl(s[i], id / V);
            w = id % V == i ? v : w;
        }
    } else {
        const int first = (int)(threadIdx.x & 63) & ~(W - 1);
        for (int j = 0; j < a.topk; j++) {
            const key_t best = reduce<W>(key[0], [](key_t p, key_t q) { return max(p, q); });
            const uint64_t m = __ballot(key[0] == best) >> first & ((1ull << W) - 1);
            const int e = __builtin_ctzll(m);
            if (lane == j) id = e;
            if (lane == e) key[0] = kExcluded;
        }
        w = __shfl(s[0], first + id);
    }
    if (lane >= a.topk) w = 0;
    if (a.renorm) {
        sum = reduce<W>(w, [](float p, float q) { return p + q; });
        w = sum == 0.0f ? 0.0f : w / sum;
    }
    *my_id = id;
    *my_weight = w * a.scale;
}

// Exclusive sums of n <= 512 values in LDS by one wave, in place; the total
// goes to at[n].
__device__ __forceinline__ void scan_wave(uint32_t* at, int n, int lane)
{
    uint32_t v[kMaxE / 64], sum = 0;
#pragma unroll
    for (int i = 0; i < kMaxE / 64; i++) {
        const int e = lane * (kMaxE / 64) + i;
        v[i] = e < n ? at[e] : 0;
        sum += v[i];
    }
    uint32_t run = sum;
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = (uint32_t)__shfl_up((int)run, d);
        if (lane >= d) run += o;
    }
    uint32_t before = run - sum;
#pragma unroll
    for (int i = 0; i < kMaxE / 64; i++) {
        const int e = lane * (kMaxE / 64) + i;
        if (e < n) at[e] = before;
        before += v[i];
    }
    if (lane == 63) at[n] = run;
}

// Places n entries (token, choice), the first one `first`, into the sorted
// order: base[e] is where the first of them for expert e goes.  Each wave
// takes a run of entries; its rank inside 64 is the number of lower lanes with
// the same expert.
__device__ __forceinline__ void place_entries(const RouteArgs& a, int64_t first, int n, const uint32_t* base,
                                              uint32_t* wave_at)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int per = (n + kWaves * 64 - 1) / (kWaves * 64) * 64;
    const int lo = wave * per, hi = min(n, lo + per);
    const int32_t* ids = a.ids + first;
    for (int i = threadIdx.x; i < kWaves * a.E; i += kThreads) wave_at[i] = 0;
    __syncthreads();
    uint32_t* mine = wave_at + wave * a.E;
    for (int j = lo + lane; j < hi; j += 64) atomicAdd(&mine[ids[j]], 1u);
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kThreads) {
        uint32_t run = base[e];
        for (int w = 0; w < kWaves; w++) {
            const uint32_t c = wave_at[w * a.E + e];
            wave_at[w * a.E + e] = run;
            run += c;
        }
    }
    __syncthreads();
    int bits = 0;
    while ((1 << bits) < a.E) bits++;
    for (int j0 = lo; j0 < hi; j0 += 64) {
        const int j = j0 + lane;
        const bool live = j < hi;
        const int e = live ? ids[j] : 0;
        uint64_t same = __ballot(live);
        for (int b = 0; b < bits; b++) {
            const uint64_t m = __ballot(e >> b & 1);
            same &= (e >> b & 1) ? m : ~m;
        }
        if (live) {
            const int rank = __popcll(same & ((1ull << lane) - 1));
            const uint32_t pos = mine[e] + rank;
            a.rows[pos] = (int32_t)((uint32_t)(first + j) / (uint32_t)a.topk);
            a.slots[first + j] = (int32_t)pos;
            wave_fence();
            if (rank == 0) mine[e] += __popcll(same);
        }
        wave_fence();
    }
}

// Choices of a workgroup's tokens, 64 / W tokens a wave at a time.  With one
// workgroup also the sorted order; otherwise its counts.
// A few tokens are bound by latency, each being a chain of topk maxima over
// lanes, so a workgroup takes few of them (16 waves of 64 / W) and the launch as
// many workgroups; many tokens by the vector instructions (choose).
template <int DT, int W, int V>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a)
{
    extern __shared__ int lds[];
    uint32_t* count = (uint32_t*)lds;                // [E + 1]
    uint32_t* wave_at = count + kMaxE + 4;           // [waves][E], or the tokens' groups
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & (W - 1), sub = (threadIdx.x & 63) / W;
    constexpr int PER = kWaves * 64 / W;
    const int t0 = blockIdx.x * a.tokens_per_wg, t1 = min(a.T, t0 + a.tokens_per_wg);
    for (int e = threadIdx.x; e < a.E; e += kThreads) count[e] = 0;
    __syncthreads();
    int* mine = (int*)wave_at + (wave * (64 / W) + sub) * group_ints(a.E, a.groups);
    for (int t = t0; t < t1; t += PER) {
        const int mt = t + wave * (64 / W) + sub;
        // lanes of one wave choose together; those past the end repeat the last token
        int id;
        float w;
        choose<DT, W, V>(a, min(mt, t1 - 1), lane, mine, &id, &w);
        if (mt < t1 && lane < a.topk) {
            const int64_t at = (int64_t)mt * a.topk + lane;
            a.ids[at] = id;
            a.weights[at] = w;
            atomicAdd(&count[id], 1u);
        }
    }
    __syncthreads();
    if (a.counts) {
        const int width = (a.E + 1) & ~1;
        for (int e = threadIdx.x; e < width; e += kThreads)
            a.counts[(int64_t)blockIdx.x * width + e] = e < a.E ? (uint16_t)count[e] : 0;
        return;
    }
    if (threadIdx.x < 64) scan_wave(count, a.E, threadIdx.x);
    __syncthreads();
    for (int e = threadIdx.x; e <= a.E; e += kThreads) a.offsets[e] = (int32_t)count[e];
    place_entries(a, 0, a.T * a.topk, count, wave_at);
}

// The sorted order of the tokens of wgs_per_sort routing workgroups: where the
// first of them for each expert goes is the sum of all counts of lower experts
// and of this one's in lower workgroups.  Every workgroup adds all counts up
// (512 x E of 16 bits, from L2): 8192 tokens at 8 of 256 experts take 11.9 us,
// most of it the latency of one phase after the other (24 with one load of a
// thread under way at a time).
__global__ __launch_bounds__(kThreads) void route_sort_kernel(RouteArgs a)
{
    extern __shared__ int lds[];
    uint32_t* base = (uint32_t*)lds;                 // [E + 1]
    uint32_t* before = base + kMaxE + 4;             // [E]
    uint32_t* wave_at = before + kMaxE;              // [waves][E]
    for (int e = threadIdx.x; e < a.E; e += kThreads) base[e] = before[e] = 0;
    __syncthreads();
    // thread (slice, pair) adds up every `slices`-th workgroup's counts of two
    // experts; many loads under way
    const int pairs = (a.E + 1) / 2, slices = kThreads / pairs, pair = threadIdx.x % pairs, slice = threadIdx.x / pairs;
    const int g0 = blockIdx.x * a.wgs_per_sort;
    if (slice < slices) {
        const uint32_t* c = (const uint32_t*)a.counts + pair;
        uint32_t all[2] = {0, 0}, low[2] = {0, 0};
        for (int g = slice; g < a.wgs; g += 16 * slices) {
            uint32_t v[16];
#pragma unroll
            for (int i = 0; i < 16; i++) v[i] = c[(int64_t)min(g + i * slices, a.wgs - 1) * pairs];
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int at = g + i * slices;
                const uint32_t x = at < a.wgs ? v[i] & 0xFFFFu : 0, y = at < a.wgs ? v[i] >> 16 : 0;
                all[0] += x;
                all[1] += y;
                low[0] += at < g0 ? x : 0;
                low[1] += at < g0 ? y : 0;
            }
        }
        atomicAdd(&base[2 * pair], all[0]);
        atomicAdd(&before[2 * pair], low[0]);
        if (2 * pair + 1 < a.E) {
            atomicAdd(&base[2 * pair + 1], all[1]);
            atomicAdd(&before[2 * pair + 1], low[1]);
        }
    }
    __syncthreads();
    if (threadIdx.x < 64) scan_wave(base, a.E, threadIdx.x);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i <= a.E; i += kThreads) a.offsets[i] = (int32_t)base[i];
    __syncthreads();
    for (int i = threadIdx.x; i < a.E; i += kThreads) base[i] += before[i];
    __syncthreads();
    const int64_t t0 = (int64_t)g0 * a.tokens_per_wg, t1 = min((int64_t)a.T, t0 + (int64_t)a.wgs_per_sort * a.tokens_per_wg);
    place_entries(a, t0 * a.topk, (int)(t1 - t0) * a.topk, base, wave_at);
}

__global__ void route_nothing_kernel(int32_t* offsets, int n)
{
    for (int i = threadIdx.x; i < n; i += blockDim.x) offsets[i] = 0;
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Lanes of a token (a power of two, at least QUICK_MAX_TOPK).
int lanes_of(int64_t E) { return E <= 16 ? 16 : E <= 32 ? 32 : 64; }

// Experts of a lane.
int places_of(int64_t E) { return E <= 256 ? ceil_div(E, 64) : E <= 384 ? 6 : 8; }

// Workgroups, and the tokens each takes: 16 waves' worth at least.
void route_plan(int64_t T, int64_t E, int* per, int* wgs)
{
    const int64_t least = kWaves * 64 / lanes_of(E);
    const int64_t p = std::min<int64_t>(kMaxTokens, std::max(least, (int64_t)ceil_div(T, kWgs)));
    *per = (int)p;
    *wgs = ceil_div(T, p);
}

template <int DT>
void launch_route(const RouteArgs& a, int wgs, size_t lds, hipStream_t hs)
{
    const dim3 grid(wgs), block(kThreads);
#define QUICK_ROUTE(W, V) route_kernel<DT, W, V><<<grid, block, lds, hs>>>(a)
    if (a.E <= 16) QUICK_ROUTE(16, 1);
    else if (a.E <= 32) QUICK_ROUTE(32, 1);
    else if (a.E <= 64) QUICK_ROUTE(64, 1);
    else if (a.E <= 128) QUICK_ROUTE(64, 2);
    else if (a.E <= 192) QUICK_ROUTE(64, 3);
    else if (a.E <= 256) QUICK_ROUTE(64, 4);
    else if (a.E <= 384) QUICK_ROUTE(64, 6);
    else QUICK_ROUTE(64, 8);
#undef QUICK_ROUTE
}

// ---------------------------------------------------------------------------
// combine
// ---------------------------------------------------------------------------

constexpr int kCombineThreads = 256;

struct CombineArgs {
    const uint16_t* y;
    const uint16_t* residual;
    uint16_t* out;
    const int32_t* slots;
    const float* weights;
    int64_t R, D;
    int32_t topk;
    uint32_t parts;    // workgroups of one token
};

// A thread owns eight columns (or one, VEC = 1) of a token and adds its topk
// rows up in binary32; all of its loads (at most 8 rows at a time) are in
// flight together.  Bound by the bytes: every row of y is read once, so past
// the caches (8192 tokens, 8 rows of 4096: 104 us, 5.8 TB/s, the rate of a
// copy; 120 us through them).
template <int DT, int VEC, int KB>
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(CombineArgs a)
{
    const int64_t t = blockIdx.x / a.parts;
    const int64_t c = ((int64_t)(blockIdx.x % a.parts) * kCombineThreads + threadIdx.x) * VEC;
    if (c >= a.D) return;
    float sum[VEC];
    auto add = [&](const u4_t& raw, float w) {
#pragma unroll
        for (int i = 0; i < VEC; i++)
            sum[i] += w * from16<DT>((uint16_t)(raw[i / 2] >> (16 * (i % 2))));
    };
    auto load = [&](const uint16_t* p) {
        u4_t raw = {0, 0, 0, 0};
        if constexpr (VEC == 8) raw = __builtin_nontemporal_load((const u4_t*)p);
        else raw[0] = *p;
        return raw;
    };
#pragma unroll
    for (int i = 0; i < VEC; i++) sum[i] = 0;
    u4_t res = {0, 0, 0, 0};
    if (a.residual) res = load(a.residual + t * a.D + c);
    for (int j0 = 0; j0 < a.topk; j0 += KB) {
        u4_t raw[KB];
        float w[KB];
#pragma unroll
        for (int j = 0; j < KB; j++) {
            const int at = min(j0 + j, a.topk - 1);
            const int64_t slot = a.slots[t * a.topk + at];
            const bool use = j0 + j < a.topk && slot >= 0 && slot < a.R;
            w[j] = a.weights[t * a.topk + at];
            raw[j] = u4_t{0, 0, 0, 0};
            if (use) raw[j] = load(a.y + slot * a.D + c);
            else w[j] = 0;
        }
#pragma unroll
        for (int j = 0; j < KB; j++) add(raw[j], w[j]);
    }
    if (a.residual) add(res, 1.0f);
    uint16_t* o = a.out + t * a.D + c;
    if constexpr (VEC == 8)
        *(u4_t*)o = u4_t{to16x2<DT>(sum[0], sum[1]), to16x2<DT>(sum[2], sum[3]), to16x2<DT>(sum[4], sum[5]),
                         to16x2<DT>(sum[6], sum[7])};
    else
        *o = to16<DT>(sum[0]);
}

template <int DT, int VEC>
void launch_combine(const CombineArgs& a, uint32_t grid, hipStream_t hs)
{
    if (a.topk == 1) combine_kernel<DT, VEC, 1><<<grid, kCombineThreads, 0, hs>>>(a);
    else if (a.topk == 2) combine_kernel<DT, VEC, 2><<<grid, kCombineThreads, 0, hs>>>(a);
    else if (a.topk <= 4) combine_kernel<DT, VEC, 4><<<grid, kCombineThreads, 0, hs>>>(a);
    else combine_kernel<DT, VEC, 8><<<grid, kCombineThreads, 0, hs>>>(a);
}

}  // namespace

extern "C" size_t quick_moe_route_workspace_bytes(int64_t T, int64_t E, int64_t topk)
{
    if (T <= 0 || E < 1 || E > kMaxE || topk < 1 || topk > QUICK_MAX_TOPK || T * topk >= ((int64_t)1 << 31)) return 0;
    int per, wgs;
    route_plan(T, E, &per, &wgs);
    return wgs > 1 ? (size_t)wgs * ((E + 1) & ~1) * sizeof(uint16_t) : 0;
}

extern "C" int quick_moe_route(const void* logits, int dtype, int64_t T, int64_t E, const quick_route_t* route,
                               const float* bias, int32_t* ids, float* weights, int32_t* offsets, int32_t* rows, int32_t* slots,
                               void* workspace, size_t workspace_bytes, void* stream)
{
    if (!route || dtype < QUICK_F16 || dtype > QUICK_F32) return QUICK_ERR_INVALID_ARG;
    const quick_route_t& r = *route;
    if (r.score != QUICK_SCORE_SOFTMAX && r.score != QUICK_SCORE_SIGMOID) return QUICK_ERR_INVALID_ARG;
    if (r.group_best < 1 || r.group_best > 2) return QUICK_ERR_INVALID_ARG;
    if (T < 0 || E < 1 || E > kMaxE || r.topk < 1 || r.topk > QUICK_MAX_TOPK || T > ((int64_t)1 << 30) ||
        T * r.topk >= ((int64_t)1 << 31))
        return QUICK_ERR_SHAPE;
    if (r.groups < 1 || r.groups > QUICK_MAX_GROUPS || E % r.groups != 0 || r.topk_groups < 1 ||
        r.topk_groups > r.groups || r.topk > r.topk_groups * (E / r.groups))
        return QUICK_ERR_SHAPE;
    if (!offsets) return QUICK_ERR_INVALID_ARG;
    if (T && (!logits || !ids || !weights || !rows || !slots)) return QUICK_ERR_INVALID_ARG;
    if (!aligned(logits, dtype == QUICK_F32 ? 4 : 2) || !aligned(bias, 4) || !aligned(ids, 4) ||
        !aligned(weights, 4) || !aligned(offsets, 4) || !aligned(rows, 4) || !aligned(slots, 4))
        return QUICK_ERR_ALIGNMENT;
    hipStream_t hs = (hipStream_t)stream;
    (void)hipGetLastError();
    if (T == 0) {
        route_nothing_kernel<<<1, 256, 0, hs>>>(offsets, (int)E + 1);
        return launched();
    }
    const size_t need = quick_moe_route_workspace_bytes(T, E, r.topk);
    if (need && (!workspace || workspace_bytes < need)) return QUICK_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return QUICK_ERR_ALIGNMENT;
    RouteArgs a;
    a.logits = logits;
    a.bias = bias;
    a.ids = ids;
    a.weights = weights;
    a.offsets = offsets;
    a.rows = rows;
    a.slots = slots;
    a.counts = need ? (uint16_t*)workspace : nullptr;
    a.T = (int32_t)T;
    a.E = (int32_t)E;
    a.topk = r.topk;
    a.groups = r.groups;
    a.topk_groups = r.topk_groups;
    a.group_best = r.group_best;
    a.group_size = (int32_t)(E / r.groups);
    a.group_inv = ((1u << 20) + a.group_size - 1) / a.group_size;
    const int lanes = lanes_of(E), places = places_of(E);
    const int whole = lanes == 64 && a.group_size % places == 0 ? a.group_size / places : 0;
    a.group_lanes = whole <= 32 && (whole & (whole - 1)) == 0 ? whole : 0;
    a.sigmoid = r.score == QUICK_SCORE_SIGMOID;
    a.renorm = r.renormalize != 0;
    a.by_score = a.sigmoid || bias || (r.groups > 1 && r.group_best > 1);
    a.scale = r.scale;
    route_plan(T, E, &a.tokens_per_wg, &a.wgs);
    const size_t head = (kMaxE + 4) * sizeof(int);
    const size_t sorted = kWaves * E * sizeof(int);
    const size_t grouped =
        r.groups > 1 ? kWaves * 64 / lanes_of(E) * group_ints((int)E, r.groups) * sizeof(int) : 0;
    const size_t lds = head + std::max(sorted, grouped);
    if (dtype == QUICK_F16) launch_route<QUICK_F16>(a, a.wgs, lds, hs);
    else if (dtype == QUICK_BF16) launch_route<QUICK_BF16>(a, a.wgs, lds, hs);
    else launch_route<QUICK_F32>(a, a.wgs, lds, hs);
    int st = launched();
    if (st || a.wgs == 1) return st;
    a.wgs_per_sort = std::max(1, kSortEntries / (a.tokens_per_wg * a.topk));
    route_sort_kernel<<<ceil_div(a.wgs, a.wgs_per_sort), kThreads, head + kMaxE * sizeof(int) + sorted, hs>>>(a);
    return launched();
}

extern "C" int quick_moe_combine(const void* y, int dtype, int64_t R, int64_t D, const int32_t* slots,
                                 const float* weights, int64_t T, int64_t topk, const void* residual, void* out,
                                 void* stream)
{
    if (dtype != QUICK_F16 && dtype != QUICK_BF16) return QUICK_ERR_INVALID_ARG;
    if (T < 0 || R < 0 || D < 1 || D >= ((int64_t)1 << 31) || topk < 1 || topk > QUICK_MAX_TOPK ||
        T >= ((int64_t)1 << 31) || R >= ((int64_t)1 << 31))
        return QUICK_ERR_SHAPE;
    if (T == 0) return QUICK_OK;
    if (!slots || !weights || !out || (R && !y)) return QUICK_ERR_INVALID_ARG;
    if (!aligned(y, 2) || !aligned(residual, 2) || !aligned(out, 2) || !aligned(slots, 4) || !aligned(weights, 4))
        return QUICK_ERR_ALIGNMENT;
    const bool wide = D % 8 == 0 && aligned(y, 16) && aligned(residual, 16) && aligned(out, 16);
    CombineArgs a{(const uint16_t*)y, (const uint16_t*)residual, (uint16_t*)out, slots, weights, R, D, (int32_t)topk, 0};
    a.parts = (uint32_t)ceil_div(D, kCombineThreads * (wide ? 8 : 1));
    if (T * a.parts >= ((int64_t)1 << 24)) return QUICK_ERR_SHAPE;
    const uint32_t grid = (uint32_t)(T * a.parts);
    hipStream_t hs = (hipStream_t)stream;
    (void)hipGetLastError();
    if (dtype == QUICK_F16) {
        if (wide) launch_combine<QUICK_F16, 8>(a, grid, hs);
        else launch_combine<QUICK_F16, 1>(a, grid, hs);
    } else {
        if (wide) launch_combine<QUICK_BF16, 8>(a, grid, hs);
        else launch_combine<QUICK_BF16, 1>(a, grid, hs);
    }
    return launched();
}
