// Products with weights in microscaled 4-bit floating point on the scaled
// matrix instructions of gfx950, 16x16x128 (few rows) and 32x32x64.
//
// y[m][n] = sum over blocks b of 2^(xs[m][b] + ws[n][b] - 254) *
//           sum over the 32 channels of b of x[m][k] * w[n][k]
//
// The former takes, per lane, 32 consecutive channels of one row (16
// bytes of codes, four registers) and that block's scale byte, for both
// operands: lane l holds row l % 16 and block l / 16 of the step's four.  So a
// 16-byte load of a row of codes is an operand as it stands, and so is a
// lane's share of a packed weight unit, which one wave-wide load fetches from
// 1 KiB of consecutive memory.  Nothing is converted or moved on the way.
// The weights are the A operand (result rows), so that a lane ends with four
// consecutive columns of one row of y.
#include <algorithm>
#include <type_traits>

#include "quick_mx.h"
#include "quick_mx_forms.h"
#include "quick_mx_quant.h"
#include "quick_mx_scales.h"

namespace {

using namespace quick;

typedef int i8_t __attribute__((ext_vector_type(8)));

// The cache policy of a load of data that nothing reads again: non-temporal.
constexpr int kOnce = 2;

struct MxArgs {
    const uint8_t* codes;      // [T][K/2]
    const uint8_t* scales;     // [T][K/32]
    const uint8_t* packed;
    const uint8_t* pscales;
    uint16_t* y;
    const uint16_t* bias;      // [E][N] in logical order, or null
    const int32_t* rows;       // [R] row of x of each routed row, or null
    const int32_t* offsets;    // [E + 1] (grouped form)
    int32_t M, N, K;           // M: rows of y
    int32_t T, E;              // rows of x, experts (grouped form)
    int32_t gated, bf16;
    int32_t wide;              // y is on 16 bytes
    int32_t lead;              // 1: each column tile has a workgroup more, that writes nothing
};

__device__ __forceinline__ f4_t mx_mfma(u4_t a, u4_t b, f4_t c, uint32_t sa, uint32_t sb)
{
    const i8_t aa = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i8_t bb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(aa, bb, c, 4, 4, 0, (int)sa, 0, (int)sb);
}

__device__ __forceinline__ float bias_at(const MxArgs& a, const uint16_t* bias, int n)
{
    return a.bf16 ? from16<QUICK_BF16>(bias[n]) : from16<QUICK_F16>(bias[n]);
}

__device__ __forceinline__ float silu(float v) { return v / (1.0f + __expf(-v)); }

// Four consecutive columns n.. of row m (cols: columns of y); columns past the
// end are left out, and rows whose start is not on 8 bytes go value by value.
__device__ __forceinline__ void store4(const MxArgs& a, int64_t m, int n, int cols, f4_t v)
{
    uint16_t* p = a.y + m * cols + n;
    const u2_t h = a.bf16 ? u2_t{to16x2<QUICK_BF16>(v[0], v[1]), to16x2<QUICK_BF16>(v[2], v[3])}
                          : u2_t{to16x2<QUICK_F16>(v[0], v[1]), to16x2<QUICK_F16>(v[2], v[3])};
    if (cols % 4 == 0) {
        if (n < cols) *(u2_t*)p = h;
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (n + i < cols) p[i] = (uint16_t)(h[i / 2] >> (16 * (i % 2)));
    }
}

// A tile's place: rows m0 .. m1 - 1 of y, and the expert.
struct Tile {
    int m0, m1, e;
};

// The grouped form's tiles of BM rows, each of one expert, in the order of the
// experts: a lane counts those of eight experts.  Offsets that are not in
// order are taken as the largest so far, and within 0..M.
template <int BM>
struct GroupedTiles {
    static constexpr int PER = QUICK_MAX_EXPERTS / 64;
    int at[PER + 1], tiles, upto, all;

    __device__ __forceinline__ GroupedTiles(const MxArgs& a)
    {
        const int lane = threadIdx.x & 63;
        int top = 0;
#pragma unroll
        for (int i = 0; i <= PER; i++) {
            at[i] = min(max(a.offsets[min(lane * PER + i, a.E)], 0), a.M);
            if (i < PER) top = max(top, at[i]);
        }
        // running maximum over all earlier experts
        int run = top;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(run, d);
            if (lane >= d) run = max(run, o);
        }
        int low = __shfl_up(run, 1);
        if (lane == 0) low = 0;
        tiles = 0;
#pragma unroll
        for (int i = 0; i <= PER; i++) low = at[i] = max(at[i], low);
#pragma unroll
        for (int i = 0; i < PER; i++) tiles += (at[i + 1] - at[i] + BM - 1) / BM;
        upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        all = __builtin_amdgcn_readlane(upto, 63);
    }

    // Tile number t < all.
    __device__ __forceinline__ Tile find(int t) const
    {
        const int lane = threadIdx.x & 63;
        const int who = __builtin_ctzll(__ballot(upto > t));
        int n = t - (upto - tiles);
        Tile r = {0, 0, 0};
        bool found = false;
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int here = (at[i + 1] - at[i] + BM - 1) / BM;
            if (!found && n < here) {
                r.e = lane * PER + i;
                r.m0 = at[i] + n * BM;
                r.m1 = min(r.m0 + BM, at[i + 1]);
                found = true;
            }
            n -= found ? 0 : here;
        }
        r.e = __builtin_amdgcn_readlane(r.e, who);
        r.m0 = __builtin_amdgcn_readlane(r.m0, who);
        r.m1 = __builtin_amdgcn_readlane(r.m1, who);
        return r;
    }
};

// Wait until at most V vector-memory operations of this wave are outstanding.
template <int V>
__device__ __forceinline__ void wait_vm()
{
    __builtin_amdgcn_s_waitcnt(0x0F70 | (V & 15) | ((V >> 4) << 14));
}
// Wait until this wave's LDS accesses are done.
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }
// Workgroup barrier that orders nothing by itself (the waits before it do);
// the compiler moves no memory access across it.
__device__ __forceinline__ void barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Few rows: 16 rows, WK waves that share out the K steps (128 channels) of NT
// column tiles.  A workgroup takes `groups` runs of NT column tiles one after
// the other.  Operands go from memory straight into registers, D steps ahead,
// also across the end of a run; at the end of one the waves' sums are added up
// through LDS in the order of the waves, by waves that take turns.  Bound by
// the weights' bytes and the start of a launch (7B q, k, v, 26 MB, one row: 8.2
// us with the quantisation; a copy kernel reads 26 MB in 6.8).
// TAIL: K is not a multiple of 128; the blocks past its end are read as zero.
// ONCE: the weights come past the caches.
// XQ >= 0: activations x of that 16-bit type, at most kFusedRows rows; the
// workgroup quantises them into LDS while its first weights are under way.
template <int NT, int WK, int D, bool GRP, bool TAIL, bool ONCE, int XQ>
__global__ __launch_bounds__(64 * WK) void mx_stream_kernel(MxArgs a, int groups)
{
    constexpr int BM = 16;
    __shared__ f4_t part[2][WK][NT][64];
    extern __shared__ __attribute__((aligned(16))) uint8_t xq[];    // XQ: [M][K/2] codes, [M][K/32] scales
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, row = lane & 15, blk = lane >> 4;
    Tile t;
    if constexpr (GRP) {
        const GroupedTiles<BM> tiles(a);
        if ((int)blockIdx.y >= tiles.all) return;
        t = tiles.find(blockIdx.y);
    } else {
        t.m0 = blockIdx.y * BM;
        t.m1 = min(t.m0 + BM, a.M);
        t.e = 0;
    }
    const int KS = (a.K + 127) / 128, KQ = (KS + 3) / 4, KB = a.K / 32, NTT = (a.N + 15) / 16;
    const int g0 = blockIdx.x * groups, g1 = min(g0 + groups, (NTT + NT - 1) / NT);
    const uint8_t* pw = uniform(a.packed + (int64_t)t.e * NTT * KS * 1024);
    const uint8_t* ps = uniform(a.pscales + (int64_t)t.e * NTT * KQ * 256);
    const uint32_t xbytes = (uint32_t)((int64_t)a.T * (a.K / 2)), xsbytes = (uint32_t)((int64_t)a.T * KB);
    int r = min(t.m0 + row, t.m1 - 1);
    if (GRP && a.rows) r = min(max(a.rows[r], 0), a.T - 1);
    const uint32_t xo = (uint32_t)r * (uint32_t)(a.K / 2) + blk * 16;
    const uint32_t so = (uint32_t)r * (uint32_t)KB + (TAIL ? blk : 0);
    const int per = (KS + WK - 1) / WK, s0 = wave * per;
    f4_t acc[NT];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NT; j++) acc[j] = f4_t{0, 0, 0, 0};
    };
    u4_t w[D][NT], x[D];
    uint32_t ws[D][NT], xs[D];
    int lg = g0, ls = 0;    // run and step that are loaded next
    auto load = [&](int d) __attribute__((always_inline)) {
        // past the last run or step: empty buffers, which read as zero
        const int s = s0 + ls, tiles = min(NT, NTT - lg * NT);
        const bool in = s < KS && lg < g1;
        const rsrc_t rw = make_rsrc(pw + (int64_t)lg * NT * KS * 1024, in ? (uint32_t)tiles * KS * 1024 : 0);
        const rsrc_t rp = make_rsrc(ps + (int64_t)lg * NT * KQ * 256, in ? (uint32_t)tiles * KQ * 256 : 0);
#pragma unroll
        for (int j = 0; j < NT; j++) {
            w[d][j] = bits_as<u4_t>(__builtin_amdgcn_raw_buffer_load_b128(rw, (uint32_t)(j * KS) * 1024 + lane * 16, s * 1024,
                                                                          ONCE ? kOnce : 0));
            ws[d][j] = ld32(rp, (uint32_t)(j * KQ) * 256 + lane * 4, (s >> 2) * 256);
        }
        if constexpr (XQ < 0) {
            const rsrc_t rx = make_rsrc(a.codes, in ? xbytes : 0), rs = make_rsrc(a.scales, in ? xsbytes : 0);
            const bool block = !TAIL || s * 4 + blk < KB;
            x[d] = ld128(rx, block ? xo : 0xFFFFFFF0u, s * 64);
            if constexpr (TAIL) xs[d] = ld8(rs, block ? so : 0xFFFFFFF0u, s * 4);
            else xs[d] = ld32(rs, so, s * 4);
        }
        if (++ls == per) {
            ls = 0;
            lg++;
        }
    };
    const uint16_t* bias = a.bias ? a.bias + (int64_t)t.e * a.N : nullptr;
    // The sums of run g, by wave (its number here) mod WK.  Two buffers: a
    // wave that adds up one run is past it when the run after the next is
    // written, since all meet in between.
    auto flush = [&](int g) __attribute__((always_inline)) {
        f4_t(*to)[NT][64] = part[(g - g0) & 1];
#pragma unroll
        for (int j = 0; j < NT; j++) to[wave][j][lane] = acc[j];
        wait_lds();
        barrier();
        clear();
        if ((g - g0) % WK != wave) return;
        f4_t v[NT];
#pragma unroll
        for (int j = 0; j < NT; j++) {
            v[j] = f4_t{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < WK; k++) v[j] += to[k][j][lane];
        }
        const int m = t.m0 + row;
        if (m >= t.m1) return;
        if (!a.gated) {
#pragma unroll
            for (int j = 0; j < NT; j++) {
                const int n = (g * NT + j) * 16 + blk * 4;
                if (bias)
#pragma unroll
                    for (int c = 0; c < 4; c++) v[j][c] += n + c < a.N ? bias_at(a, bias, n + c) : 0.0f;
                store4(a, m, n, a.N, v[j]);
            }
        } else if constexpr (NT % 2 == 0) {
#pragma unroll
            for (int j = 0; j < NT; j += 2) {
                const int n = (g * NT + j) * 8 + blk * 4;    // column of y
                f4_t h;
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    float gate = v[j][c], up = v[j + 1][c];
                    if (bias && n < a.N / 2) {
                        gate += bias_at(a, bias, n + c);
                        up += bias_at(a, bias, a.N / 2 + n + c);
                    }
                    h[c] = silu(gate) * up;
                }
                store4(a, m, n, a.N / 2, h);
            }
        }
    };
    clear();
#pragma unroll
    for (int d = 0; d < D; d++) load(d);
    if constexpr (XQ >= 0) {
        // a piece of eight values a thread; four threads have a block
        const int pieces = a.M * (a.K / 8);
        for (int p0 = 0; p0 < pieces; p0 += 64 * WK) {
            const int p = p0 + threadIdx.x;
            const u4_t raw[1] = {((const u4_t*)a.codes)[min(p, pieces - 4 + (int)(threadIdx.x & 3))]};
            float v[8];
            unpack8<XQ>(raw, v);
            const uint32_t scale = block_scale(max_of_quad(amax8(v)));
            const uint32_t c = block_codes(v, scale);
            if (p < pieces) {
                *(uint32_t*)(xq + p * 4) = c;
                if ((p & 3) == 0) xq[a.M * (a.K / 2) + p / 4] = (uint8_t)scale;
            }
        }
        wait_lds();
        barrier();
    }
    int g = g0, s = 0;    // run and step that are multiplied next
    const int total = (g1 - g0) * per;
    for (int f = 0; f < total; f += D) {
#pragma unroll
        for (int d = 0; d < D; d++) {
            if (f + d < total) {
                uint32_t sx;
                if constexpr (XQ >= 0) {
                    const int at = (s0 + s) * 4 + blk, xr = min(row, a.M - 1);
                    const bool in = at < KB;
                    const u4_t v = *(const u4_t*)(xq + xr * (a.K / 2) + (in ? at : 0) * 16);
                    const uint32_t b = xq[a.M * (a.K / 2) + xr * KB + (in ? at : 0)];
                    x[d] = in ? v : u4_t{0, 0, 0, 0};
                    sx = in ? b : 0;
                } else {
                    sx = TAIL ? xs[d] : xs[d] >> (8 * blk);
                }
                const uint32_t sh = (uint32_t)((s0 + s) & 3) * 8;
#pragma unroll
                for (int j = 0; j < NT; j++) acc[j] = mx_mfma(w[d][j], x[d], acc[j], ws[d][j] >> sh, sx);
                load(d);
                if (++s == per) {
                    flush(g);
                    s = 0;
                    g++;
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// tiled kernel: more rows than fit one or two operands
// ---------------------------------------------------------------------------

typedef float f16_t __attribute__((ext_vector_type(16)));

template <int OA, int OB>
__device__ __forceinline__ f16_t mx_mfma32(u4_t a, u4_t b, f16_t c, uint32_t sa, uint32_t sb)
{
    const i8_t aa = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i8_t bb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(aa, bb, c, 4, 4, OA, (int)sa, OB, (int)sb);
}

// 16 bytes per lane from a buffer straight into LDS: lane l writes bytes
// 16 l .. 16 l + 15 after the wave-uniform address dst.
template <int AUX>
__device__ __forceinline__ void dma16(rsrc_t r, void* dst, uint32_t voff, uint32_t soff)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)dst, 16, voff, soff, 0, AUX);
}

// The stages of a tiled kernel in LDS.
struct Ring {
    uint8_t *st0, *st1, *st2, *st3, *st4, *st5, *st6, *st7;
};

// A BM x BN tile of y by WM x WN waves of MB x NB blocks of 32 x 32, on the
// 32x32x64 instruction (twice the flops of the 16x16x128 one per operand byte
// and issue slot).  Codes of both operands go from memory straight into LDS,
// a ring of NS stages of 128 channels (one object each, so that reads of one
// are not taken to depend on the copies under way into another):
//  * activations: 16 rows of 64 bytes a copy.  The 16-byte piece c of row r
//    lies at place c ^ (r / 4 % 4) of the row, which spreads the reads of a
//    block (32 rows, one or two pieces) over all banks;
//  * weights: one packed unit a copy, as it lies in memory.
// The scales of four steps are copied together, into NS / 4 buffers.  Operands
// are read from LDS a step, or half a one, before they are multiplied.
// What bounds it: the largest tiles the clock, 1.7 GHz under their power, and at
// that clock the waits: the matrix instructions are busy 59 % of the cycles, a
// wave waits for a barrier or for a count 30 % of its time (2048 rows of 70B
// gate+up 464 us, 4.1 PFLOP/s; a loop of nothing but the instruction on random
// operands reaches 6.4, at 1.5 GHz); the smaller ones the latency of memory, a
// few stages of a tile's own columns being all that is under way (333 rows of
// 13B down 24 us, 2.0 PFLOP/s).
// ONCE: the weights come past the caches.
// TAIL: K is not a multiple of 128.
template <int BM, int BN, int WM, int WN, int NS, bool GRP, bool TAIL, bool ONCE>
__device__ __forceinline__ void tiled_product(const MxArgs& a, Tile t, int nt, Ring ring, bool leads)
{
    constexpr int W = WM * WN, MB = BM / WM / 32, NB = BN / WN / 32;
    constexpr int XC = BM / 16, IM = (XC + W - 1) / W, IN = BN / 16 / W, NI = IM + IN;    // copies a wave and step
    constexpr int STAGE = (BM + BN) * 64, XS = BM < 64 ? 64 : BM;
    static_assert(IN * W * 16 == BN && (NS == 4 || NS == 8), "weight copies are shared out evenly");
    // Operands go to registers a whole step before they are multiplied, but in
    // the largest tile, whose accumulators leave room for half a step.
    constexpr bool AHEAD = BM * BN < 65536;
    uint8_t* const sc0 = ring.st0 + STAGE;
    uint8_t* const sc1 = ring.st4 + (NS == 8 ? STAGE : 0);
    auto scale_buffer = [&](auto which) __attribute__((always_inline)) -> uint8_t* {
        if constexpr (decltype(which)::value % (NS / 4) == 0) return sc0;
        else return sc1;
    };
    auto stage = [&](auto which) __attribute__((always_inline)) -> uint8_t* {
        constexpr int S = decltype(which)::value % NS;
        if constexpr (S == 0) return ring.st0;
        else if constexpr (S == 1) return ring.st1;
        else if constexpr (S == 2) return ring.st2;
        else if constexpr (S == 3) return ring.st3;
        else if constexpr (S == 4) return ring.st4;
        else if constexpr (S == 5) return ring.st5;
        else if constexpr (S == 6) return ring.st6;
        else return ring.st7;
    };
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = wave % WM, wn = wave / WM, col = lane & 31, half = lane >> 5;

    const int KS = (a.K + 127) / 128, KQ = (KS + 3) / 4, KB = a.K / 32, NTT = (a.N + 15) / 16;
    const int64_t first = (int64_t)t.e * NTT + nt * (BN / 16);
    const int tiles = min(BN / 16, NTT - nt * (BN / 16));
    const uint8_t* pw = uniform(a.packed + first * KS * 1024);
    const uint8_t* ps = uniform(a.pscales + first * KQ * 256);
    const uint32_t xbytes = (uint32_t)((int64_t)a.T * (a.K / 2)), wbytes = uniform((uint32_t)tiles * KS * 1024);
    const uint32_t xsbytes = (uint32_t)((int64_t)a.T * KB), wsbytes = (uint32_t)tiles * KQ * 256;

    // this wave's copies: rows of activations, units of weights.  Rows past
    // the tile's end repeat its last one; steps past the last one, and units
    // past the last tile, are read from an empty buffer: as zero
    uint32_t xo[IM], wo[IN];
    const int piece = (lane & 3) ^ (lane >> 4 & 3);
    auto source = [&](int r) __attribute__((always_inline)) {
        r = min(t.m0 + r, t.m1 - 1);
        if (GRP && a.rows) r = min(max(a.rows[r], 0), a.T - 1);
        return (uint32_t)r;
    };
#pragma unroll
    for (int i = 0; i < IM; i++)
        xo[i] = source(min(i * W + wave, XC - 1) * 16 + (lane >> 2)) * (uint32_t)(a.K / 2) + piece * 16;
#pragma unroll
    for (int i = 0; i < IN; i++) wo[i] = (uint32_t)(i * W + wave) * KS * 1024 + lane * 16;
    auto copy_step = [&](uint8_t* st, int s) __attribute__((always_inline)) {
        const rsrc_t rx = make_rsrc(a.codes, s < KS ? xbytes : 0), rw = make_rsrc(pw, s < KS ? wbytes : 0);
#pragma unroll
        for (int i = 0; i < IM; i++)
            dma16<0>(rx, st + min(i * W + wave, XC - 1) * 1024, !TAIL || s * 4 + piece < KB ? xo[i] : 0xFFFFFFF0u, s * 64);
#pragma unroll
        for (int i = 0; i < IN; i++) dma16<ONCE ? kOnce : 0>(rw, st + BM * 64 + (i * W + wave) * 1024, wo[i], s * 1024);
    };
    // scales of four steps: a copy of 64 rows' 16 bytes each, and of four
    // weight tiles'; the last waves may repeat a copy
    constexpr int CM = XS / 64, CN = BN / 64, CI = (CM + CN + W - 1) / W;
    uint32_t so[CI], sbytes[CI];
    const uint8_t* sbase[CI];
#pragma unroll
    for (int i = 0; i < CI; i++) {
        const int c = min(i * W + wave, CM + CN - 1);
        const bool rows = c < CM;
        so[i] = rows ? row_scales(source(c * 64 + lane), KB) : tile_scales((c - CM) * 4 + (lane >> 4), KQ, lane);
        sbase[i] = uniform(rows ? a.scales : ps);
        sbytes[i] = uniform(rows ? xsbytes : wsbytes);
    }
    auto copy_scales = [&](uint8_t* sc, int q) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CI; i++) {
            const int c = min(i * W + wave, CM + CN - 1);
            const BufferPlace p = scale_copy(so[i], c < CM, q);
            if (!TAIL || c >= CM) dma16<0>(make_rsrc(sbase[i], q < KQ ? sbytes[i] : 0), sc + c * 1024, p.lane, p.uniform);
        }
    };
    // TAIL: a row's scales start anywhere, and past its end is the next row's:
    // a thread each row, byte by byte, zero past the end
    uint32_t raw[TAIL ? 16 : 1];
    const uint32_t my_row = TAIL ? source(min((int)threadIdx.x, BM - 1)) * (uint32_t)KB : 0;
    auto load_tail = [&](int q) __attribute__((always_inline)) {
        if constexpr (TAIL) {
            const rsrc_t rs = make_rsrc(a.scales, xsbytes);
#pragma unroll
            for (int b = 0; b < 16; b++) raw[b] = ld8(rs, q * 16 + b < KB ? my_row + q * 16 + b : 0xFFFFFFF0u, 0);
        }
    };
    auto write_tail = [&](uint8_t* sc) __attribute__((always_inline)) {
        if constexpr (TAIL) {
            u4_t v;
#pragma unroll
            for (int d = 0; d < 4; d++)
                v[d] = raw[4 * d] | raw[4 * d + 1] << 8 | raw[4 * d + 2] << 16 | raw[4 * d + 3] << 24;
            if (threadIdx.x < BM) *(u4_t*)(sc + threadIdx.x * 16) = v;
        }
    };

    f16_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int c = 0; c < 16; c++) acc[i][j][c] = 0;

    // a block's operand: row or column col; pieces half (channels 0..63 of a
    // step) and 2 + half
    const int xr = (wm * MB * 32 + col) * 64 + (half ^ (col >> 2 & 3)) * 16;
    const int wr = BM * 64 + (wn * NB * 2 + (col >> 4)) * 1024 + half * 256 + (col & 15) * 16;
    const int xsr = (wm * MB * 32 + col) * 16;
    const int wsr = XS * 16 + (wn * NB * 2 + (col >> 4)) * 256 + (half * 16 + (col & 15)) * 4;
    // the second word's address is kept apart: of two reads made one the
    // compiler no longer knows the object, and waits for all copies under way
    int wsr2 = wsr + 128;
    asm volatile("" : "+v"(wsr2));
    u4_t x[AHEAD ? 4 : 2][MB], w[AHEAD ? 4 : 2][NB], xs[MB];
    uint32_t ws[NB][2];
    // half step h of a step: AHEAD keeps two steps, the odd ones in 2 and 3
    auto read = [&](const uint8_t* st, auto step, auto which) __attribute__((always_inline)) {
        constexpr int h = decltype(which)::value, p = AHEAD ? decltype(step)::value % 2 * 2 + h : h;
#pragma unroll
        for (int j = 0; j < NB; j++) w[p][j] = *(const u4_t*)(st + wr + j * 2048 + h * 512);
#pragma unroll
        for (int i = 0; i < MB; i++) x[p][i] = *(const u4_t*)(st + (xr ^ (h * 32)) + i * 2048);
    };
    // scales of steps 4 q ..: a row's byte of block 2 h + half of step j is
    // byte 2 h of word j here; zero for steps past the last one, which lie in
    // the next row's scales
    auto read_scales = [&](const uint8_t* sc, int q, u4_t (&to)[MB], uint32_t (&tw)[NB][2])
                           __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MB; i++) {
            const u4_t v = *(const u4_t*)(sc + xsr + i * 512);
#pragma unroll
            for (int c = 0; c < 4; c++) to[i][c] = q * 4 + c < KS ? v[c] >> (8 * half) : 0;
        }
#pragma unroll
        for (int j = 0; j < NB; j++) {
            tw[j][0] = *(const uint32_t*)(sc + wsr + j * 512);
            tw[j][1] = *(const uint32_t*)(sc + wsr2 + j * 512);
        }
    };
    auto multiply = [&](auto step, auto which) __attribute__((always_inline)) {
        constexpr int S = decltype(step)::value, h = decltype(which)::value, p = AHEAD ? S % 2 * 2 + h : h;
#pragma unroll
        for (int i = 0; i < MB; i++)
#pragma unroll
            for (int j = 0; j < NB; j++)
                acc[i][j] = mx_mfma32<S, 2 * h>(w[p][j], x[p][i], acc[i][j], ws[j][h], xs[i][S]);
    };

    constexpr std::integral_constant<int, 0> I0;
    constexpr std::integral_constant<int, 1> I1;
    load_tail(0);
    write_tail(sc0);
    copy_scales(sc0, 0);
    if constexpr (NS == 8) {
        load_tail(1);
        write_tail(sc1);
        copy_scales(sc1, 1);
    }
    auto first_copies = [&]<int... I>(std::integer_sequence<int, I...>) __attribute__((always_inline)) {
        ((copy_step(stage(std::integral_constant<int, I>{}), I), __builtin_amdgcn_sched_barrier(0)), ...);
    };
    first_copies(std::make_integer_sequence<int, AHEAD ? NS : NS - 1>{});
    wait_vm<(AHEAD ? NS - 1 : NS - 2) * NI>();
    wait_lds();
    barrier();
    read_scales(sc0, 0, xs, ws);
    read(ring.st0, I0, I0);
    if constexpr (AHEAD) read(ring.st0, I0, I1);
    // Order of a half step: one matrix instruction, then some of the LDS reads
    // and copies that are issued under it.
    auto interleave = [&](auto reads, auto copies) __attribute__((always_inline)) {
        constexpr int N = MB * NB, R = (decltype(reads)::value + N - 1) / N, C = decltype(copies)::value;
        constexpr int EACH = C > 0 ? (N + (C > 0 ? C : 1) - 1) / (C > 0 ? C : 1) : 1, AT = C > 0 ? (C + N - 1) / N : 0;
#pragma unroll
        for (int i = 0; i < N; i++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
            if constexpr (C > 0)
                if (i % EACH == 0) __builtin_amdgcn_sched_group_barrier(0x020, AT, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Step s.  After the barrier: the copies of step s + 1 have arrived (those
    // of later ones may be under way), and every wave has read all of step
    // s - 1 (AHEAD: s), whose stage is filled next.
    auto turn = [&](int s, auto unrolled) __attribute__((always_inline)) {
        constexpr int U = decltype(unrolled)::value, S = U % 4;
        constexpr int FREED = AHEAD ? 0 : 1;      // the step after which scales are in registers
        wait_vm<(AHEAD ? NS - 2 : NS - 3) * NI>();
        wait_lds();
        barrier();
        __builtin_amdgcn_sched_barrier(0);
        uint8_t* sc = scale_buffer(std::integral_constant<int, U / 4>{});
        if constexpr (S == FREED) {
            // the scales of this step's four are in registers
            load_tail(s / 4 + NS / 4);
            copy_scales(sc, s / 4 + NS / 4);
        }
        if constexpr (S == 2) write_tail(sc);
        constexpr std::integral_constant<int, U + 1> NEXT;
        constexpr std::integral_constant<int, NI + (S == FREED ? CI : 0)> COPIES;
        u4_t nx[MB];
        uint32_t nw[NB][2];
        auto next_scales = [&]() __attribute__((always_inline)) {
            read_scales(scale_buffer(std::integral_constant<int, U / 4 + 1>{}), s / 4 + 1, nx, nw);
        };
        constexpr int SR = S == 3 ? MB + 2 * NB : 0;
        if constexpr (AHEAD) {
            copy_step(stage(unrolled), s + NS);
            if constexpr (S == 3) next_scales();
            read(stage(NEXT), NEXT, I0);
            multiply(std::integral_constant<int, S>{}, I0);
            interleave(std::integral_constant<int, MB + NB + SR>{}, COPIES);
            read(stage(NEXT), NEXT, I1);
            multiply(std::integral_constant<int, S>{}, I1);
            interleave(std::integral_constant<int, MB + NB>{}, I0);
        } else {
            copy_step(stage(std::integral_constant<int, U + NS - 1>{}), s + NS - 1);
            read(stage(unrolled), unrolled, I1);
            multiply(std::integral_constant<int, S>{}, I0);
            interleave(std::integral_constant<int, MB + NB>{}, COPIES);
            if constexpr (S == 3) next_scales();
            read(stage(NEXT), NEXT, I0);
            multiply(std::integral_constant<int, S>{}, I1);
            interleave(std::integral_constant<int, MB + NB + SR>{}, I0);
        }
        if constexpr (S == 3) {
#pragma unroll
            for (int i = 0; i < MB; i++) xs[i] = nx[i];
#pragma unroll
            for (int j = 0; j < NB; j++)
#pragma unroll
                for (int h = 0; h < 2; h++) ws[j][h] = nw[j][h];
        }
    };
    auto four = [&](int s, auto at) __attribute__((always_inline)) {
        constexpr int U = decltype(at)::value;
        turn(s, std::integral_constant<int, U>{});
        turn(s + 1, std::integral_constant<int, U + 1>{});
        turn(s + 2, std::integral_constant<int, U + 2>{});
        turn(s + 3, std::integral_constant<int, U + 3>{});
    };
    if constexpr (NS == 4) {
        for (int s = 0; s < KS; s += 4) four(s, I0);
    } else {
        // (with a way out in the middle of the loop the compiler no longer
        // tells the stages apart, and waits for copies under way)
        int s = 0;
        for (; s + 4 < KS; s += 8) {
            four(s, I0);
            four(s + 4, std::integral_constant<int, 4>{});
        }
        if (s < KS) four(s, I0);
    }
    wait_vm<0>();
    wait_lds();
    __syncthreads();

    if (leads) return;

    // Rows of y of a wave's blocks go through LDS (a region of its own), from
    // where a lane takes 16 consecutive bytes.  Lane: row col of a block;
    // accumulator 4 b + c is column 8 b + 4 half + c.
    uint8_t* mine = wave < (W + 1) / 2 ? ring.st0 + wave * (NB * 2048) : ring.st1 + (wave - (W + 1) / 2) * (NB * 2048);
    static_assert((W + 1) / 2 * NB * 2048 <= STAGE, "the waves' regions fit two stages");
    const uint16_t* bias = a.bias ? a.bias + (int64_t)t.e * a.N : nullptr;
    const int n0 = nt * BN + wn * NB * 32;
    auto finish = [&](auto type, auto gating) __attribute__((always_inline)) {
        constexpr int DT = decltype(type)::value;
        constexpr bool G = decltype(gating)::value;
        constexpr int OB = G ? 2 : 4, PIECES = NB * OB;    // eight-column runs of a block, 16-byte pieces of a row
        const int cols = G ? a.N / 2 : a.N, c0 = G ? n0 / 2 : n0;
        const bool wide = cols % 8 == 0 && a.wide;
#pragma unroll
        for (int i = 0; i < MB; i++) {
#pragma unroll
            for (int j = 0; j < NB; j++)
#pragma unroll
                for (int b = 0; b < OB; b++) {
                    const int n = c0 + (j * OB + b) * 8 + half * 4;
                    f4_t v = {acc[i][j][4 * b], acc[i][j][4 * b + 1], acc[i][j][4 * b + 2], acc[i][j][4 * b + 3]};
                    f4_t up;
                    if constexpr (G)
#pragma unroll
                        for (int c = 0; c < 4; c++) up[c] = acc[i][j][4 * (b + 2) + c];
                    if (bias) {
#pragma unroll
                        for (int c = 0; c < 4; c++) {
                            const int at = min(n + c, cols - 1);
                            v[c] += from16<DT>(bias[at]);
                            if constexpr (G) up[c] += from16<DT>(bias[cols + at]);
                        }
                    }
                    if constexpr (G)
#pragma unroll
                        for (int c = 0; c < 4; c++) v[c] = silu(v[c]) * up[c];
                    const u2_t h = {to16x2<DT>(v[0], v[1]), to16x2<DT>(v[2], v[3])};
                    *(u2_t*)(mine + col * (PIECES * 16) + ((j * OB + b) ^ (col % PIECES)) * 16 + half * 8) = h;
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int r0 = (wm * MB + i) * 32;
#pragma unroll
            for (int k = 0; k < PIECES / 2; k++) {
                const int r = k * (64 / PIECES) + lane / PIECES, p = lane % PIECES;
                const u4_t v = *(const u4_t*)(mine + r * (PIECES * 16) + (p ^ (r % PIECES)) * 16);
                const int m = t.m0 + r0 + r, n = c0 + p * 8;
                if (m >= t.m1 || n >= cols) continue;
                uint16_t* o = a.y + (int64_t)m * cols + n;
                if (wide) {
                    *(u4_t*)o = v;
                } else {
                    // rows that do not start on 16 bytes
#pragma unroll
                    for (int c = 0; c < 8; c++)
                        if (n + c < cols) o[c] = (uint16_t)(v[c / 2] >> (16 * (c % 2)));
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    };
    constexpr std::integral_constant<int, QUICK_F16> F16;
    constexpr std::integral_constant<int, QUICK_BF16> BF16;
    if (a.gated) {
        if (a.bf16) finish(BF16, std::true_type{});
        else finish(F16, std::true_type{});
    } else {
        if (a.bf16) finish(BF16, std::false_type{});
        else finish(F16, std::false_type{});
    }
}

template <int BM, int BN, int WM, int WN, int NS, bool GRP, bool TAIL, bool ONCE>
__global__ __launch_bounds__(64 * WM * WN, NS == 8 ? 1 : 2) void mx_tiled_kernel(MxArgs a, int row_tiles)
{
    constexpr int STAGE = (BM + BN) * 64, SC = ((BM < 64 ? 64 : BM) + BN) * 16, S8 = NS == 8 ? STAGE : 16;
    // No more than eight objects, the number that the compiler tells apart in
    // its waits: the scales lie behind the stages that are filled and read at
    // the same turns
    __shared__ __attribute__((aligned(16))) uint8_t st0[STAGE + SC], st1[STAGE], st2[STAGE], st3[STAGE],
        st4[NS == 8 ? STAGE + SC : 16], st5[S8], st6[S8], st7[S8];
    const Ring ring = {st0, st1, st2, st3, st4, st5, st6, st7};

    // Workgroups go to the eight dies in turn: each die gets a run of tiles.
    // A run goes over bands of eight row tiles, in a band over the column
    // tiles, row tiles first: what is under way on a die at a time is near
    // square, and shares its operands in the die's L2.
    const int col_tiles = (a.N + BN - 1) / BN;
    auto place = [&](int rows, int* mt, int* nt) {
        const int per = (rows * col_tiles + 7) / 8, idx = blockIdx.x % 8 * per + blockIdx.x / 8;
        if ((int)blockIdx.x / 8 >= per || idx >= rows * col_tiles) return false;
        const int band = idx / (8 * col_tiles), in = idx - band * 8 * col_tiles, high = min(8, rows - 8 * band);
        *nt = in / high;
        *mt = band * 8 + in % high;
        return true;
    };
    // A leading workgroup goes through its column's steps as the others do, on
    // the last row alone, a little ahead of them.
    bool leads = false;
    int mt, nt;
    Tile t;
    if constexpr (GRP) {
        const GroupedTiles<BM> tiles(a);
        if (!place(tiles.all, &mt, &nt)) return;
        t = tiles.find(mt);
    } else {
        if (!place(row_tiles + a.lead, &mt, &nt)) return;
        mt -= a.lead;
        leads = mt < 0;
        t.m0 = leads ? a.M - 1 : mt * BM;
        t.m1 = min(t.m0 + BM, a.M);
        t.e = 0;
    }
    // A tile that is half empty or more, as an expert's last one often is, is
    // multiplied as a lower one (4096 rows over 8 experts of 28672 x 4096:
    // 358 us, 377 without)
    if constexpr (BM >= 128) {
        const int rows = uniform(t.m1 - t.m0);
        if constexpr (BM >= 256) {
            if (rows <= BM / 4) return tiled_product<BM / 4, BN, WM, WN, NS, GRP, TAIL, ONCE>(a, t, nt, ring, leads);
        }
        if (rows <= BM / 2) return tiled_product<BM / 2, BN, WM, WN, NS, GRP, TAIL, ONCE>(a, t, nt, ring, leads);
    }
    tiled_product<BM, BN, WM, WN, NS, GRP, TAIL, ONCE>(a, t, nt, ring, leads);
}

// f(std::true_type) or f(std::false_type).
template <class F>
void with_bool(bool b, F f)
{
    if (b) f(std::true_type{});
    else f(std::false_type{});
}

// About 1536 workgroups (six for each compute unit), fewer where there are not
// so many column tiles; each takes as many runs as that leaves.
template <int NT, bool GRP>
int launch_stream(const MxArgs& a, const MxPlan& p, int xq, hipStream_t hs)
{
    constexpr int WK = 8, D = NT == 4 ? 2 : 4;
    const int64_t rows = p.row_tiles, runs = p.columns;
    if (rows > 65535) return QUICK_ERR_SHAPE;
    if (a.gated && NT % 2 != 0) return QUICK_ERR_UNSUPPORTED;
    int st = QUICK_OK;
    const int groups = (int)ceil_div(runs, std::max<int64_t>(1, 1536 / rows));
    const dim3 grid((uint32_t)ceil_div(runs, groups), (uint32_t)rows), block(64 * WK);
    with_bool(p.tail, [&](auto tail) {
        with_bool(p.once, [&](auto once) {
            constexpr bool TAIL = decltype(tail)::value, ONCE = decltype(once)::value;
            if (xq < 0) {
                mx_stream_kernel<NT, WK, D, GRP, TAIL, ONCE, -1><<<grid, block, 0, hs>>>(a, groups);
            } else if constexpr (!GRP && NT <= 2) {
                const size_t lds = (size_t)a.M * (a.K / 2 + a.K / 32);
                if (xq == QUICK_F16)
                    mx_stream_kernel<NT, WK, D, false, TAIL, ONCE, QUICK_F16><<<grid, block, lds, hs>>>(a, groups);
                else
                    mx_stream_kernel<NT, WK, D, false, TAIL, ONCE, QUICK_BF16><<<grid, block, lds, hs>>>(a, groups);
            } else {
                st = QUICK_ERR_UNSUPPORTED;    // no codes to read
            }
        });
    });
    return st;
}

template <int BM, int BN, int WM, int WN, int NS, bool GRP>
int launch_tiled(MxArgs a, const MxPlan& p, hipStream_t hs)
{
    a.lead = p.lead;
    const int64_t grid = ceil_div((p.row_tiles + p.lead) * p.columns, 8) * 8;
    if (grid > (1 << 22)) return QUICK_ERR_SHAPE;
    const dim3 g((uint32_t)grid), block(64 * WM * WN);
    int st = QUICK_OK;
    with_bool(p.tail, [&](auto tail) {
        with_bool(p.once, [&](auto once) {
            constexpr bool TAIL = decltype(tail)::value, ONCE = decltype(once)::value;
            // no tail in the largest form, weights past the caches in the lower
            // ones alone (form_takes, plan_product)
            if constexpr ((TAIL && BM * BN >= 65536) || (ONCE && BM > 64))
                st = QUICK_ERR_UNSUPPORTED;
            else
                mx_tiled_kernel<BM, BN, WM, WN, NS, GRP, TAIL, ONCE><<<g, block, 0, hs>>>(a, (int)p.row_tiles);
        });
    });
    return st;
}

// xq >= 0: the activations are 16-bit values of that type, and few.
template <bool GRP>
int launch_mx(const MxArgs& a, int xq, hipStream_t hs)
{
    const MxPlan p = plan_product({a.M, a.N, a.K, a.E, GRP, a.gated != 0, xq >= 0});
    (void)hipGetLastError();
    int st = QUICK_ERR_UNSUPPORTED;
    switch (p.form) {
    case 0: st = launch_stream<1, GRP>(a, p, xq, hs); break;
    case 1: st = launch_stream<2, GRP>(a, p, xq, hs); break;
    case 2: st = launch_stream<4, GRP>(a, p, xq, hs); break;
    case 3: st = launch_tiled<32, 128, 1, 4, 4, GRP>(a, p, hs); break;
    case 4: st = launch_tiled<64, 64, 2, 2, 8, GRP>(a, p, hs); break;
    case 5: st = launch_tiled<64, 128, 1, 4, 8, GRP>(a, p, hs); break;
    case 6: st = launch_tiled<64, 128, 1, 4, 4, GRP>(a, p, hs); break;
    case 7: st = launch_tiled<128, 128, 2, 2, 4, GRP>(a, p, hs); break;
    case 8: st = launch_tiled<128, 256, 2, 4, 4, GRP>(a, p, hs); break;
    case 9: st = launch_tiled<256, 256, 2, 4, 4, GRP>(a, p, hs); break;
    }
    return st ? st : launched();
}

int check_product(int64_t rows, int64_t M, int64_t N, int64_t K, int dtype, int activation)
{
    if (dtype != QUICK_F16 && dtype != QUICK_BF16) return QUICK_ERR_INVALID_ARG;
    if (activation != QUICK_ACT_NONE && activation != QUICK_ACT_SILU_GATE) return QUICK_ERR_INVALID_ARG;
    if (rows < 0 || M < 0 || M > (1 << 22) || rows > (1 << 24) || K > (1 << 22) ||
        (K > 0 && rows * K >= ((int64_t)1 << 33)))
        return QUICK_ERR_SHAPE;
    int st = quick_mxfp4_packed_sizes(N, K, nullptr, nullptr);
    if (st) return st;
    return activation == QUICK_ACT_SILU_GATE && N % 32 != 0 ? QUICK_ERR_SHAPE : QUICK_OK;
}

int check_pointers(const void* codes, const void* scales, const void* packed, const void* pscales, const void* y,
                   const void* bias)
{
    if (!codes || !scales || !packed || !pscales || !y) return QUICK_ERR_INVALID_ARG;
    if (!aligned(codes, 16) || !aligned(scales, 4) || !aligned(packed, 16) || !aligned(pscales, 4) || !aligned(y, 8) ||
        !aligned(bias, 2))
        return QUICK_ERR_ALIGNMENT;
    return QUICK_OK;
}

MxArgs make_args(const void* codes, const void* scales, const void* packed, const void* pscales, void* y, int dtype,
                 int64_t M, int64_t N, int64_t K, const void* bias, int activation)
{
    MxArgs a;
    a.codes = (const uint8_t*)codes;
    a.scales = (const uint8_t*)scales;
    a.packed = (const uint8_t*)packed;
    a.pscales = (const uint8_t*)pscales;
    a.y = (uint16_t*)y;
    a.bias = (const uint16_t*)bias;
    a.rows = a.offsets = nullptr;
    a.M = a.T = (int32_t)M;
    a.N = (int32_t)N;
    a.K = (int32_t)K;
    a.E = 1;
    a.gated = activation == QUICK_ACT_SILU_GATE;
    a.bf16 = dtype == QUICK_BF16;
    a.wide = aligned(y, 16);
    a.lead = 0;
    return a;
}

// Bytes of the codes of M rows in a workspace, the scales after them.
size_t code_bytes(int64_t M, int64_t K) { return (size_t)ceil_div(M * (K / 2), 256) * 256; }

}  // namespace

extern "C" int quick_mxfp4_gemm(const void* codes, const void* scales, const void* packed, const void* packed_scales,
                                void* y, int dtype, int64_t M, int64_t N, int64_t K, const void* bias, int activation,
                                void* stream)
{
    int st = check_product(M, M, N, K, dtype, activation);
    if (st || M == 0) return st;
    st = check_pointers(codes, scales, packed, packed_scales, y, bias);
    if (st) return st;
    return launch_mx<false>(make_args(codes, scales, packed, packed_scales, y, dtype, M, N, K, bias, activation), -1,
                            (hipStream_t)stream);
}

extern "C" size_t quick_mxfp4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    if (M <= 0 || fused_quantisation(M, K) || check_product(M, M, N, K, QUICK_F16, QUICK_ACT_NONE)) return 0;
    return code_bytes(M, K) + (size_t)(M * (K / 32));
}

extern "C" int quick_mxfp4_linear(const void* x, const void* packed, const void* packed_scales, void* y, int dtype,
                                  int64_t M, int64_t N, int64_t K, const void* bias, int activation, void* workspace,
                                  size_t workspace_bytes, void* stream)
{
    int st = check_product(M, M, N, K, dtype, activation);
    if (st || M == 0) return st;
    const size_t need = quick_mxfp4_linear_workspace_bytes(M, N, K);
    if (!x) return QUICK_ERR_INVALID_ARG;
    if (!aligned(x, 16)) return QUICK_ERR_ALIGNMENT;
    if (need && (!workspace || workspace_bytes < need)) return QUICK_ERR_WORKSPACE;
    if (!need) {
        st = check_pointers(x, packed_scales, packed, packed_scales, y, bias);
        if (st) return st;
        // no codes in memory: the launch reads x in their place
        return launch_mx<false>(make_args(x, nullptr, packed, packed_scales, y, dtype, M, N, K, bias, activation), dtype,
                                (hipStream_t)stream);
    }
    uint8_t* codes = (uint8_t*)workspace;
    uint8_t* scales = codes + code_bytes(M, K);
    st = check_pointers(codes, scales, packed, packed_scales, y, bias);
    if (st) return st;
    st = quick_mxfp4_quantize(x, dtype, K, M, K, codes, scales, stream);
    if (st) return st;
    return launch_mx<false>(make_args(codes, scales, packed, packed_scales, y, dtype, M, N, K, bias, activation), -1,
                            (hipStream_t)stream);
}

extern "C" int quick_mxfp4_grouped_gemm(const void* codes, const void* scales, const int32_t* rows,
                                        const int32_t* offsets, const void* packed, const void* packed_scales, void* y,
                                        int dtype, int64_t T, int64_t R, int64_t E, int64_t N, int64_t K,
                                        const void* bias, int activation, void* stream)
{
    int st = check_product(T, R, N, K, dtype, activation);
    if (st) return st;
    if (E < 1 || E > QUICK_MAX_EXPERTS) return QUICK_ERR_SHAPE;
    if (R == 0) return QUICK_OK;
    if (T == 0 || (!rows && T < R)) return QUICK_ERR_SHAPE;
    if (!offsets) return QUICK_ERR_INVALID_ARG;
    st = check_pointers(codes, scales, packed, packed_scales, y, bias);
    if (st) return st;
    if (!aligned(offsets, 4) || !aligned(rows, 4)) return QUICK_ERR_ALIGNMENT;
    MxArgs a = make_args(codes, scales, packed, packed_scales, y, dtype, R, N, K, bias, activation);
    a.T = (int32_t)T;
    a.E = (int32_t)E;
    a.rows = rows;
    a.offsets = offsets;
    return launch_mx<true>(a, -1, (hipStream_t)stream);
}
