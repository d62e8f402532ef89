// Low-rank adapters of many requests: the tokens' order by adapter, and
// y + s (x A^T) B^T over it.
#include <algorithm>

#include "quick_device.h"
#include "quick_lora.h"

namespace {

using namespace quick;

typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));

constexpr int kMaxE = QUICK_MAX_EXPERTS;
constexpr int kThreads = 256;       // of the second product
constexpr int kDownThreads = 512;   // of the first

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------------------
// order
// ---------------------------------------------------------------------------

constexpr int kGroupWaves = 16;

// One workgroup: every wave counts a run of the tokens, the counts are summed
// by adapter, then by wave, and each wave places its run; tokens of one wave's
// 64 that share an adapter by their lanes' order.  The last of the E + 1 classes
// is that of no adapter.
__global__ __launch_bounds__(64 * kGroupWaves) void lora_group_kernel(const int32_t* ids, int T, int E, int32_t* offsets,
                                                                      int32_t* rows)
{
    extern __shared__ uint32_t lds[];
    uint32_t* count = lds;               // [waves][E + 1]
    uint32_t* total = lds + kGroupWaves * (E + 1);   // [E + 2]
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, C = E + 1;
    const int per = (int)(((int64_t)T + kGroupWaves * 64 - 1) / (kGroupWaves * 64)) * 64;
    const int lo = min(T, wave * per), hi = min(T, lo + per);
    auto of = [&](int i) {
        const int e = ids[i];
        return e >= 0 && e < E ? e : E;
    };
    for (int i = threadIdx.x; i < kGroupWaves * C; i += 64 * kGroupWaves) count[i] = 0;
    __syncthreads();
    uint32_t* mine = count + wave * C;
    for (int i = lo + lane; i < hi; i += 64) atomicAdd(&mine[of(i)], 1u);
    __syncthreads();
    for (int e = threadIdx.x; e < C; e += 64 * kGroupWaves) {
        uint32_t sum = 0;
        for (int w = 0; w < kGroupWaves; w++) {
            const uint32_t n = count[w * C + e];
            count[w * C + e] = sum;
            sum += n;
        }
        total[e] = sum;
    }
    __syncthreads();
    if (wave == 0) {
        uint32_t before = 0;
        for (int e0 = 0; e0 < C; e0 += 64) {
            const uint32_t n = e0 + lane < C ? total[e0 + lane] : 0;
            uint32_t run = n;
            for (int d = 1; d < 64; d *= 2) {
                const uint32_t o = (uint32_t)__shfl_up((int)run, d);
                if (lane >= d) run += o;
            }
            if (e0 + lane < C) {
                total[e0 + lane] = before + run - n;
                offsets[e0 + lane] = (int32_t)(before + run - n);
            }
            before += (uint32_t)__shfl((int)run, 63);
        }
    }
    __syncthreads();
    int bits = 0;
    while ((1 << bits) < C) bits++;
    for (int i0 = lo; i0 < hi; i0 += 64) {
        const int i = i0 + lane;
        const bool live = i < hi;
        const int e = live ? of(i) : 0;
        uint64_t same = __ballot(live);
        for (int b = 0; b < bits; b++) {
            const uint64_t m = __ballot(e >> b & 1);
            same &= (e >> b & 1) ? m : ~m;
        }
        if (live) {
            const int rank = __popcll(same & ((1ull << lane) - 1));
            rows[total[e] + mine[e] + rank] = i;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (rank == 0) mine[e] += __popcll(same);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------

struct LoraArgs {
    const uint8_t *x, *a, *b, *y;
    uint8_t* out;
    const float* scales;
    const int32_t *offsets, *rows;
    float* low;           // [slices][R][rank] x . A^T over a slice of the channels
    int64_t ldx, ldy, ldo;
    int32_t T, K, N, E, rank, R, slices, slice;   // slice: channels of one
    int32_t parts;        // workgroups of a tile in the second product
};

template <int DT>
__device__ __forceinline__ f4_t mfma16(u4_t a, u4_t b, f4_t c)
{
    if constexpr (DT == QUICK_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(bits_as<h8_t>(a), bits_as<h8_t>(b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(bits_as<b8_t>(a), bits_as<b8_t>(b), c, 0, 0, 0);
}

// Tile of rows of one adapter: rows first .. first + count - 1 of the order.
struct RowTile {
    int e, first, count;    // e == E: rows without an adapter; count == 0: no tile
};

__device__ __forceinline__ int clamped(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Rows of class e of the order: of adapter e, or (e == E) those without one.
__device__ __forceinline__ int rows_of(const LoraArgs& a, int e, int& first)
{
    first = clamped(a.offsets[e], 0, a.R);
    return (e < a.E ? clamped(a.offsets[e + 1], first, a.R) : a.R) - first;
}

// Inclusive sums over the lanes of a wave.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_from(int v)
{
    return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, true);
}
__device__ __forceinline__ int sums_upto(int v)
{
    v = add_from<0x111, 0xF>(v);
    v = add_from<0x112, 0xF>(v);
    v = add_from<0x114, 0xF>(v);
    v = add_from<0x118, 0xF>(v);
    v = add_from<0x142, 0xA>(v);
    return add_from<0x143, 0xC>(v);
}

// The index'th tile of H rows of all.  Every wave works it out by itself, its
// lanes adding up the tiles of the classes.
template <int H>
__device__ __forceinline__ RowTile find_tile(const LoraArgs& a, int index)
{
    const int lane = threadIdx.x & 63, per = (a.E + 64) / 64;    // classes of a lane
    int sum = 0, first;
    for (int e = lane * per; e < min((lane + 1) * per, a.E + 1); e++) sum += (rows_of(a, e, first) + H - 1) / H;
    const int upto = sums_upto(sum);
    RowTile t{0, 0, 0};
    const uint64_t m = __ballot(upto > index);
    if (!m) return t;
    const int from = __builtin_ctzll(m);
    if (lane == from) {
        int at = upto - sum;
        for (int e = lane * per; e < min((lane + 1) * per, a.E + 1); e++) {
            const int n = rows_of(a, e, first), tiles = (n + H - 1) / H;
            if (index < at + tiles) {
                t = RowTile{e, first + (index - at) * H, min(H, n - (index - at) * H)};
                break;
            }
            at += tiles;
        }
    }
    return {__builtin_amdgcn_readlane(t.e, from), __builtin_amdgcn_readlane(t.first, from),
            __builtin_amdgcn_readlane(t.count, from)};
}

// low = x . A^T of a tile of 16 TM RW rows and a slice of the channels.  Of eight
// waves RW share the rows out, 16 TM each, and the others the channels, each
// taking 128 (64 of many rows) at a time; the rows of A (16 RT of them) are the instruction's
// rows, those of x its columns, both straight from memory, 16 bytes a lane; the
// waves' sums meet in LDS.
// A tile is a chain of latencies: offsets, rows, operands, LDS (4096 tokens of
// 5120 channels, rank 64: 19 us, 7 by its bytes).
template <int DT, int RT, int TM, int RW>
__global__ __launch_bounds__(kDownThreads) void lora_down_kernel(LoraArgs a)
{
    constexpr int KW = kDownThreads / 64 / RW, ROWS = 16 * TM * RW;
    constexpr int STEPS = TM > 1 ? 2 : 4, TAKE = 32 * STEPS;    // of 32 channels whose operands are loaded together
    __shared__ float sums[KW][ROWS][16 * RT + 4];
    const RowTile t = find_tile<ROWS>(a, blockIdx.x);
    if (t.count == 0 || t.e == a.E) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const int row0 = wave % RW * 16 * TM, part = wave / RW;
    const int k0 = blockIdx.y * a.slice, k1 = min(a.K, k0 + a.slice);
    // (lanes without a row, or behind the rank, read another one, and their sums go nowhere)
    const uint8_t* x[TM];
#pragma unroll
    for (int m = 0; m < TM; m++) {
        const int row = a.rows[t.first + min(row0 + m * 16 + c, t.count - 1)];
        x[m] = a.x + 2 * ((int64_t)(row >= 0 && row < a.T ? row : 0) * a.ldx + g * 8);
    }
    const uint8_t* w[RT];
#pragma unroll
    for (int r = 0; r < RT; r++)
        w[r] = a.a + 2 * (((int64_t)t.e * a.rank + min(r * 16 + c, a.rank - 1)) * a.K + g * 8);
    f4_t acc[TM][RT];
#pragma unroll
    for (int m = 0; m < TM; m++)
#pragma unroll
        for (int r = 0; r < RT; r++) acc[m][r] = f4_t{0, 0, 0, 0};
    if (row0 < t.count) {
        for (int k = k0 + part * TAKE; k < k1; k += KW * TAKE) {
            u4_t xv[STEPS][TM], wv[STEPS][RT];
            if (k + TAKE <= k1) {
#pragma unroll
                for (int s = 0; s < STEPS; s++) {
#pragma unroll
                    for (int m = 0; m < TM; m++) xv[s][m] = *(const u4_t*)(x[m] + 2 * (k + s * 32));
#pragma unroll
                    for (int r = 0; r < RT; r++) wv[s][r] = *(const u4_t*)(w[r] + 2 * (k + s * 32));
                }
            } else {
                // the last channels: eights behind the end are zero in both
#pragma unroll
                for (int s = 0; s < STEPS; s++) {
                    const bool in = k + s * 32 + g * 8 < k1;
                    const int64_t at = in ? k + s * 32 : k0 - g * 8;
#pragma unroll
                    for (int m = 0; m < TM; m++) {
                        const u4_t v = *(const u4_t*)(x[m] + 2 * at);
                        xv[s][m] = in ? v : u4_t{0, 0, 0, 0};
                    }
#pragma unroll
                    for (int r = 0; r < RT; r++) {
                        const u4_t v = *(const u4_t*)(w[r] + 2 * at);
                        wv[s][r] = in ? v : u4_t{0, 0, 0, 0};
                    }
                }
            }
#pragma unroll
            for (int s = 0; s < STEPS; s++)
#pragma unroll
                for (int m = 0; m < TM; m++)
#pragma unroll
                    for (int r = 0; r < RT; r++) acc[m][r] = mfma16<DT>(wv[s][r], xv[s][m], acc[m][r]);
        }
#pragma unroll
        for (int m = 0; m < TM; m++)
#pragma unroll
            for (int r = 0; r < RT; r++) *(f4_t*)&sums[part][row0 + m * 16 + c][r * 16 + g * 4] = acc[m][r];
    }
    __syncthreads();
    // four columns a thread (the rank is a multiple of eight)
    for (int i = threadIdx.x; i < ROWS * 4 * RT; i += kDownThreads) {
        const int row = i / (4 * RT), r = i % (4 * RT) * 4;
        if (row >= t.count || r >= a.rank) continue;
        f4_t v = *(const f4_t*)&sums[0][row][r];
#pragma unroll
        for (int n = 1; n < KW; n++) v += *(const f4_t*)&sums[n][row][r];
        *(f4_t*)(a.low + ((int64_t)blockIdx.y * a.R + t.first + row) * a.rank + r) = v;
    }
}

// Swaps b of the lanes c < 8 of each 16 with a of the lanes c + 8.
__device__ __forceinline__ void swap_eights(u4_t& a, u4_t& b, bool low)
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t x = low ? b[i] : a[i];
        const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, false);    // (row_ror:8)
        a[i] = low ? a[i] : y;
        b[i] = low ? y : b[i];
    }
}

// out = y + low . B^T of a tile of 16 TM rows, 64 columns a wave at a time.  The
// rows of B are the instruction's rows, in an order that leaves a lane twice 8
// consecutive columns of its token, and four lanes 64 bytes: row 4 g + i of tile
// j is column 32 (j / 2) + 8 g + 4 (j % 2) + i.  The sums of low over the slices,
// scaled and rounded, are the other operand and stay in registers for all columns.  With a rank of 8 or 16 a lane group's
// 16 bytes of B are of another tile (or of two), and both operands are zero but
// for that group's lanes, so that every load is full.
// A lane's loads and stores of y, and its loads of B, are of the two halves of
// eight rows' 128 bytes, put in the product's order by an exchange of lanes
// eight apart: two loads of 64 bytes of a line wait for each other (4096 tokens,
// 15360 columns of rank 64: 99.6 us with the first product, 90.4 so).
// Bound by the bytes of y and out for many rows: there 64 us, 3.9 TB/s, of 44 at
// the rate of a copy; the rest is B, 126 MB through L2, and the start of a tile.
template <int DT, int RS, int TM>
__global__ __launch_bounds__(kThreads, RS == 4 && TM == 4 ? 1 : 2) void lora_up_kernel(LoraArgs a)
{
    constexpr int STEPS = RS ? RS : 1;      // of 32 ranks (RS == 0: rank 8 or 16)
    const RowTile t = find_tile<16 * TM>(a, blockIdx.x / a.parts);
    if (t.count == 0) return;
    const bool bare = t.e == a.E;
    if (bare && a.out == a.y) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    // (what is behind the rows, the columns or the rank is read from another place and goes nowhere)
    const bool front = c < 8;
    int row[TM][2];
#pragma unroll
    for (int m = 0; m < TM; m++)
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const int at = m * 16 + 8 * k + (c & 7), x = a.rows[t.first + min(at, t.count - 1)];
            row[m][k] = at < t.count && x >= 0 && x < a.T ? x : -1;
        }
    // with a low rank every lane group holds the same of it (8 g % rank)
    const int per = RS ? 1 : 32 / a.rank, mine = RS ? 0 : g * 8 / a.rank;
    u4_t low[STEPS][TM];
    if (!bare) {
        // the sums over the slices once a workgroup
        __shared__ u4_t lows[16 * TM][4 * STEPS + 1];
        const float scale = a.scales ? a.scales[t.e] : 1.0f;
        const int pieces = a.rank / 8;
        for (int i = threadIdx.x; i < 16 * TM * pieces; i += kThreads) {
            const int x = i / pieces, r = i - x * pieces;
            const float* from = a.low + ((int64_t)t.first + min(x, t.count - 1)) * a.rank + r * 8;
            f4_t u{0, 0, 0, 0}, v{0, 0, 0, 0};
#pragma unroll 4
            for (int n = 0; n < a.slices; n++) {
                u += *(const f4_t*)(from + (int64_t)n * a.R * a.rank);
                v += *(const f4_t*)(from + (int64_t)n * a.R * a.rank + 4);
            }
            u *= scale;
            v *= scale;
            lows[x][r] = u4_t{to16x2<DT>(u[0], u[1]), to16x2<DT>(u[2], u[3]), to16x2<DT>(v[0], v[1]), to16x2<DT>(v[2], v[3])};
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < STEPS; s++)
#pragma unroll
            for (int m = 0; m < TM; m++) {
                low[s][m] = lows[m * 16 + c][RS ? s * 4 + g : g % pieces];
                if (RS && s * 32 + g * 8 >= a.rank) low[s][m] = u4_t{0, 0, 0, 0};
            }
    }
    const uint8_t* b = a.b + 2 * (int64_t)(bare ? 0 : t.e) * a.N * a.rank;
    u4_t w[STEPS][4], y[TM][2];
    auto load_b = [&](int n0) {
        if (bare) return;
#pragma unroll
        for (int s = 0; s < STEPS; s++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                // with a low rank load j is that of tiles per * j .. per * j + per - 1
                if (per * j >= 4) continue;
                const int tile = RS ? j : per * j + mine, r = RS ? s * 32 + g * 8 : g * 8 % a.rank;
                if constexpr (RS > 1) {
                    // (of a pair of steps in the order of y's lines)
                    const int x = s % 2 * 8 + (c & 7), n = min(n0 + (tile >> 1) * 32 + (x >> 2) * 8 + (tile & 1) * 4 + (x & 3), a.N - 1);
                    w[s][j] = *(const u4_t*)(b + 2 * ((int64_t)n * a.rank + min(s / 2 * 64 + (c >> 3) * 32 + g * 8, a.rank - 8)));
                } else {
                    const int n = min(n0 + (tile >> 1) * 32 + (c >> 2) * 8 + (tile & 1) * 4 + (c & 3), a.N - 1);
                    w[s][j] = *(const u4_t*)(b + 2 * ((int64_t)n * a.rank + min(r, a.rank - 8)));
                    if (RS && s == STEPS - 1 && r >= a.rank) w[s][j] = u4_t{0, 0, 0, 0};
                }
            }
    };
    // a load has 128 bytes of eight rows: of lanes c and c + 8 the two halves of the row (c & 7) or (c & 7) + 8
    const int column = (c >> 3) * 32 + g * 8;
    auto load_y = [&](int n0) {
#pragma unroll
        for (int m = 0; m < TM; m++)
#pragma unroll
            for (int k = 0; k < 2; k++)
                y[m][k] = *(const u4_t*)(a.y + 2 * ((int64_t)max(row[m][k], 0) * a.ldy + min(n0 + column, a.N - 8)));
    };
    const int step = a.parts * 256;
    int n0 = ((int)(blockIdx.x % a.parts) * 4 + wave) * 64;
    load_b(n0);
    load_y(n0);
    for (; n0 < a.N; n0 += step) {
        f4_t acc[TM][4];
#pragma unroll
        for (int m = 0; m < TM; m++)
#pragma unroll
            for (int j = 0; j < 4; j++) acc[m][j] = f4_t{0, 0, 0, 0};
        if (bare) {
        } else if constexpr (RS == 0) {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const bool here = mine == j % per;
                const u4_t v = per == 4 ? w[0][0] : w[0][j / 2];
#pragma unroll
                for (int m = 0; m < TM; m++)
                    acc[m][j] = mfma16<DT>(here ? v : u4_t{0, 0, 0, 0}, here ? low[0][m] : u4_t{0, 0, 0, 0}, acc[m][j]);
            }
        } else {
#pragma unroll
            for (int s = 0; s < STEPS; s++)
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    if (RS > 1 && s % 2 == 0) swap_eights(w[s][j], w[s + 1][j], front);
                    if (RS > 1 && s * 32 + g * 8 >= a.rank) w[s][j] = u4_t{0, 0, 0, 0};
                }
#pragma unroll
            for (int s = 0; s < STEPS; s++)
#pragma unroll
                for (int m = 0; m < TM; m++)
#pragma unroll
                    for (int j = 0; j < 4; j++) acc[m][j] = mfma16<DT>(w[s][j], low[s][m], acc[m][j]);
        }
        // the next columns' operands take the place of these as they are done with
        load_b(n0 + step);
#pragma unroll
        for (int m = 0; m < TM; m++) {
            if (!bare) {
                swap_eights(y[m][0], y[m][1], front);
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const f4_t v = acc[m][h * 2 + i / 2];
                        y[m][h][i] = to16x2<DT>(from16<DT>((uint16_t)y[m][h][i]) + v[i % 2 * 2],
                                                from16<DT>((uint16_t)(y[m][h][i] >> 16)) + v[i % 2 * 2 + 1]);
                    }
                swap_eights(y[m][0], y[m][1], front);
            }
#pragma unroll
            for (int k = 0; k < 2; k++)
                if (row[m][k] >= 0 && n0 + column < a.N)
                    *(u4_t*)(a.out + 2 * ((int64_t)row[m][k] * a.ldo + n0 + column)) = y[m][k];
        }
        load_y(n0 + step);
    }
}

// Rows of a tile: 64 where the adapters have three 16s or more each on average.
int tile_rows(int64_t R, int64_t E) { return R >= 48 * E ? 64 : 16; }

// Most tiles there can be (the rows without an adapter are one more class).
int64_t tiles_of(int64_t R, int64_t E)
{
    const int64_t h = tile_rows(R, E);
    return R / h + std::min(E + 1, R);
}

// Slices of the channels: a workgroup for each compute unit and some more, whole
// rounds of its waves (64 channels each with 64 rows, 128 with 16), and 16 at
// most, as the second product adds them up (512 tokens, 5120 channels: 27.2 us,
// 29.2 with eight).  What it counts are the most tiles there can be, and with 64
// rows LDS holds one workgroup a unit, so that a few more than the units run a
// round of their own: 4096 tokens, 5120 channels to 15360, rank 64, of four
// adapters with 1024 each, 64 tiles of 4 slices, take 83 us, of five with 819, 65
// tiles, 104.
void slices_of(int64_t R, int64_t K, int64_t E, int32_t* slices, int32_t* slice)
{
    const int64_t round = tile_rows(R, E) == 64 ? 512 : 1024, rounds = ceil_div(K, round);
    const int64_t n = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(rounds, 16), 320 / tiles_of(R, E)));
    *slice = (int32_t)(ceil_div(rounds, n) * round);
    *slices = (int32_t)ceil_div(K, *slice);
}

template <int DT, int TM>
void launch_lora(LoraArgs a, hipStream_t hs)
{
    const uint32_t tiles = (uint32_t)tiles_of(a.R, a.E);
    // columns: enough workgroups for the chip, and no more, as each begins with the sums over the slices; those of one
    // eighth follow each other eight apart, on one die, whose cache then holds their part of B (15360 columns of rank
    // 64 of four adapters, 1024 tokens: 31.5 us, 36.8 with the tiles on the dies; 4096: the same within 1 %)
    const int64_t most = ceil_div(a.N, 256), want = ceil_div(ceil_div(512, tiles), 8) * 8;
    a.parts = (int32_t)std::min(most, want);
    const dim3 down(tiles, a.slices), up(tiles * a.parts);
    // (LDS does not hold the sums of 128 ranks of 64 rows by eight waves)
    constexpr int RW = TM > 1 ? 2 : 1;
    if (a.rank <= 16) lora_down_kernel<DT, 1, TM, 1><<<down, kDownThreads, 0, hs>>>(a);
    else if (a.rank <= 32) lora_down_kernel<DT, 2, TM, 1><<<down, kDownThreads, 0, hs>>>(a);
    else if (a.rank <= 64) lora_down_kernel<DT, 4, TM, 1><<<down, kDownThreads, 0, hs>>>(a);
    else lora_down_kernel<DT, 8, TM / RW, RW><<<down, kDownThreads, 0, hs>>>(a);
    if (a.rank == 8 || a.rank == 16) lora_up_kernel<DT, 0, TM><<<up, kThreads, 0, hs>>>(a);
    else if (a.rank <= 32) lora_up_kernel<DT, 1, TM><<<up, kThreads, 0, hs>>>(a);
    else if (a.rank <= 64) lora_up_kernel<DT, 2, TM><<<up, kThreads, 0, hs>>>(a);
    else lora_up_kernel<DT, 4, TM><<<up, kThreads, 0, hs>>>(a);
}

}  // namespace

extern "C" int quick_lora_group(const int32_t* ids, int64_t T, int64_t E, int32_t* offsets, int32_t* rows, void* stream)
{
    if (T < 0 || T >= (1 << 24) || E < 1 || E > kMaxE) return QUICK_ERR_SHAPE;
    if (!offsets || (T && (!ids || !rows))) return QUICK_ERR_INVALID_ARG;
    if (!aligned(ids, 4) || !aligned(offsets, 4) || !aligned(rows, 4)) return QUICK_ERR_ALIGNMENT;
    (void)hipGetLastError();
    const size_t lds = (kGroupWaves * (E + 1) + E + 2) * sizeof(uint32_t);
    lora_group_kernel<<<1, 64 * kGroupWaves, lds, (hipStream_t)stream>>>(ids, (int)T, (int)E, offsets, rows);
    return launched();
}

extern "C" size_t quick_lora_workspace_bytes(int64_t R, int64_t K, int64_t E, int64_t rank)
{
    if (R < 1 || R >= (1 << 24) || K < 1 || K > (1 << 20) || E < 1 || E > kMaxE || rank < 1 || rank > QUICK_LORA_MAX_RANK)
        return 0;
    int32_t slices, slice;
    slices_of(R, K, E, &slices, &slice);
    return (size_t)slices * R * rank * sizeof(float);
}

extern "C" int quick_lora_add(const void* x, int64_t ldx, int dtype, int64_t T, int64_t K, int64_t N, int64_t E, int64_t rank,
                              const void* a, const void* b, const float* scales, const int32_t* offsets, const int32_t* rows,
                              int64_t R, const void* y, int64_t ldy, void* out, int64_t ldo, void* workspace,
                              size_t workspace_bytes, void* stream)
{
    if (dtype != QUICK_F16 && dtype != QUICK_BF16) return QUICK_ERR_INVALID_ARG;
    const int64_t limit = (int64_t)1 << 40;
    if (T < 0 || T >= (1 << 24) || R < 0 || R > T || K < 8 || K > (1 << 20) || K % 8 || N < 8 || N > (1 << 20) || N % 8 ||
        E < 1 || E > kMaxE || rank < 8 || rank > QUICK_LORA_MAX_RANK || rank % 8 || ldx < K || ldx >= limit || ldy < N ||
        ldy >= limit || ldo < N || ldo >= limit)
        return QUICK_ERR_SHAPE;
    if (R == 0) return QUICK_OK;
    if (!x || !a || !b || !offsets || !rows || !y || !out) return QUICK_ERR_INVALID_ARG;
    if (out == y && ldo != ldy) return QUICK_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(a, 16) || !aligned(b, 16) || !aligned(y, 16) || !aligned(out, 16) || ldx % 8 || ldy % 8 ||
        ldo % 8 || !aligned(scales, 4) || !aligned(offsets, 4) || !aligned(rows, 4))
        return QUICK_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < quick_lora_workspace_bytes(R, K, E, rank)) return QUICK_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return QUICK_ERR_ALIGNMENT;
    LoraArgs g{(const uint8_t*)x, (const uint8_t*)a, (const uint8_t*)b, (const uint8_t*)y, (uint8_t*)out, scales, offsets,
               rows, (float*)workspace, ldx, ldy, ldo, (int32_t)T, (int32_t)K, (int32_t)N, (int32_t)E, (int32_t)rank,
               (int32_t)R};
    slices_of(R, K, E, &g.slices, &g.slice);
    hipStream_t hs = (hipStream_t)stream;
    (void)hipGetLastError();
    const bool tall = tile_rows(R, E) == 64;
    if (dtype == QUICK_F16) {
        if (tall) launch_lora<QUICK_F16, 4>(g, hs);
        else launch_lora<QUICK_F16, 1>(g, hs);
    } else {
        if (tall) launch_lora<QUICK_BF16, 4>(g, hs);
        else launch_lora<QUICK_BF16, 1>(g, hs);
    }
    return launched();
}
