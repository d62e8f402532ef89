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
constexpr int kThreads = 256;

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

// The workgroup's tile of H rows, the index'th of all: the first wave adds the
// adapters' tiles up, eight to a lane (and the rows without one).
template <int H>
__device__ __forceinline__ RowTile find_tile(const LoraArgs& a, int index, int (&space)[3])
{
    constexpr int PER = kMaxE / 64;
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        int first[PER + 1], n[PER + 1], sum = 0;
#pragma unroll
        for (int i = 0; i <= PER; i++) {
            // the last lane also has the rows without an adapter
            const int e = i < PER ? lane * PER + i : lane == 63 ? a.E : a.E + 1;
            first[i] = n[i] = 0;
            if (e <= a.E) {
                first[i] = clamped(a.offsets[e], 0, a.R);
                const int end = e < a.E ? clamped(a.offsets[e + 1], first[i], a.R) : a.R;
                n[i] = i < PER && e == a.E ? 0 : end - first[i];
            }
            sum += (n[i] + H - 1) / H;
        }
        int upto = sum;
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 63 && index >= upto) space[2] = 0;
        int at = upto - sum;
        if (index >= at && index < upto) {
#pragma unroll
            for (int i = 0; i <= PER; i++) {
                const int tiles = (n[i] + H - 1) / H;
                if (index >= at && index < at + tiles) {
                    space[0] = i < PER ? lane * PER + i : a.E;
                    space[1] = first[i] + (index - at) * H;
                    space[2] = min(H, n[i] - (index - at) * H);
                }
                at += tiles;
            }
        }
    }
    __syncthreads();
    return {(int)uniform((uint32_t)space[0]), (int)uniform((uint32_t)space[1]), (int)uniform((uint32_t)space[2])};
}

// low = x . A^T of a tile of 16 TM rows and a slice of the channels.  Waves take
// every fourth 128 channels; the rows of A (16 RT of them) are the instruction's
// rows, those of x its columns, both straight from memory, 16 bytes a lane; the
// waves' sums meet in LDS.
template <int DT, int RT, int TM>
__global__ __launch_bounds__(kThreads) void lora_down_kernel(LoraArgs a)
{
    __shared__ int space[3];
    __shared__ float sums[4][16][16 * RT + 4];
    const RowTile t = find_tile<16 * TM>(a, blockIdx.x, space);
    if (t.count == 0 || t.e == a.E) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const int k0 = blockIdx.y * a.slice, k1 = min(a.K, k0 + a.slice);
    const uint8_t* x[TM];
    bool live[TM];
#pragma unroll
    for (int m = 0; m < TM; m++) {
        const int at = m * 16 + c;
        const int row = at < t.count ? a.rows[t.first + at] : -1;
        live[m] = row >= 0 && row < a.T;
        x[m] = a.x + 2 * ((int64_t)(live[m] ? row : 0) * a.ldx);
    }
    const uint8_t* w = a.a + 2 * (int64_t)t.e * a.rank * a.K;
    f4_t acc[TM][RT];
#pragma unroll
    for (int m = 0; m < TM; m++)
#pragma unroll
        for (int r = 0; r < RT; r++) acc[m][r] = f4_t{0, 0, 0, 0};
    for (int k = k0 + wave * 128; k < k1; k += 512) {
#pragma unroll
        for (int s = 0; s < 4; s++) {
            const int at = k + s * 32 + g * 8;
            u4_t xv[TM], wv[RT];
#pragma unroll
            for (int m = 0; m < TM; m++) {
                xv[m] = u4_t{0, 0, 0, 0};
                if (at < k1 && live[m]) xv[m] = *(const u4_t*)(x[m] + 2 * at);
            }
#pragma unroll
            for (int r = 0; r < RT; r++) {
                wv[r] = u4_t{0, 0, 0, 0};
                if (at < k1 && r * 16 + c < a.rank) wv[r] = *(const u4_t*)(w + 2 * ((int64_t)(r * 16 + c) * a.K + at));
            }
#pragma unroll
            for (int m = 0; m < TM; m++)
#pragma unroll
                for (int r = 0; r < RT; r++) acc[m][r] = mfma16<DT>(wv[r], xv[m], acc[m][r]);
        }
    }
#pragma unroll
    for (int m = 0; m < TM; m++) {
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; r++) *(f4_t*)&sums[wave][c][r * 16 + g * 4] = acc[m][r];
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * 16 * RT; i += kThreads) {
            const int row = i / (16 * RT), r = i % (16 * RT);
            if (m * 16 + row < t.count && r < a.rank)
                a.low[((int64_t)blockIdx.y * a.R + t.first + m * 16 + row) * a.rank + r] =
                    sums[0][row][r] + sums[1][row][r] + sums[2][row][r] + sums[3][row][r];
        }
    }
}

// out = y + low . B^T of a tile of 16 TM rows and 256 columns, 64 a wave.  The
// rows of B are the instruction's rows, in an order that leaves a lane 16
// consecutive columns of its token: row 4 g + i of tile j is column 16 g + 4 j +
// i.  With a rank of 8 or 16 a lane group's 16 bytes are of another tile (or of
// two), and both operands are zero but for that group's lanes, so that every
// load is full.
template <int DT, int RS, int TM>
__global__ __launch_bounds__(kThreads) void lora_up_kernel(LoraArgs a)
{
    // RS: the rank's steps of 32 (0: rank 8 or 16)
    constexpr int R32 = RS ? RS * 32 : 32, ROW = R32 + 8;
    __shared__ int space[3];
    __shared__ __align__(16) uint16_t low[16 * TM][ROW];
    const RowTile t = find_tile<16 * TM>(a, blockIdx.x, space);
    if (t.count == 0) return;
    const bool bare = t.e == a.E;
    if (bare && a.out == a.y) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.y * 256 + wave * 64;
    f4_t acc[TM][4];
#pragma unroll
    for (int m = 0; m < TM; m++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc[m][j] = f4_t{0, 0, 0, 0};
    if (!bare) {
        const float scale = a.scales ? a.scales[t.e] : 1.0f;
        for (int i = threadIdx.x; i < 16 * TM * R32; i += kThreads) {
            const int row = i / R32, r = i % R32;
            float v = 0;
            if (row < t.count && r < a.rank)
                for (int s = 0; s < a.slices; s++) v += a.low[((int64_t)s * a.R + t.first + row) * a.rank + r];
            low[row][r] = to16<DT>(v * scale);
        }
        __syncthreads();
        const uint8_t* b = a.b + 2 * (int64_t)t.e * a.N * a.rank;
        // column of this lane's row of tile j
        auto column = [&](int j) { return n0 + (c >> 2) * 16 + j * 4 + (c & 3); };
        if constexpr (RS == 0) {
            // 2 or 4 tiles of one load
            const int per = 32 / a.rank, mine = g * 8 / a.rank, r = g * 8 % a.rank;
            for (int j0 = 0; j0 < 4; j0 += per) {
                const int n = column(j0 + mine);
                u4_t w = {0, 0, 0, 0};
                if (n < a.N) w = *(const u4_t*)(b + 2 * ((int64_t)n * a.rank + r));
#pragma unroll
                for (int m = 0; m < TM; m++) {
                    const u4_t v = *(const u4_t*)&low[m * 16 + c][r];
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        if (j >= j0 && j < j0 + per)
                            acc[m][j] = mfma16<DT>(mine == j - j0 ? w : u4_t{0, 0, 0, 0},
                                                   mine == j - j0 ? v : u4_t{0, 0, 0, 0}, acc[m][j]);
                }
            }
        } else {
#pragma unroll
            for (int s = 0; s < RS; s++) {
                u4_t w[4];
                const int r = s * 32 + g * 8;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const int n = column(j);
                    w[j] = u4_t{0, 0, 0, 0};
                    if (n < a.N && r < a.rank) w[j] = *(const u4_t*)(b + 2 * ((int64_t)n * a.rank + r));
                }
#pragma unroll
                for (int m = 0; m < TM; m++) {
                    const u4_t v = *(const u4_t*)&low[m * 16 + c][r];
#pragma unroll
                    for (int j = 0; j < 4; j++) acc[m][j] = mfma16<DT>(w[j], v, acc[m][j]);
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < TM; m++) {
        const int at = m * 16 + c;
        const int row = at < t.count ? a.rows[t.first + at] : -1;
        if (row < 0 || row >= a.T) continue;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int n = n0 + g * 16 + h * 8;
            if (n >= a.N) continue;
            const u4_t y = *(const u4_t*)(a.y + 2 * ((int64_t)row * a.ldy + n));
            u4_t o;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const f4_t v = acc[m][h * 2 + i / 2];
                o[i] = to16x2<DT>(from16<DT>((uint16_t)y[i]) + v[i % 2 * 2], from16<DT>((uint16_t)(y[i] >> 16)) + v[i % 2 * 2 + 1]);
            }
            *(u4_t*)(a.out + 2 * ((int64_t)row * a.ldo + n)) = bare ? y : o;
        }
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

// Slices of the channels: enough workgroups for the chip, 512 channels or more.
void slices_of(int64_t R, int64_t K, int64_t E, int32_t* slices, int32_t* slice)
{
    const int64_t n = std::max<int64_t>(1, std::min(ceil_div(K, 512), 512 / tiles_of(R, E)));
    *slice = (int32_t)(ceil_div(ceil_div(K, n), 128) * 128);
    *slices = (int32_t)ceil_div(K, *slice);
}

template <int DT, int TM>
void launch_lora(const LoraArgs& a, hipStream_t hs)
{
    const uint32_t tiles = (uint32_t)tiles_of(a.R, a.E);
    const dim3 down(tiles, a.slices), up(tiles, (uint32_t)ceil_div(a.N, 256));
    if (a.rank <= 16) lora_down_kernel<DT, 1, TM><<<down, kThreads, 0, hs>>>(a);
    else if (a.rank <= 32) lora_down_kernel<DT, 2, TM><<<down, kThreads, 0, hs>>>(a);
    else if (a.rank <= 64) lora_down_kernel<DT, 4, TM><<<down, kThreads, 0, hs>>>(a);
    else lora_down_kernel<DT, 8, TM><<<down, kThreads, 0, hs>>>(a);
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
