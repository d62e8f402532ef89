// Products with weights in microscaled 4-bit floating point on the scaled
// 16x16x128 matrix instruction of gfx950.
//
// y[m][n] = sum over blocks b of 2^(xs[m][b] + ws[n][b] - 254) *
//           sum over the 32 channels of b of x[m][k] * w[n][k]
//
// The instruction takes, per lane, 32 consecutive channels of one row (16
// bytes of codes, four registers) and that block's scale byte, for both
// operands: lane l holds row l % 16 and block l / 16 of the step's four.  So a
// 16-byte load of a row of codes is an operand as it stands, and so is a
// lane's share of a packed weight unit, which one wave-wide load fetches from
// 1 KiB of consecutive memory.  Nothing is converted or moved on the way.
// The weights are the A operand (result rows), so that a lane ends with four
// consecutive columns of one row of y.
#include <algorithm>

#include "quick_device.h"
#include "quick_mx.h"

namespace {

using namespace quick;

typedef int i8_t __attribute__((ext_vector_type(8)));

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

// Tile number t of the grouped form, tiles of BM rows of one expert each in
// the order of the experts: the lanes count the tiles of eight experts each.
// Offsets that are not in order are taken as the largest so far, and within
// 0..M.  m0 == m1: there is no such tile.
template <int BM>
__device__ __forceinline__ Tile grouped_tile(const MxArgs& a, int t)
{
    constexpr int PER = QUICK_MAX_EXPERTS / 64;
    const int lane = threadIdx.x & 63;
    int at[PER + 1], top = 0;
#pragma unroll
    for (int i = 0; i <= PER; i++) {
        const int e = min(lane * PER + i, a.E);
        at[i] = min(max(a.offsets[e], 0), a.M);
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
    int tiles = 0;
#pragma unroll
    for (int i = 0; i <= PER; i++) low = at[i] = max(at[i], low);
#pragma unroll
    for (int i = 0; i < PER; i++) tiles += (at[i + 1] - at[i] + BM - 1) / BM;
    int upto = tiles;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    const uint64_t past = __ballot(upto > t);
    Tile r = {0, 0, 0};
    if (past == 0) return r;
    const int who = __builtin_ctzll(past);
    int n = t - (upto - tiles);
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

// WN x WK waves; each MT x NT blocks of 16 x 16 of y over a share of the K
// steps (128 channels), operands straight from memory into registers, D steps
// ahead.  The WK shares are added up through LDS in the order of the waves.
// TAIL: K is not a multiple of 128; the blocks past its end are read as zero.
template <int MT, int NT, int WN, int WK, int D, bool GRP, bool TAIL>
__global__ __launch_bounds__(64 * WN * WK) void mx_direct_kernel(MxArgs a)
{
    constexpr int BM = 16 * MT;
    extern __shared__ f4_t part[];    // [WK][WN][MT * NT][64]
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wn = wave % WN, wk = wave / WN, row = lane & 15, blk = lane >> 4;
    Tile t;
    if constexpr (GRP) {
        t = grouped_tile<BM>(a, blockIdx.y);
        if (t.m0 == t.m1) return;
    } else {
        t.m0 = blockIdx.y * BM;
        t.m1 = min(t.m0 + BM, a.M);
        t.e = 0;
    }
    const int KS = (a.K + 127) / 128, KQ = (KS + 3) / 4, KB = a.K / 32, NTT = (a.N + 15) / 16;
    const int nt0 = (blockIdx.x * WN + wn) * NT;
    const int tiles = max(0, min(NT, NTT - nt0));
    const int64_t first = (int64_t)t.e * NTT + min(nt0, NTT - 1);
    const uint8_t* pw = a.packed + first * KS * 1024;
    const uint8_t* ps = a.pscales + first * KQ * 256;
    const uint32_t wbytes = (uint32_t)tiles * KS * 1024, sbytes = (uint32_t)tiles * KQ * 256;
    const rsrc_t rx = make_rsrc(a.codes, (uint32_t)((int64_t)a.T * (a.K / 2)));
    const rsrc_t rs = make_rsrc(a.scales, (uint32_t)((int64_t)a.T * KB));
    uint32_t xo[MT], so[MT];
#pragma unroll
    for (int i = 0; i < MT; i++) {
        int r = min(t.m0 + i * 16 + row, t.m1 - 1);
        if (GRP && a.rows) r = min(max(a.rows[r], 0), a.T - 1);
        xo[i] = (uint32_t)r * (uint32_t)(a.K / 2) + blk * 16;
        so[i] = (uint32_t)r * (uint32_t)KB + (TAIL ? blk : 0);
    }
    const int per = (KS + WK - 1) / WK, s0 = wk * per, s1 = min(KS, s0 + per);
    f4_t acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < NT; j++) acc[i][j] = f4_t{0, 0, 0, 0};
    u4_t w[D][NT], x[D][MT];
    uint32_t ws[D][NT], xs[D][MT];
    auto load = [&](int d, int s) {
        // past the share: empty buffers, which read as zero
        const rsrc_t rw = make_rsrc(pw, s < s1 ? wbytes : 0), rp = make_rsrc(ps, s < s1 ? sbytes : 0);
        const rsrc_t qx = s < s1 ? rx : make_rsrc(a.codes, 0), qs = s < s1 ? rs : make_rsrc(a.scales, 0);
#pragma unroll
        for (int j = 0; j < NT; j++) {
            w[d][j] = ld128(rw, (uint32_t)(j * KS + s) * 1024 + lane * 16, 0);
            ws[d][j] = ld32(rp, (uint32_t)(j * KQ + (s >> 2)) * 256 + lane * 4, 0);
        }
        const bool in = !TAIL || s * 4 + blk < KB;
#pragma unroll
        for (int i = 0; i < MT; i++) {
            x[d][i] = ld128(qx, in ? xo[i] + s * 64 : 0xFFFFFFF0u, 0);
            if constexpr (TAIL) xs[d][i] = ld8(qs, in ? so[i] + s * 4 : 0xFFFFFFF0u, 0);
            else xs[d][i] = ld32(qs, so[i] + s * 4, 0);
        }
    };
#pragma unroll
    for (int d = 0; d < D; d++) load(d, s0 + d);
    for (int s = s0; s < s1; s += D) {
#pragma unroll
        for (int d = 0; d < D; d++) {
            const uint32_t sh = (uint32_t)((s + d) & 3) * 8;
            uint32_t sx[MT], sw[NT];
#pragma unroll
            for (int i = 0; i < MT; i++) sx[i] = TAIL ? xs[d][i] : xs[d][i] >> (8 * blk);
#pragma unroll
            for (int j = 0; j < NT; j++) sw[j] = ws[d][j] >> sh;
#pragma unroll
            for (int i = 0; i < MT; i++)
#pragma unroll
                for (int j = 0; j < NT; j++) acc[i][j] = mx_mfma(w[d][j], x[d][i], acc[i][j], sw[j], sx[i]);
            load(d, s + d + D);
        }
    }
    if constexpr (WK > 1) {
        f4_t* mine = part + (size_t)(wk * WN + wn) * (MT * NT * 64) + lane;
#pragma unroll
        for (int i = 0; i < MT; i++)
#pragma unroll
            for (int j = 0; j < NT; j++) mine[(i * NT + j) * 64] = acc[i][j];
        __syncthreads();
        // a wave's share of the blocks of its columns: row blocks wk, wk + WK, ...
#pragma unroll
        for (int i = 0; i < MT; i++) {
            if (i % WK != wk) continue;
#pragma unroll
            for (int j = 0; j < NT; j++) {
                f4_t v = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < WK; k++) v += part[((size_t)(k * WN + wn) * (MT * NT) + i * NT + j) * 64 + lane];
                acc[i][j] = v;
            }
        }
    }
    const uint16_t* bias = a.bias ? a.bias + (int64_t)t.e * a.N : nullptr;
#pragma unroll
    for (int i = 0; i < MT; i++) {
        if (WK > 1 && i % WK != wk) continue;
        const int m = t.m0 + i * 16 + row;
        if (m >= t.m1) continue;
        if (!a.gated) {
#pragma unroll
            for (int j = 0; j < NT; j++) {
                const int n = (nt0 + j) * 16 + blk * 4;
                f4_t v = acc[i][j];
                if (bias)
#pragma unroll
                    for (int c = 0; c < 4; c++) v[c] += n + c < a.N ? bias_at(a, bias, n + c) : 0.0f;
                store4(a, m, n, a.N, v);
            }
        } else if constexpr (NT % 2 == 0) {
#pragma unroll
            for (int j = 0; j < NT; j += 2) {
                const int n = (nt0 + j) * 8 + blk * 4;    // column of y
                f4_t g = acc[i][j], u = acc[i][j + 1], v;
                if (bias && n < a.N / 2)
#pragma unroll
                    for (int c = 0; c < 4; c++) {
                        g[c] += bias_at(a, bias, n + c);
                        u[c] += bias_at(a, bias, a.N / 2 + n + c);
                    }
#pragma unroll
                for (int c = 0; c < 4; c++) v[c] = silu(g[c]) * u[c];
                store4(a, m, n, a.N / 2, v);
            }
        }
    }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <int MT, int NT, int WN, int WK, int D, bool GRP>
void launch_direct(const MxArgs& a, int64_t row_tiles, hipStream_t hs)
{
    const dim3 grid((uint32_t)ceil_div(ceil_div(a.N, 16), NT * WN), (uint32_t)row_tiles), block(64 * WN * WK);
    const size_t lds = WK > 1 ? (size_t)WK * WN * MT * NT * 64 * sizeof(f4_t) : 0;
    if (a.K % 128) mx_direct_kernel<MT, NT, WN, WK, D, GRP, true><<<grid, block, lds, hs>>>(a);
    else mx_direct_kernel<MT, NT, WN, WK, D, GRP, false><<<grid, block, lds, hs>>>(a);
}

// Rows a tile: those of the call, or of an expert on average.
template <bool GRP>
int launch_mx(const MxArgs& a, hipStream_t hs)
{
    const int64_t rows = GRP ? ceil_div(a.M, a.E) : a.M;
    // an expert's last tile may be short: at most one such tile each
    auto tiles = [&](int bm) { return GRP ? a.M / bm + std::min(a.E, a.M) : ceil_div(a.M, bm); };
    (void)hipGetLastError();
    if (rows <= 16 && tiles(16) <= 65535) {
        if (a.gated) launch_direct<1, 2, 1, 8, 4, GRP>(a, tiles(16), hs);
        else launch_direct<1, 1, 1, 8, 4, GRP>(a, tiles(16), hs);
    } else if (rows <= 64 && tiles(32) <= 65535) {
        launch_direct<2, 2, 1, 8, 2, GRP>(a, tiles(32), hs);
    } else {
        if (tiles(64) > 65535) return QUICK_ERR_SHAPE;
        launch_direct<4, 4, 2, 2, 2, GRP>(a, tiles(64), hs);
    }
    return launched();
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
    return launch_mx<false>(make_args(codes, scales, packed, packed_scales, y, dtype, M, N, K, bias, activation),
                            (hipStream_t)stream);
}

extern "C" size_t quick_mxfp4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    if (M <= 0 || check_product(M, M, N, K, QUICK_F16, QUICK_ACT_NONE)) return 0;
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
    uint8_t* codes = (uint8_t*)workspace;
    uint8_t* scales = codes + code_bytes(M, K);
    st = check_pointers(codes, scales, packed, packed_scales, y, bias);
    if (st) return st;
    st = quick_mxfp4_quantize(x, dtype, K, M, K, codes, scales, stream);
    if (st) return st;
    return launch_mx<false>(make_args(codes, scales, packed, packed_scales, y, dtype, M, N, K, bias, activation),
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
    return launch_mx<true>(a, (hipStream_t)stream);
}
