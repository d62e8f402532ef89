// Microscaled 4-bit floating point: quantisation, its inverse, and the packed
// form of weights.
#include <algorithm>

#include "quick_mx.h"
#include "quick_mx_quant.h"

namespace {

using namespace quick;

constexpr int kThreads = 256;
constexpr int kUnroll = 4;   // pieces of eight values a thread has in flight
constexpr int64_t kMaxGrid = (1 << 24) - 1;   // workgroups: a launch has under 2^32 threads

// One thread per eight values, four neighbouring lanes per block: amax over
// the eight, over the four lanes by two lane exchanges, then one 4-byte store
// of codes and, from every fourth lane, the scale byte.  Bound by the bytes (2
// or 4 in, 17/32 out per value); x is read past the caches (22016 x 4096 bf16
// to codes and back: 72 us, 85 through them).
// A row is `pieces` pieces of eight; a workgroup takes kUnroll * kThreads of
// one row, with all loads issued before the first is used.
template <int DT>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const uint8_t* x, int64_t row_bytes, uint32_t* codes,
                                                               uint8_t* scales, int64_t pieces, uint32_t wgs_per_row)
{
    constexpr int NV = DT == QUICK_F32 ? 2 : 1;
    const uint32_t row = blockIdx.x / wgs_per_row, part = blockIdx.x % wgs_per_row;
    const int64_t p0 = (int64_t)part * (kUnroll * kThreads) + threadIdx.x;
    const uint8_t* xr = x + row * row_bytes;
    u4_t raw[kUnroll][NV];
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
        // blocks are whole (pieces is a multiple of 4), so a group of four
        // lanes is inside or outside together
        const int64_t p = std::min(p0 + u * kThreads, pieces - 4 + (int64_t)(threadIdx.x & 3));
#pragma unroll
        for (int i = 0; i < NV; i++) raw[u][i] = __builtin_nontemporal_load((const u4_t*)(xr + (p * NV + i) * 16));
    }
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
        const int64_t p = p0 + u * kThreads;
        float v[8];
        unpack8<DT>(raw[u], v);
        const uint32_t s = block_scale(max_of_quad(amax8(v)));
        const uint32_t c = block_codes(v, s);
        if (p < pieces) {
            const int64_t at = row * pieces + p;
            codes[at] = c;
            if ((threadIdx.x & 3) == 0) scales[at >> 2] = (uint8_t)s;
        }
    }
}

// One thread per eight values.  The code's value is exact in binary32 and so
// is its product with a power of two (a code has two significant bits, also
// below the normal range); then one rounding to the type.
template <int DT>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(const uint32_t* codes, const uint8_t* scales,
                                                                 uint8_t* y, int64_t pieces)
{
    const int64_t p0 = (int64_t)blockIdx.x * (kUnroll * kThreads) + threadIdx.x;
    uint32_t c[kUnroll], s[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
        const int64_t p = std::min(p0 + u * kThreads, pieces - 1);
        c[u] = codes[p];
        s[u] = scales[p >> 2];
    }
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
        const int64_t p = p0 + u * kThreads;
        const float k = bits_as<float>(s[u] == 255 ? 0x7FC00000u : s[u] == 0 ? 0x00400000u : s[u] << 23);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            // magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6 as twice their value
            const uint32_t n = c[u] >> (4 * i);
            const float m = (float)((0xC8643210u >> (4 * (n & 7))) & 15u) * 0.5f;
            v[i] = bits_as<float>(bits_as<uint32_t>(m) | (n & 8u) << 28) * k;
        }
        if (p >= pieces) continue;
        if constexpr (DT == QUICK_F32) {
            u4_t* o = (u4_t*)(y + p * 32);
            o[0] = u4_t{bits_as<uint32_t>(v[0]), bits_as<uint32_t>(v[1]), bits_as<uint32_t>(v[2]), bits_as<uint32_t>(v[3])};
            o[1] = u4_t{bits_as<uint32_t>(v[4]), bits_as<uint32_t>(v[5]), bits_as<uint32_t>(v[6]), bits_as<uint32_t>(v[7])};
        } else {
            *(u4_t*)(y + p * 16) = u4_t{to16x2<DT>(v[0], v[1]), to16x2<DT>(v[2], v[3]), to16x2<DT>(v[4], v[5]),
                                        to16x2<DT>(v[6], v[7])};
        }
    }
}

// Source row of packed column n: with gate_up, tiles of 16 gate columns and
// of the matching up columns alternate.
__device__ __forceinline__ int64_t source_row(int64_t n, int64_t N, int gate_up)
{
    return gate_up ? (n >> 5) * 16 + (n & 15) + ((n & 16) ? N / 2 : 0) : n;
}

// One thread per 16-byte operand of a lane.
__global__ __launch_bounds__(kThreads) void mx_pack_codes_kernel(const uint8_t* codes, u4_t* packed, int64_t first, int64_t E,
                                                                 int64_t N, int64_t K, int64_t NT, int64_t KS,
                                                                 int gate_up)
{
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x + first;
    if (at >= E * NT * KS * 64) return;
    const int64_t lane = at & 63, unit = at >> 6, ks = unit % KS, tile = unit / KS, nt = tile % NT, e = tile / NT;
    const int64_t n = nt * 16 + (lane & 15), b = ks * 4 + (lane >> 4);
    u4_t v = {0, 0, 0, 0};
    if (n < N && b < K / 32) v = *(const u4_t*)(codes + ((e * N + source_row(n, N, gate_up)) * (K / 2) + b * 16));
    packed[at] = v;
}

// One thread per dword of four scales (channels 128 apart).
__global__ __launch_bounds__(kThreads) void mx_pack_scales_kernel(const uint8_t* scales, uint32_t* packed, int64_t first,
                                                                  int64_t E, int64_t N, int64_t K, int64_t NT,
                                                                  int64_t KQ, int gate_up)
{
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x + first;
    if (at >= E * NT * KQ * 64) return;
    const int64_t lane = at & 63, unit = at >> 6, kq = unit % KQ, tile = unit / KQ, nt = tile % NT, e = tile / NT;
    const int64_t n = nt * 16 + (lane & 15);
    uint32_t v = 0;
    if (n < N) {
        const uint8_t* s = scales + (e * N + source_row(n, N, gate_up)) * (K / 32);
        for (int j = 0; j < 4; j++) {
            const int64_t b = (kq * 4 + j) * 4 + (lane >> 4);
            if (b < K / 32) v |= (uint32_t)s[b] << (8 * j);
        }
    }
    packed[at] = v;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int check_matrix(int64_t rows, int64_t K)
{
    return rows < 0 || rows > (1 << 24) || K <= 0 || K % 32 != 0 || K > (1 << 22) ? QUICK_ERR_SHAPE : QUICK_OK;
}

}  // namespace

extern "C" int quick_mxfp4_quantize(const void* x, int dtype, int64_t ldx, int64_t rows, int64_t K, void* codes,
                                    void* scales, void* stream)
{
    if (dtype < QUICK_F16 || dtype > QUICK_F32) return QUICK_ERR_INVALID_ARG;
    int st = check_matrix(rows, K);
    if (st) return st;
    if (ldx < K || ldx >= ((int64_t)1 << 40)) return QUICK_ERR_SHAPE;
    if (rows == 0) return QUICK_OK;
    if (!x || !codes || !scales) return QUICK_ERR_INVALID_ARG;
    const int64_t es = dtype == QUICK_F32 ? 4 : 2;
    if (!aligned(x, 16) || !aligned(codes, 16) || (rows > 1 && ldx * es % 16 != 0)) return QUICK_ERR_ALIGNMENT;
    hipStream_t hs = (hipStream_t)stream;
    // rows without a gap are one long row
    const bool flat = ldx == K || rows == 1;
    const int64_t r = flat ? 1 : rows, pieces = (flat ? rows * K : K) / 8;
    const int64_t wgs = ceil_div(pieces, kThreads * kUnroll);
    if (r * wgs > kMaxGrid) return QUICK_ERR_SHAPE;
    (void)hipGetLastError();
    const dim3 grid((uint32_t)(r * wgs)), block(kThreads);
    const auto* xx = (const uint8_t*)x;
    auto* c = (uint32_t*)codes;
    auto* s = (uint8_t*)scales;
    if (dtype == QUICK_F16)
        mx_quantize_kernel<QUICK_F16><<<grid, block, 0, hs>>>(xx, ldx * es, c, s, pieces, (uint32_t)wgs);
    else if (dtype == QUICK_BF16)
        mx_quantize_kernel<QUICK_BF16><<<grid, block, 0, hs>>>(xx, ldx * es, c, s, pieces, (uint32_t)wgs);
    else
        mx_quantize_kernel<QUICK_F32><<<grid, block, 0, hs>>>(xx, ldx * es, c, s, pieces, (uint32_t)wgs);
    return launched();
}

extern "C" int quick_mxfp4_dequantize(const void* codes, const void* scales, int dtype, int64_t rows, int64_t K, void* y,
                                      void* stream)
{
    if (dtype < QUICK_F16 || dtype > QUICK_F32) return QUICK_ERR_INVALID_ARG;
    int st = check_matrix(rows, K);
    if (st) return st;
    if (rows == 0) return QUICK_OK;
    if (!codes || !scales || !y) return QUICK_ERR_INVALID_ARG;
    if (!aligned(codes, 16) || !aligned(y, 16)) return QUICK_ERR_ALIGNMENT;
    hipStream_t hs = (hipStream_t)stream;
    const int64_t pieces = rows * K / 8, wgs = ceil_div(pieces, kThreads * kUnroll);
    if (wgs > kMaxGrid) return QUICK_ERR_SHAPE;
    (void)hipGetLastError();
    const dim3 grid((uint32_t)wgs), block(kThreads);
    const auto* c = (const uint32_t*)codes;
    const auto* s = (const uint8_t*)scales;
    auto* yy = (uint8_t*)y;
    if (dtype == QUICK_F16) mx_dequantize_kernel<QUICK_F16><<<grid, block, 0, hs>>>(c, s, yy, pieces);
    else if (dtype == QUICK_BF16) mx_dequantize_kernel<QUICK_BF16><<<grid, block, 0, hs>>>(c, s, yy, pieces);
    else mx_dequantize_kernel<QUICK_F32><<<grid, block, 0, hs>>>(c, s, yy, pieces);
    return launched();
}

extern "C" int quick_mxfp4_packed_sizes(int64_t N, int64_t K, size_t* packed_bytes, size_t* scales_bytes)
{
    if (N <= 0 || check_matrix(N, K) || N * K >= ((int64_t)1 << 33)) return QUICK_ERR_SHAPE;
    const int64_t NT = ceil_div(N, 16);
    if (packed_bytes) *packed_bytes = (size_t)(NT * ceil_div(K, 128) * 1024);
    if (scales_bytes) *scales_bytes = (size_t)(NT * ceil_div(K, 512) * 256);
    return QUICK_OK;
}

extern "C" int quick_mxfp4_pack(const void* codes, const void* scales, int64_t E, int64_t N, int64_t K, int gate_up,
                                void* packed, void* packed_scales, void* stream)
{
    int st = quick_mxfp4_packed_sizes(N, K, nullptr, nullptr);
    if (st) return st;
    if (E < 1 || E > QUICK_MAX_EXPERTS || (gate_up && N % 32 != 0)) return QUICK_ERR_SHAPE;
    if (!codes || !scales || !packed || !packed_scales) return QUICK_ERR_INVALID_ARG;
    if (!aligned(codes, 16) || !aligned(packed, 16) || !aligned(packed_scales, 4)) return QUICK_ERR_ALIGNMENT;
    hipStream_t hs = (hipStream_t)stream;
    const int64_t NT = ceil_div(N, 16), KS = ceil_div(K, 128), KQ = ceil_div(K, 512);
    (void)hipGetLastError();
    // as many launches as the limit of a grid asks for: one, as a rule
    for (int64_t first = 0, n = E * NT * KS * 64; first < n; first += kMaxGrid * kThreads) {
        const int64_t wgs = std::min(ceil_div(n - first, kThreads), kMaxGrid);
        mx_pack_codes_kernel<<<dim3((uint32_t)wgs), dim3(kThreads), 0, hs>>>((const uint8_t*)codes, (u4_t*)packed, first,
                                                                             E, N, K, NT, KS, gate_up);
    }
    for (int64_t first = 0, n = E * NT * KQ * 64; first < n; first += kMaxGrid * kThreads) {
        const int64_t wgs = std::min(ceil_div(n - first, kThreads), kMaxGrid);
        mx_pack_scales_kernel<<<dim3((uint32_t)wgs), dim3(kThreads), 0, hs>>>(
            (const uint8_t*)scales, (uint32_t*)packed_scales, first, E, N, K, NT, KQ, gate_up);
    }
    return launched();
}
