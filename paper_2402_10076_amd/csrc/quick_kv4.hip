// Rotary positions, and writing and reading the paged 4-bit cache.
#include <algorithm>

#include "quick_kv4.h"
#include "quick_mx_quant.h"

namespace {

using namespace quick;

constexpr int kThreads = 256;
constexpr int64_t kMaxGrid = (1 << 24) - 1;   // workgroups: a launch has under 2^32 threads

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------------------
// rotary positions
// ---------------------------------------------------------------------------

constexpr int kMaxChannels = 4096;

struct RotaryArgs {
    const uint8_t* x;
    uint8_t* out;
    const int32_t* positions;
    const double* freqs;
    int64_t x_token, x_head, out_token, out_head;   // elements
    int32_t H, D, half;       // half = R / 2
    int32_t pieces;           // of a head: of its pairs, then of the channels that stay
    int32_t turning;          // of those, the pairs'
    int32_t together;         // heads that a workgroup works on at a time
    int32_t heads;            // heads of a workgroup
    uint32_t parts;           // workgroups of a token
    int32_t copy;             // whether the channels that stay are to be copied
    float factor, sign;
};

template <int DT>
struct Element {
    typedef uint16_t type;
    static __device__ __forceinline__ float get(type v) { return from16<DT>(v); }
    static __device__ __forceinline__ type put(float v) { return to16<DT>(v); }
};
template <>
struct Element<QUICK_F32> {
    typedef float type;
    static __device__ __forceinline__ float get(type v) { return v; }
    static __device__ __forceinline__ type put(float v) { return v; }
};

// A workgroup turns some heads of one token: it works the token's R / 2 pairs
// of cosine and sine out once, in LDS, while its first loads are under way, and
// a thread keeps its place in the heads, four of them at a time.  The angle is a
// binary64 product, cut to its turns there, and the rest, at most half a turn, is
// binary32: two products' roundings and that of 1 / (2 pi) make an angle of 2^31
// radians off by 2^-20.6 of one at most, the cut to binary32 any by 2^-23.3.
// Bound by the bytes, x once and out once: 8192 tokens of 72 heads of 128 (64
// turned) take 54.6 us, 5.5 TB/s; a few tokens by latency (2.8 us).
template <int DT, int V, bool INTER>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a)
{
    typedef Element<DT> E;
    typedef typename E::type T;
    struct alignas(sizeof(T) * V) Vec {
        T v[V];
    };
    constexpr int BATCH = 4;
    __shared__ float2 turn[kMaxChannels / 2];
    const int64_t t = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts;
    const int wide = min(a.pieces, kThreads);
    const int first = threadIdx.x % wide, row = threadIdx.x / wide;
    const int h1 = min(a.H, (part + 1) * a.heads), h0 = row < a.together ? part * a.heads + row : h1;
    // channels of piece p: of a pair's two places, or of those that stay (once)
    auto places = [&](int p, int& c, int& d) {
        if (p >= a.turning) c = d = 2 * a.half + (p - a.turning) * V;
        else if (INTER) c = p * 2 * V, d = c + V;
        else c = p * V, d = c + a.half;
    };
    Vec u[BATCH], w[BATCH];
    auto load = [&](int p, int h) {
        int c, d;
        places(p, c, d);
        if (p >= a.turning && !a.copy) return;
#pragma unroll
        for (int i = 0; i < BATCH; i++) {
            if (h + i * a.together >= h1) continue;
            const T* x = (const T*)a.x + t * a.x_token + (h + i * a.together) * a.x_head;
            u[i] = *(const Vec*)(x + c);
            if (p < a.turning) w[i] = *(const Vec*)(x + d);
        }
    };
    load(first, h0);
    for (int i = threadIdx.x; i < a.half; i += kThreads) {
        double r = (double)a.positions[t] * a.freqs[i] * 0.15915494309189533577;   // 1 / (2 pi)
        r -= rint(r);
        float s, c;
        sincospif(2.0f * (float)r, &s, &c);
        turn[i] = make_float2(c * a.factor, s * a.factor * a.sign);
    }
    __syncthreads();
    for (int p = first; p < a.pieces; p += wide) {
        int c, d;
        places(p, c, d);
        for (int h = h0; h < h1; h += BATCH * a.together) {
            if (p != first || h != h0) load(p, h);
#pragma unroll
            for (int b = 0; b < BATCH; b++) {
                if (h + b * a.together >= h1) continue;
                T* o = (T*)a.out + t * a.out_token + (h + b * a.together) * a.out_head;
                if (p >= a.turning) {
                    if (a.copy) *(Vec*)(o + c) = u[b];
                    continue;
                }
                T in[2 * V], res[2 * V];
#pragma unroll
                for (int i = 0; i < V; i++) {
                    in[i] = u[b].v[i];
                    in[V + i] = w[b].v[i];
                }
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float2 cs = turn[p * V + i];
                    const int m = INTER ? 2 * i : i, n = INTER ? 2 * i + 1 : V + i;
                    const float x = E::get(in[m]), y = E::get(in[n]);
                    res[m] = E::put(x * cs.x - y * cs.y);
                    res[n] = E::put(y * cs.x + x * cs.y);
                }
                Vec y, z;
#pragma unroll
                for (int i = 0; i < V; i++) {
                    y.v[i] = res[i];
                    z.v[i] = res[V + i];
                }
                *(Vec*)(o + c) = y;
                *(Vec*)(o + d) = z;
            }
        }
    }
}

template <int DT, int V>
void launch_rotary(const RotaryArgs& a, int64_t T, bool inter, hipStream_t hs)
{
    const dim3 grid((uint32_t)(T * a.parts));
    if (inter) rotary_kernel<DT, V, true><<<grid, kThreads, 0, hs>>>(a);
    else rotary_kernel<DT, V, false><<<grid, kThreads, 0, hs>>>(a);
}

// ---------------------------------------------------------------------------
// the cache
// ---------------------------------------------------------------------------

struct CacheArgs {
    const uint8_t *k, *v;                                  // write: 16-bit keys and values
    uint8_t *k_out, *v_out;                                // read
    int64_t k_token, k_head, v_token, v_head;              // elements
    const int32_t* slots;
    uint8_t* cache;
    int64_t T, slots_end;
    int32_t heads;
};

// A workgroup writes one head of 16 tokens (32 with D = 64, 8 with D = 256): a
// thread holds eight channels of a token's key and of its value, four
// neighbouring lanes a block, as in quick_mxfp4_quantize.  Tokens that follow
// each other share the 128-byte lines of the values' order, and one workgroup
// writes them.
// Bound by the bytes: 2 in, 17/32 out per value; a few tokens by the launch (3
// us).  8192 tokens of 32 heads of 128: 33 us, 5.1 TB/s, with slots in order; 42
// with slots in random order, whose parts of lines make twice the bytes written.
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void kv4_write_kernel(CacheArgs a)
{
    typedef Kv4<D> L;
    constexpr int P = D / 8, TOKENS = kThreads / P;
    const int h = blockIdx.x % a.heads, p = threadIdx.x % P;
    const int64_t t = (int64_t)(blockIdx.x / a.heads) * TOKENS + threadIdx.x / P;
    // the lanes of a block share a token, so they stay together
    if (t >= a.T) return;
    u4_t raw[2];
    raw[0] = __builtin_nontemporal_load((const u4_t*)(a.k + 2 * (t * a.k_token + h * a.k_head + p * 8)));
    raw[1] = __builtin_nontemporal_load((const u4_t*)(a.v + 2 * (t * a.v_token + h * a.v_head + p * 8)));
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.slots_end) return;
    uint8_t* page = a.cache + ((slot / kPage) * a.heads + h) * L::kBytes;
    const int s = (int)(slot % kPage);
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const u4_t one[1] = {raw[i]};
        float v[8];
        unpack8<DT>(one, v);
        const uint32_t scale = block_scale(max_of_quad(amax8(v)));
        const uint32_t codes = block_codes(v, scale);
        if (i == 0) {
            *(uint32_t*)(page + L::key(s, p)) = codes;
            if (p % 4 == 0) page[L::key_scale(s, p / 4)] = (uint8_t)scale;
        } else {
            uint8_t* to = page + L::value(s, p);
            if constexpr (L::kLane == 8) *(uint32_t*)to = codes;
            else {
                *(uint16_t*)to = (uint16_t)codes;
                *(uint16_t*)(to + 2 * L::kLane) = (uint16_t)(codes >> 16);
            }
            if (p % 4 == 0) page[L::value_scale(s, p / 4)] = (uint8_t)scale;
        }
    }
}

// Value of a code times a power of two, as in quick_mxfp4_dequantize: exact in
// binary32 but for the type's end.
__device__ __forceinline__ float code_value(uint32_t n, float k)
{
    const float m = (float)((0xC8643210u >> (4 * (n & 7))) & 15u) * 0.5f;
    return bits_as<float>(bits_as<uint32_t>(m) | (n & 8u) << 28) * k;
}

// The same threads the other way (those 8192 tokens: 32.5 us, 5.2 TB/s).
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(CacheArgs a)
{
    typedef Kv4<D> L;
    constexpr int P = D / 8, TOKENS = kThreads / P;
    const int h = blockIdx.x % a.heads, p = threadIdx.x % P;
    const int64_t t = (int64_t)(blockIdx.x / a.heads) * TOKENS + threadIdx.x / P;
    if (t >= a.T) return;
    const int64_t slot = a.slots[t];
    const bool inside = slot >= 0 && slot < a.slots_end;
    const uint8_t* page = a.cache + ((inside ? slot / kPage : 0) * a.heads + h) * L::kBytes;
    const int s = inside ? (int)(slot % kPage) : 0;
    uint32_t codes[2] = {0, 0}, scale[2] = {0, 0};
    if (inside) {
        const uint8_t* from = page + L::value(s, p);
        codes[0] = *(const uint32_t*)(page + L::key(s, p));
        scale[0] = page[L::key_scale(s, p / 4)];
        if constexpr (L::kLane == 8) codes[1] = *(const uint32_t*)from;
        else codes[1] = *(const uint16_t*)from | (uint32_t)*(const uint16_t*)(from + 2 * L::kLane) << 16;
        scale[1] = page[L::value_scale(s, p / 4)];
    }
    const int64_t at = (t * a.heads + h) * D + p * 8;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        uint8_t* y = i ? a.v_out : a.k_out;
        if (!y) continue;
        const float k = bits_as<float>(scale[i] == 255 ? 0x7FC00000u : scale[i] == 0 ? 0x00400000u : scale[i] << 23);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = code_value(codes[i] >> (4 * j), k);
        if constexpr (DT == QUICK_F32) {
            u4_t* o = (u4_t*)(y + at * 4);
            o[0] = u4_t{bits_as<uint32_t>(v[0]), bits_as<uint32_t>(v[1]), bits_as<uint32_t>(v[2]), bits_as<uint32_t>(v[3])};
            o[1] = u4_t{bits_as<uint32_t>(v[4]), bits_as<uint32_t>(v[5]), bits_as<uint32_t>(v[6]), bits_as<uint32_t>(v[7])};
        } else {
            *(u4_t*)(y + at * 2) = u4_t{to16x2<DT>(v[0], v[1]), to16x2<DT>(v[2], v[3]), to16x2<DT>(v[4], v[5]),
                                        to16x2<DT>(v[6], v[7])};
        }
    }
}

template <int DT>
void launch_write(const CacheArgs& a, int64_t D, uint32_t grid, hipStream_t hs)
{
    if (D == 64) kv4_write_kernel<DT, 64><<<grid, kThreads, 0, hs>>>(a);
    else if (D == 128) kv4_write_kernel<DT, 128><<<grid, kThreads, 0, hs>>>(a);
    else kv4_write_kernel<DT, 256><<<grid, kThreads, 0, hs>>>(a);
}
template <int DT>
void launch_read(const CacheArgs& a, int64_t D, uint32_t grid, hipStream_t hs)
{
    if (D == 64) kv4_read_kernel<DT, 64><<<grid, kThreads, 0, hs>>>(a);
    else if (D == 128) kv4_read_kernel<DT, 128><<<grid, kThreads, 0, hs>>>(a);
    else kv4_read_kernel<DT, 256><<<grid, kThreads, 0, hs>>>(a);
}

int check_cache(int64_t T, int64_t heads, int64_t D, int64_t pages)
{
    if (T < 0 || T >= (1 << 24) || heads < 1 || heads > QUICK_KV4_MAX_HEADS || pages < 1 || pages >= (1 << 25))
        return QUICK_ERR_SHAPE;
    return D == 64 || D == 128 || D == 256 ? QUICK_OK : QUICK_ERR_UNSUPPORTED;
}

// Workgroups of a cache kernel; 0: more than a launch holds.
uint32_t cache_grid(int64_t T, int64_t heads, int64_t D)
{
    const int64_t n = ceil_div(T, kThreads / (D / 8)) * heads;
    return n > kMaxGrid ? 0 : (uint32_t)n;
}

}  // namespace

extern "C" int quick_rotary(const void* x, int dtype, int64_t x_token, int64_t x_head, int64_t T, int64_t H, int64_t D,
                            const int32_t* positions, const double* freqs, int64_t R, int interleaved, int inverse,
                            float factor, void* out, int64_t out_token, int64_t out_head, void* stream)
{
    if (dtype < QUICK_F16 || dtype > QUICK_F32) return QUICK_ERR_INVALID_ARG;
    const int64_t limit = (int64_t)1 << 40;
    if (T < 0 || T >= (1 << 24) || H < 1 || H > 65535 || D < 1 || D > kMaxChannels || R < 0 || R > D || R % 2 != 0 ||
        x_token < 0 || x_token >= limit || x_head < 0 || x_head >= limit || out_token < 0 || out_token >= limit ||
        out_head < 0 || out_head >= limit)
        return QUICK_ERR_SHAPE;
    if (T == 0) return QUICK_OK;
    if (!x || !out || !positions || (R && !freqs)) return QUICK_ERR_INVALID_ARG;
    const int64_t es = dtype == QUICK_F32 ? 4 : 2;
    if (!aligned(x, es) || !aligned(out, es) || !aligned(positions, 4) || !aligned(freqs, 8)) return QUICK_ERR_ALIGNMENT;
    RotaryArgs a{(const uint8_t*)x, (uint8_t*)out, positions, freqs, x_token, x_head, out_token, out_head};
    a.H = (int32_t)H;
    a.D = (int32_t)D;
    a.half = (int32_t)(R / 2);
    // 16 bytes at a time where both places of a pair, the channels that stay and every head begin at a multiple
    const int64_t v = 16 / es;
    const bool wide = aligned(x, 16) && aligned(out, 16) && x_token % v == 0 && x_head % v == 0 && out_token % v == 0 &&
                      out_head % v == 0 && D % v == 0 && (R / 2) % v == 0;
    const int64_t vec = wide ? v : 1;
    a.turning = (int32_t)(R / 2 / vec);
    a.pieces = a.turning + (int32_t)((D - R) / vec);
    a.copy = x != out;
    a.together = std::max(1, kThreads / a.pieces);
    // enough workgroups for the chip from few tokens, whole rounds of a workgroup's threads each
    const int64_t rounds = ceil_div(H, a.together);
    const int64_t parts = std::max<int64_t>(1, std::min(rounds, ceil_div(512, T)));
    a.heads = (int32_t)(ceil_div(rounds, parts) * a.together);
    a.parts = (uint32_t)ceil_div(H, a.heads);
    a.factor = factor;
    a.sign = inverse ? -1.0f : 1.0f;
    if (T * a.parts > kMaxGrid) {
        a.heads = (int32_t)H;
        a.parts = 1;
        if (T > kMaxGrid) return QUICK_ERR_SHAPE;
    }
    hipStream_t hs = (hipStream_t)stream;
    (void)hipGetLastError();
    if (dtype == QUICK_F16) {
        if (wide) launch_rotary<QUICK_F16, 8>(a, T, interleaved != 0, hs);
        else launch_rotary<QUICK_F16, 1>(a, T, interleaved != 0, hs);
    } else if (dtype == QUICK_BF16) {
        if (wide) launch_rotary<QUICK_BF16, 8>(a, T, interleaved != 0, hs);
        else launch_rotary<QUICK_BF16, 1>(a, T, interleaved != 0, hs);
    } else {
        if (wide) launch_rotary<QUICK_F32, 4>(a, T, interleaved != 0, hs);
        else launch_rotary<QUICK_F32, 1>(a, T, interleaved != 0, hs);
    }
    return launched();
}

extern "C" int quick_kv4_write(const void* k, const void* v, int dtype, int64_t k_token, int64_t k_head, int64_t v_token,
                               int64_t v_head, const int32_t* slots, int64_t T, int64_t heads, int64_t D, void* cache,
                               int64_t pages, void* stream)
{
    if (dtype != QUICK_F16 && dtype != QUICK_BF16) return QUICK_ERR_INVALID_ARG;
    const int st = check_cache(T, heads, D, pages);
    if (st) return st;
    const int64_t limit = (int64_t)1 << 40;
    for (int64_t s : {k_token, k_head, v_token, v_head})
        if (s < 0 || s >= limit) return QUICK_ERR_SHAPE;
    if (T == 0) return QUICK_OK;
    if (!k || !v || !slots || !cache) return QUICK_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4) || !aligned(cache, 16) || k_token % 8 || k_head % 8 ||
        v_token % 8 || v_head % 8)
        return QUICK_ERR_ALIGNMENT;
    CacheArgs a{};
    a.k = (const uint8_t*)k;
    a.v = (const uint8_t*)v;
    a.k_token = k_token;
    a.k_head = k_head;
    a.v_token = v_token;
    a.v_head = v_head;
    a.slots = slots;
    a.cache = (uint8_t*)cache;
    a.T = T;
    a.slots_end = pages * kPage;
    a.heads = (int32_t)heads;
    const uint32_t grid = cache_grid(T, heads, D);
    if (!grid) return QUICK_ERR_SHAPE;
    (void)hipGetLastError();
    if (dtype == QUICK_F16) launch_write<QUICK_F16>(a, D, grid, (hipStream_t)stream);
    else launch_write<QUICK_BF16>(a, D, grid, (hipStream_t)stream);
    return launched();
}

extern "C" int quick_kv4_read(const void* cache, int64_t pages, const int32_t* slots, int64_t T, int64_t heads, int64_t D,
                              int dtype, void* k, void* v, void* stream)
{
    if (dtype < QUICK_F16 || dtype > QUICK_F32) return QUICK_ERR_INVALID_ARG;
    const int st = check_cache(T, heads, D, pages);
    if (st) return st;
    if (T == 0 || (!k && !v)) return QUICK_OK;
    if (!slots || !cache) return QUICK_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4) || !aligned(cache, 16)) return QUICK_ERR_ALIGNMENT;
    CacheArgs a{};
    a.k_out = (uint8_t*)k;
    a.v_out = (uint8_t*)v;
    a.slots = slots;
    a.cache = (uint8_t*)const_cast<void*>(cache);
    a.T = T;
    a.slots_end = pages * kPage;
    a.heads = (int32_t)heads;
    const uint32_t grid = cache_grid(T, heads, D);
    if (!grid) return QUICK_ERR_SHAPE;
    (void)hipGetLastError();
    if (dtype == QUICK_F16) launch_read<QUICK_F16>(a, D, grid, (hipStream_t)stream);
    else if (dtype == QUICK_BF16) launch_read<QUICK_BF16>(a, D, grid, (hipStream_t)stream);
    else launch_read<QUICK_F32>(a, D, grid, (hipStream_t)stream);
    return launched();
}
