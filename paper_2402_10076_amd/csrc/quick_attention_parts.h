// What the kernels of quick_attention.hip and quick_attention_tiled.hip share:
// arguments, the softmax's reference, and codes as operands.
#pragma once
#include "quick_attention_plan.h"
#include "quick_device.h"
#include "quick_kv4.h"

namespace quick {

typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef float f16_t __attribute__((ext_vector_type(16)));

// Keeps a seldom taken branch a branch: the compiler would rather work both
// sides out and select.
__device__ __forceinline__ void seldom() { asm volatile("" ::); }
// v, of which the compiler then knows nothing: addresses made of it are worked out
// where they are used and hold no registers through a loop before that.
__device__ __forceinline__ int late(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// Softmax weights are 2^(s - m), m within a reference of the scores seen so
// far: set kLift below their largest, and again only when one passes it by
// kRoom, so that most pages need no exchange between lanes and no rescaling.
// Of f16 weights are then at most 2^14, which it holds, and those down to 2^-30
// of the largest still count in it.  Bf16 holds far smaller ones, and values near
// binary32's end, whose products with weights above 1 it could not: there they
// are at most 1, the first largest 2^-8.
// Weights are rounded to the type, as the matrix instruction takes its operands,
// and their sum is not: half a step of each weight more in the result, and on the
// whole a tenth to a third more error than with weights of 32 bits (float16 2.3e-4
// to 2.7e-4 relative, 2.0e-4 to 2.1e-4 so; bfloat16 2.0e-3 to 2.1e-3, 1.6e-3).
template <int DT>
constexpr float kRoom = DT == QUICK_F16 ? 14.0f : 0.0f;
template <int DT>
constexpr float kLift = kRoom<DT> - 8.0f;
constexpr float kNothing = -3.4028234663852886e38f;   // a reference before any score (the least number)

// A column's reference.  A weight's exponent is fma(score, scale, -m), rounded
// once, so it is the same function of the score for every token, whatever m is,
// and whether one passes kRoom is asked of that value itself.  But m, a binary32
// number, comes no nearer to a score than half its last place.  Where one is to
// pass kFar (whose last place is 2^-3) the pages are gone through again in a form
// of the loop for far scores: it takes them less `base`, the column's largest when
// its reference was set, with m = -kLift.  (base is zero otherwise.)  In one form
// for both a base cost 2 to 5 % of calls of 64 and of 256 channels.
constexpr float kFar = 1048576.0f;
struct Reference {
    float m, base;

    // To the column's largest score, if its weight has passed the room.  Returns what the sums so far are multiplied
    // by.  Without FAR away is set where that needs a base.
    template <int DT, bool FAR>
    __device__ __forceinline__ float raise(float top, float scale, bool& away)
    {
        const bool up = fmaf(FAR ? top - base : top, scale, -m) > kRoom<DT>;
        const float near = fmaf(top, scale, -kLift<DT>);
        const bool far = fabsf(near) > kFar;
        Reference to = *this;
        if (up) to = FAR && far ? Reference{-kLift<DT>, top} : Reference{near, 0.0f};
        const float f = __builtin_amdgcn_exp2f(FAR ? above(to, scale) : m - to.m);
        *this = to;
        away |= !FAR && up && far;
        return f;
    }
    // How far this one lies above another.
    __device__ __forceinline__ float above(const Reference& o, float scale) const { return fmaf(base - o.base, scale, m - o.m); }
    // Logarithm of a sum of weights.
    __device__ __forceinline__ float log_sum(float l, float scale) const
    {
        return l == 0 ? -INFINITY : (fmaf(base, scale, m) + __log2f(l)) * 0.69314718055994531f;
    }
};
constexpr Reference kNoReference{kNothing, 0.0f};
// The forms of a loop over pages.
struct Near {
    static constexpr bool far = false;
};
struct Far {
    static constexpr bool far = true;
};

struct AttnArgs {
    AttnShape s;
    const uint8_t* q;
    const uint8_t* cache;
    const int32_t* table;
    uint8_t* out;
    float* lse;
    float* part;          // [2 * workers][columns][D] sums of a part of an item's pages
    f4_t* part_ref;       // [2 * workers][columns] their references (m, base) and sums of weights
    int32_t* joins;       // [workers][8] the item that a worker leaves unfinished
    int64_t q_token, q_head;
    int32_t pages, workers;
    int32_t group_inv;    // c / group == c * group_inv >> 16 for c < 128
    int32_t whole;        // a worker takes an item and no more; nothing to join
    int32_t ranked;       // ... the longest sequences first
    float scale;          // of the scores times log2(e), without its sign
    uint32_t q_sign;      // changes q's sign where the scale is negative
};

// What the joining kernel is told of an item that a worker leaves unfinished.
__device__ __forceinline__ void set_join(int (&join)[8], const Walk& w, const Tile& t, int columns, int take, int slot)
{
    const int rest = t.cost - take;
    join[0] = 1 + (int)((rest + w.share - 1) / w.share);    // parts
    join[1] = slot;
    join[2] = w.j * columns;
    join[3] = t.columns;
    join[4] = t.first;
    join[5] = w.h;
}

// Two values of byte BYTE of a word of codes times the scale, as 16-bit pair.
template <int DT, int BYTE>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, float scale)
{
    if constexpr (DT == QUICK_F16) return bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, BYTE));
    else return bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, BYTE));
}
template <int DT>
__device__ __forceinline__ u4_t code_words(uint32_t w, float scale)
{
    return u4_t{code_pair<DT, 0>(w, scale), code_pair<DT, 1>(w, scale), code_pair<DT, 2>(w, scale),
                code_pair<DT, 3>(w, scale)};
}
// Two values rounded to nearest even, as a pair.
template <int DT>
__device__ __forceinline__ uint32_t pair16(float a, float b)
{
    typedef float f2_t __attribute__((ext_vector_type(2)));
    if constexpr (DT == QUICK_F16) return bits_as<uint32_t>(__builtin_convertvector((f2_t{a, b}), h2_t));
    else return bits_as<uint32_t>(__builtin_convertvector((f2_t{a, b}), b2_t));
}
// The scale that byte i of a word of scales stands for, for code_pair: its byte is
// the exponent.  The conversion reads nothing else of a scale (tried with every
// code, exponent and 64 patterns of the other bits), so those hold what comes.
__device__ __forceinline__ float scale_of(uint32_t w, int i) { return bits_as<float>(i == 3 ? w >> 1 : w << (23 - 8 * i)); }
// Bits lo <= i < hi of a word, any lo and hi.
__device__ __forceinline__ uint32_t bits_between(int lo, int hi)
{
    const uint32_t below = hi >= 32 ? ~0u : hi <= 0 ? 0u : (1u << hi) - 1;
    return below & (lo >= 32 ? 0u : lo <= 0 ? ~0u : ~0u << lo);
}
// v where bit i of a word is set, else minus infinity.
__device__ __forceinline__ float where_bit(float v, uint32_t bits, int i)
{
    const uint32_t m = (uint32_t)((int32_t)(bits << (31 - i)) >> 31);
    return bits_as<float>((bits_as<uint32_t>(v) & m) | (0xFF800000u & ~m));
}
template <int DT>
__device__ __forceinline__ f4_t mfma16(u4_t a, u4_t b, f4_t c)
{
    if constexpr (DT == QUICK_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(bits_as<h8_t>(a), bits_as<h8_t>(b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(bits_as<b8_t>(a), bits_as<b8_t>(b), c, 0, 0, 0);
}
// Nonzero bits 7, 15, 23, 31 where a byte of scales is beyond the type (its
// block would be infinite or NaN): above 140 with f16, 252 with bf16.
template <int DT>
__device__ __forceinline__ uint32_t beyond(uint32_t w)
{
    return ((w & 0x7F7F7F7Fu) + (DT == QUICK_F16 ? 0x73737373u : 0x03030303u)) & w & 0x80808080u;
}
// 255 where a byte has its bit 7 of those.
__device__ __forceinline__ uint32_t whole_bytes(uint32_t bits) { return (bits << 1) - (bits >> 7); }

// Eight sums of a column to its row of out.
template <int DT>
__device__ __forceinline__ u4_t rounded8(const float (&v)[8], float f)
{
    return u4_t{pair16<DT>(v[0] * f, v[1] * f), pair16<DT>(v[2] * f, v[3] * f), pair16<DT>(v[4] * f, v[5] * f),
                pair16<DT>(v[6] * f, v[7] * f)};
}

// Operands of two tiles of 16 channels from the same byte of eight tokens: w
// holds four tokens of one 16 (a) and of the next (b), eight channels (W == 4)
// or four of each; the byte's two channels go to the two operands.
template <int DT, int W, int Y>
__device__ __forceinline__ void value_words(const uint32_t (&a)[W], const uint32_t (&b)[W], const float (&sa)[4],
                                            const float (&sb)[4], u4_t& lo, u4_t& hi)
{
    uint32_t p[8];
    if constexpr (W == 4) {
#pragma unroll
        for (int e = 0; e < 4; e++) {
            p[e] = code_pair<DT, Y>(a[e], sa[e]);
            p[4 + e] = code_pair<DT, Y>(b[e], sb[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 2; e++) {
            p[2 * e] = code_pair<DT, Y>(a[e], sa[2 * e]);
            p[2 * e + 1] = code_pair<DT, Y + 2>(a[e], sa[2 * e + 1]);
            p[4 + 2 * e] = code_pair<DT, Y>(b[e], sb[2 * e]);
            p[5 + 2 * e] = code_pair<DT, Y + 2>(b[e], sb[2 * e + 1]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        lo[i] = __builtin_amdgcn_perm(p[2 * i + 1], p[2 * i], 0x05040100u);
        hi[i] = __builtin_amdgcn_perm(p[2 * i + 1], p[2 * i], 0x07060302u);
    }
}

// The tiled kernel: workgroups that the chip holds (two a compute unit, one of 256
// columns or of 256 channels, whose registers leave a wave a SIMD; of 2 sequences
// of 4096 tokens the last 2048 as queries, 8 cache heads of 256 read by 4 each: 662
// us, 698 with twice as many), least share, and what an item costs beside its pages.
constexpr int tiled_workers(int64_t D, int64_t columns) { return D > 128 || columns > 128 ? 256 : 512; }
constexpr int kTiledShare = 10, kTiledStart = 6;
void launch_tiled_attention(const AttnArgs& a, int dtype, int64_t D, int columns, hipStream_t hs);

}  // namespace quick
