// Quantisation of a block of 32 values that is spread over four lanes, eight
// values each (l, l ^ 1, l ^ 2, l ^ 3).
#pragma once
#include "quick_device.h"

namespace quick {

// The larger of a value and its neighbours' in a group of four lanes.
__device__ __forceinline__ uint32_t max_of_quad(uint32_t v)
{
    // lanes (1,0,3,2), then (2,3,0,1) of each four
    const uint32_t a = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
    return max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x4E, 0xF, 0xF, true));
}

// Scale byte of a block whose largest magnitude has these binary32 bits
// (which order as integers): its exponent less that of the largest code,
// 4 <= 6 < 8; 255 with an infinity or a NaN.
__device__ __forceinline__ uint32_t block_scale(uint32_t amax)
{
    const int e = (int)(amax >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}

// Codes of eight values, the first in the lowest nibble: v * 2^(127 - s),
// exact in binary32 (a power of two; small results that go below the normal
// range would be rounded to code 0 in any case), then to the nearest code.
__device__ __forceinline__ uint32_t block_codes(const float (&v)[8], uint32_t s)
{
    const float k = bits_as<float>((254u - min(s, 253u)) << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * k, v[1] * k, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * k, v[3] * k, 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * k, v[5] * k, 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * k, v[7] * k, 1.0f, 3);
    return s == 255u ? 0u : c;
}

// Eight values of a 16-byte load (DT 16-bit) or of two (f32).
template <int DT>
__device__ __forceinline__ void unpack8(const u4_t (&raw)[DT == QUICK_F32 ? 2 : 1], float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if constexpr (DT == QUICK_F32) v[i] = bits_as<float>(raw[i / 4][i % 4]);
        else v[i] = from16<DT>((uint16_t)(raw[0][i / 2] >> (16 * (i % 2))));
    }
}

__device__ __forceinline__ uint32_t amax8(const float (&v)[8])
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) a = max(a, bits_as<uint32_t>(v[i]) & 0x7FFFFFFFu);
    return a;
}

}  // namespace quick
