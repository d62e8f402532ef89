// Places in a page of the 4-bit cache (the layout of quick_attention.h): plain
// arithmetic that writing, reading and attention share.
#pragma once
#include <cstdint>

#include "quick_attention.h"

namespace quick {

constexpr int kPage = QUICK_KV4_PAGE;

// Bytes of a page's head, and where its four parts begin.
template <int D>
struct Kv4 {
    static constexpr int kKeys = 0, kKeyScales = 32 * D, kValues = 34 * D, kValueScales = 66 * D, kBytes = 68 * D;
    static constexpr int kLane = (D < 128 ? D : 128) / 16;   // channels of a lane in 128 (or 64) of values

    // The four bytes of channels 8 p .. 8 p + 7 of token t's key.
    static constexpr __host__ __device__ int key(int t, int p) { return kKeys + t * (D / 2) + p * 4; }
    // Of its value: four bytes, or (D == 64) two times two, kLane * 2 apart.
    static constexpr __host__ __device__ int value(int t, int p)
    {
        return kValues + (p / 16) * 4096 + (t / 4) * (32 * kLane) +
               ((p % 16) * 8 / kLane * 4 + t % 4) * (kLane / 2);
    }
    static constexpr __host__ __device__ int key_scale(int t, int b) { return kKeyScales + b * 64 + t % 16 * 4 + t / 16; }
    static constexpr __host__ __device__ int value_scale(int t, int b)
    {
        return kValueScales + b * 64 + t % 16 / 4 * 16 + t / 16 * 4 + t % 4;
    }
};

}  // namespace quick
