// Device helpers shared by the kernels of quick_mx.hip, quick_mx_gemm.hip and
// quick_moe.hip: vector types, raw buffers, and 16-bit conversions.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "quick_mx.h"

namespace quick {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u2_t __attribute__((ext_vector_type(2)));
typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef __bf16 b2_t __attribute__((ext_vector_type(2)));

template <class To, class From>
__device__ __forceinline__ To bits_as(const From& v)
{
    static_assert(sizeof(To) == sizeof(From), "size mismatch");
    return __builtin_bit_cast(To, v);
}

// Raw buffers: a wave-uniform descriptor (base, byte size), a per-lane byte
// offset and a wave-uniform one.  What lies at or beyond the size by the
// per-lane offset reads as zero, word by word; the uniform offset is added
// behind that check (by the compiler's documentation), so a read that may
// pass the end has all of its offset in the lane.
typedef __amdgpu_buffer_rsrc_t rsrc_t;

__device__ __forceinline__ rsrc_t make_rsrc(const void* p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ u4_t ld128(rsrc_t r, uint32_t voff, uint32_t soff)
{
    return bits_as<u4_t>(__builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 0));
}
__device__ __forceinline__ uint32_t ld32(rsrc_t r, uint32_t voff, uint32_t soff)
{
    return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, voff, soff, 0);
}
__device__ __forceinline__ uint32_t ld8(rsrc_t r, uint32_t voff, uint32_t soff)
{
    return (uint32_t)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, voff, soff, 0);
}

// A value that is the same in every lane, kept in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p)
{
    const uint64_t v = (uint64_t)p;
    return (const uint8_t*)((uint64_t)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v));
}

// 16-bit types in memory, by QUICK_F16 / QUICK_BF16.
template <int DT>
__device__ __forceinline__ float from16(uint16_t v)
{
    if constexpr (DT == QUICK_F16) return (float)bits_as<_Float16>(v);
    else return bits_as<float>((uint32_t)v << 16);
}
// Round to nearest even.
template <int DT>
__device__ __forceinline__ uint16_t to16(float v)
{
    if constexpr (DT == QUICK_F16) return bits_as<uint16_t>((_Float16)v);
    else return bits_as<uint16_t>((__bf16)v);
}
template <int DT>
__device__ __forceinline__ uint32_t to16x2(float a, float b)
{
    return (uint32_t)to16<DT>(a) | (uint32_t)to16<DT>(b) << 16;
}

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Status after a launch.
inline int launched() { return hipGetLastError() == hipSuccess ? QUICK_OK : QUICK_ERR_HIP; }

}  // namespace quick
