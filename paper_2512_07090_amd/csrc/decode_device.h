// Device code that the kernels over caches share: rows to and from registers, sums over the lanes that hold one
// query, and partial results on their way from one workgroup to another.
#pragma once

#include "tf_kernels.h"

namespace tf {

#ifdef __HIPCC__
constexpr float kLowest = -1e30f;  // "no key yet": finite, so differences of two of them are 0
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// eight consecutive elements of a row as floats
__device__ __forceinline__ void load8(const uint16_t* p, float* x)
{
    const uint4 r = *reinterpret_cast<const uint4*>(p);
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float* x)
{
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store_out(uint16_t* p, float v)
{
    const unsigned u = __float_as_uint(v);
    *p = (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);  // round to nearest even
}
__device__ __forceinline__ void store_out(float* p, float v) { *p = v; }

// sum over the four lanes that share lane % 16
__device__ __forceinline__ float wave_group_sum(float v)
{
    const FloatPair a = swap16(v, v);
    v = a.first + a.second;
    const FloatPair b = swap32(v, v);
    return b.first + b.second;
}
__device__ __forceinline__ float wave_group_max(float v)
{
    const FloatPair a = swap16(v, v);
    v = fmaxf(a.first, a.second);
    const FloatPair b = swap32(v, v);
    return fmaxf(b.first, b.second);
}

// Two floats to or from memory past the caches that are not shared between the dies (relaxed, device
// scope): written and read this way, a partial result needs no cache to be written back or
// invalidated on its way from one workgroup to another.
struct Float2 { float x, y; };
__device__ __forceinline__ void put_shared(float* p, Float2 v)
{
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Float2 get_shared(const float* p)
{
    return __builtin_bit_cast(Float2, __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
#endif

}  // namespace tf
