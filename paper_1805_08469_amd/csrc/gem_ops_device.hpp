// gem_ops_device.hpp -- device code that the worker's operators share: elements of
// either type, 16-byte vectors of them, and reductions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gemk {

using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

constexpr float kInf = __builtin_inff();
constexpr float kLn2 = 0.693147180559945309417f;
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float load(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float load(const uint16_t* p, int64_t i)
{
    return __uint_as_float(static_cast<uint32_t>(p[i]) << 16);
}

// Two binary32 values rounded to bfloat16 (nearest even), the first in the low half.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    using f32x2 = float __attribute__((ext_vector_type(2)));
    using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

__device__ __forceinline__ void store(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void store(uint16_t* p, int64_t i, float v)
{
    p[i] = static_cast<uint16_t>(bf16_pair(v, v));
}

// 16 bytes of elements.
template <class T> constexpr int kVec = 16 / static_cast<int>(sizeof(T));

__device__ __forceinline__ void unpack(u32x4 v, float (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
}
__device__ __forceinline__ void unpack(u32x4 v, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ u32x4 pack(const float (&x)[4])
{
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}
__device__ __forceinline__ u32x4 pack(const float (&x)[8])
{
    return u32x4{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = __builtin_fmaxf(v, __shfl_xor(v, m));
    return v;
}

}  // namespace gemk
