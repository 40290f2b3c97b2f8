// What the gradient kernels of the microscaled operators share: bf16 matrix operands, and gradients cut into exact bf16 parts.
#pragma once

#include "mx.hpp"

namespace maxk {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ void local_fence()  // orders LDS only: loads and stores of memory stay under way
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// the upper halves of two floats
__device__ __forceinline__ uint32_t uppers(float low, float high)
{
    return __builtin_amdgcn_perm(__float_as_uint(high), __float_as_uint(low), 0x07060302u);
}
__device__ __forceinline__ float upper_part(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

// x = sum of its parts, each of at most 8 significant bits (x of 24, 11 or 8)
template <int P>
__device__ __forceinline__ void split(float x, float* part)
{
    part[0] = x;  // (its upper half is what is kept)
    if constexpr (P > 1) part[1] = x - upper_part(x);
    if constexpr (P > 2) part[2] = part[1] - upper_part(part[1]);
}

}  // namespace maxk
