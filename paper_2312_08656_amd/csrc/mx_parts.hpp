// What the gradient kernels of the microscaled operators share: bf16 matrix operands, and gradients cut into bf16 parts.
#pragma once

#include <type_traits>

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

// x = sum of its parts, each of at most 8 significant bits (x of 24, 11 or 8).  Bits of x below 2^-133, the least that bf16 has, are dropped: an fp32 value of
// 2^-110 or more has none, and a gradient that small is lost in any sum with one that is not.
template <int P>
__device__ __forceinline__ void split(float x, float* part)
{
    part[0] = x;  // (its upper half is what is kept)
    if constexpr (P > 1) part[1] = x - upper_part(x);
    if constexpr (P > 2) part[2] = part[1] - upper_part(part[1]);
}

// Tiles lie in LDS as the rows come, bf16, and are read transposed: a lane's operand is 8 rows of one column, and ds_read_b64_tr_b16 gives
// 16 lanes 4 rows of 16 columns from 32 bytes of each of the rows.  The four rows of a read fall on different banks by the place of their bytes:
// rows are multiples of 128 bytes, byte b of row r lies at b ^ 32 (r % 4).
__device__ __forceinline__ int at_byte(int row, int byte, int pitch) { return row * pitch + (byte ^ (row & 3) << (pitch % 256 ? 5 : 6)); }

typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ s16x4 read_transposed(const uint8_t* p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}

// A lane's operand for a product of 32 x 32 outputs over the 16 rows from `row` (a multiple of 4) on: 8 rows of a column of block `block` of 32
__device__ __forceinline__ bf16x8 transposed_operand(const uint8_t* base, int pitch, int block, int row, int lane)
{
    const int r = (lane >> 5) * 8 + (lane & 15) / 4, byte = (lane >> 4 & 1) * 32 + (lane & 3) * 8;
    const uint8_t* p = base + at_byte(r, byte + (block & 3) * 64, pitch) + block / 4 * 256 + row * pitch;
    const s16x4 low = read_transposed(p), high = read_transposed(p + 4 * pitch);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A buffer in memory whose bounds the hardware minds: what is read past its end is 0, what is written there is dropped.  (offsets of 32 bits)
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int kNowhere = (int)0x80000000;  // an offset past any end
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000);
}

// How dH comes: CBSR by the bytes of a column, dense in 16-byte pieces (V) or element by element
enum Kind { kCbsr1, kCbsr2, kCbsr4, kF32, kF32V, kBf16, kBf16V, kF16, kF16V };
template <int KIND> using column_t = std::conditional_t<KIND == kCbsr1, uint8_t, std::conditional_t<KIND == kCbsr2, uint16_t, uint32_t>>;
__host__ __device__ constexpr int type_of(int kind) { return kind <= kF32V ? MAXK_VALUE_F32 : kind <= kBf16V ? MAXK_VALUE_BF16 : MAXK_VALUE_F16; }
__host__ __device__ constexpr int parts_of(int kind) { return kind <= kF32V ? 3 : kind <= kBf16V ? 1 : 2; }
__host__ __device__ constexpr int piece_of(int kind) { return kind == kF32V ? 4 : kind == kBf16V || kind == kF16V ? 8 : 1; }  // columns

}  // namespace maxk
