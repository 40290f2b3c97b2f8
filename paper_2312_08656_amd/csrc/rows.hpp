// What the kernels that work row by row share: units of 8 columns at any element's alignment, and sums and maxima over the lanes that share a row.
#pragma once

#include <type_traits>

#include "mx.hpp"

namespace maxk {

constexpr int kRowUnit = 8;  // columns a lane takes at a time

// to the nearest stored value, halfway cases to even; NaN stays NaN
template <int VT>
__device__ __forceinline__ value_store_t<VT> round_value(float x)
{
    if constexpr (VT == MAXK_VALUE_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    else return narrow_value<VT>(x);
}
template <int VT>
__device__ __forceinline__ float rounded(float x) { return widen_value<VT>(round_value<VT>(x)); }

// 16 bytes from any address: one access of the memory pipeline, which takes any alignment (a row's start is only an element's)
__device__ __forceinline__ uint4 read16(const void* p)
{
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
__device__ __forceinline__ void write16(void* p, uint4 v) { __builtin_memcpy(p, &v, 16); }

template <int VT>
struct RawUnit { uint4 w[VT == MAXK_VALUE_F32 ? 2 : 1]; };

template <int VT>
__device__ __forceinline__ float raw_value(const RawUnit<VT>& u, int j)  // j: a constant once unrolled
{
    const uint4 v = u.w[VT == MAXK_VALUE_F32 ? j / 4 : 0];
    if constexpr (VT == MAXK_VALUE_F32) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        return __uint_as_float(w[j % 4]);
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (VT == MAXK_VALUE_BF16) return __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
        else return widen_value<VT>((uint16_t)(w[j / 2] >> (16 * (j & 1))));
    }
}

template <int VT>
__device__ __forceinline__ RawUnit<VT> whole_unit(const value_store_t<VT>* p)
{
    RawUnit<VT> u;
    u.w[0] = read16(p);
    if constexpr (VT == MAXK_VALUE_F32) u.w[1] = read16(p + 4);
    return u;
}
template <int VT>
__device__ __forceinline__ void store_whole_unit(value_store_t<VT>* p, const float (&x)[kRowUnit])
{
    value_store_t<VT> v[kRowUnit];
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j) v[j] = round_value<VT>(x[j]);
    __builtin_memcpy(p, v, sizeof(v));
}

// the same past the caches, to an address of whole 16 bytes
template <int VT>
__device__ __forceinline__ void store_unit_once(value_store_t<VT>* p, const float (&x)[kRowUnit])
{
    typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
    value_store_t<VT> v[kRowUnit];
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j) v[j] = round_value<VT>(x[j]);
    u32x4v w[VT == MAXK_VALUE_F32 ? 2 : 1];
    __builtin_memcpy(&w, v, sizeof(v));
    __builtin_nontemporal_store(w[0], reinterpret_cast<u32x4v*>(p));
    if constexpr (VT == MAXK_VALUE_F32) __builtin_nontemporal_store(w[1], reinterpret_cast<u32x4v*>(p + 4));
}

// Unit at p, of which `valid` columns (less than 1: none) belong to the row.  What lies behind a row is read where it belongs to the matrix, which ends at
// `end`.  (Values are taken out apart from it: a lane's units are under way together.)
template <int VT>
__device__ __forceinline__ RawUnit<VT> fetch_row_unit(const value_store_t<VT>* p, int valid, const value_store_t<VT>* end)
{
    RawUnit<VT> u = {};
    const bool some = valid > 0, whole = p + kRowUnit <= end;
    if (some && whole) u = whole_unit<VT>(p);
    if (some && !whole) {  // the matrix's last columns
        value_store_t<VT> v[kRowUnit];
#pragma unroll
        for (int j = 0; j < kRowUnit; ++j) v[j] = j < valid ? p[j] : value_store_t<VT>(0);
        __builtin_memcpy(&u, v, sizeof(v));
    }
    return u;
}
// its values, `fill` in the columns that do not belong to the row
template <int VT>
__device__ __forceinline__ void unit_values(const RawUnit<VT>& u, int valid, float fill, float (&x)[kRowUnit])
{
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j) x[j] = j < valid ? raw_value<VT>(u, j) : fill;
}
template <int VT>
__device__ __forceinline__ void load_row_unit(const value_store_t<VT>* p, int valid, const value_store_t<VT>* end, float fill, float (&x)[kRowUnit])
{
    unit_values<VT>(fetch_row_unit<VT>(p, valid, end), valid, fill, x);
}

// A lane's unit at p, of which `valid` elements (less than 1: none) belong to the row
template <typename T>
__device__ __forceinline__ void store_values(T* p, int valid, const T (&v)[kRowUnit])
{
    if (valid >= kRowUnit) {
        __builtin_memcpy(p, v, sizeof(v));
        return;
    }
    // a row's last columns: four, two and one of them
    const bool four = valid >= 4, two = valid > 0 && (valid & 2), one = valid > 0 && (valid & 1);
    if (four) __builtin_memcpy(p, v, 4 * sizeof(v[0]));
    const T v0 = v[0], v1 = v[1], v2 = v[2], v4 = v[4], v5 = v[5], v6 = v[6];  // (values: of two places in an array one would be taken in memory)
    const T a = four ? v4 : v0, b = four ? v5 : v1, c = four ? v6 : v2;
    const int at = four ? 4 : 0;
    if (two) {
        const T pair[2] = {a, b};
        __builtin_memcpy(p + at, pair, sizeof(pair));
    }
    if (one) p[two ? at + 2 : at] = two ? c : a;
}
template <int VT>
__device__ __forceinline__ void store_row_unit(value_store_t<VT>* p, int valid, const float (&x)[kRowUnit])
{
    value_store_t<VT> v[kRowUnit];
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j) v[j] = round_value<VT>(x[j]);
    store_values(p, valid, v);
}

// ---- over the L lanes (a power of two, up to 64) that share a row: every lane has the result, the same bits ----

template <int CONTROL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CONTROL, 0xF, 0xF, true); }
__device__ __forceinline__ uint32_t xor_lane(uint32_t x, std::integral_constant<int, 1>) { return dpp<0xB1>(x); }   // quad_perm [1,0,3,2]
__device__ __forceinline__ uint32_t xor_lane(uint32_t x, std::integral_constant<int, 2>) { return dpp<0x4E>(x); }   // quad_perm [2,3,0,1]
// (of lanes that agree in each group of 4, and of 8)
__device__ __forceinline__ uint32_t xor_lane(uint32_t x, std::integral_constant<int, 4>) { return dpp<0x141>(x); }  // row_half_mirror
__device__ __forceinline__ uint32_t xor_lane(uint32_t x, std::integral_constant<int, 8>) { return dpp<0x140>(x); }  // row_mirror
__device__ __forceinline__ uint32_t xor_lane(uint32_t x, std::integral_constant<int, 16>)
{
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return (threadIdx.x & 16) ? r[0] : r[1];
}
__device__ __forceinline__ uint32_t xor_lane(uint32_t x, std::integral_constant<int, 32>)
{
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return (threadIdx.x & 32) ? r[0] : r[1];
}

template <int S, typename T>
__device__ __forceinline__ T other_lane(T x)  // of lane ^ S, in a reduction that goes S = 1, 2, 4, ...
{
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, xor_lane(__builtin_bit_cast(uint32_t, x), std::integral_constant<int, S>{}));
    else {
        const uint2 w = __builtin_bit_cast(uint2, x);
        return __builtin_bit_cast(T, make_uint2(xor_lane(w.x, std::integral_constant<int, S>{}), xor_lane(w.y, std::integral_constant<int, S>{})));
    }
}

template <int L, typename T, typename F>
__device__ __forceinline__ T over_lanes(T x, F&& f)
{
    if constexpr (L > 1) x = f(x, other_lane<1>(x));
    if constexpr (L > 2) x = f(x, other_lane<2>(x));
    if constexpr (L > 4) x = f(x, other_lane<4>(x));
    if constexpr (L > 8) x = f(x, other_lane<8>(x));
    if constexpr (L > 16) x = f(x, other_lane<16>(x));
    if constexpr (L > 32) x = f(x, other_lane<32>(x));
    return x;
}

constexpr auto kAdd = [](auto a, auto b) { return a + b; };

// Sum over the L lanes of a row, L up to 64 within a wavefront, or a workgroup of L threads (`room`: L / 64 values in LDS, free again behind the next barrier)
template <int L, typename T>
__device__ __forceinline__ T row_sum(T x, T* room)
{
    if constexpr (L <= kWave) return over_lanes<L>(x, kAdd);
    else {
        x = over_lanes<kWave>(x, kAdd);
        if ((threadIdx.x & 63) == 0) room[threadIdx.x / kWave] = x;
        __syncthreads();
        T sum = room[0];
#pragma unroll
        for (int i = 1; i < L / kWave; ++i) sum += room[i];
        return sum;
    }
}

}  // namespace maxk
