// Microscaled storage written and read (include/maxk.h): X into codes and scales, and back.
#include "mx.hpp"

namespace maxk {
namespace {

__device__ __forceinline__ uint32_t exponent_field(float x) { return (__float_as_uint(x) >> 23) & 255u; }

// nearest 4-bit code of |x| / 2^(s - 127), halfway cases to the even code: in quarters, sizes below 2 lie 2 apart, below 4 4, above 8
__device__ __forceinline__ uint32_t e2m1_code(float x, float inverse)
{
    const float a = fminf(fabsf(x) * inverse, 6.f);
    const uint32_t code = a < 2.f ? (uint32_t)__builtin_rintf(a * 2.f) : a < 4.f ? 2u + (uint32_t)__builtin_rintf(a) : 4u + (uint32_t)__builtin_rintf(a * 0.5f);
    return code | (__float_as_uint(x) >> 31 << 3);
}

// one thread a block
template <int VT>
__global__ void quantize_kernel(const value_store_t<VT>* X, int64_t N, int din, int nb, int format, uint8_t* codes, uint8_t* scales)
{
    const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (at >= N * nb) return;
    const int64_t row = at / nb;
    const int first = (int)(at % nb) * kMxBlock;
    const int n = min(kMxBlock, din - first);
    float amax = 0.f;
    bool finite = true;
    for (int c = 0; c < n; ++c) {
        const float x = widen_value<VT>(X[row * din + first + c]);
        finite = finite && exponent_field(x) != 255u;
        amax = fmaxf(amax, fabsf(x));
    }
    uint32_t s = finite ? exponent_field(amax) : 255u;
    if (format == MAXK_MX_4 && finite) s = s > 2u ? s - 2u : 0u;
    scales[at] = (uint8_t)s;
    for (int c = 0; c < kMxBlock; c += 2) {
        uint32_t code[2] = {0u, 0u};
        for (int j = 0; j < 2; ++j) {
            if (c + j >= n || !finite) continue;
            const float x = widen_value<VT>(X[row * din + first + c + j]);
            if (format == MAXK_MX_8) code[j] = (uint32_t)(int)fminf(fmaxf(__builtin_rintf(ldexpf(x, 133 - (int)s)), -127.f), 127.f) & 255u;
            else code[j] = e2m1_code(ldexpf(x, 127 - (int)s), 1.f);
        }
        if (format == MAXK_MX_8) {
            codes[at * 32 + c] = (uint8_t)code[0];
            codes[at * 32 + c + 1] = (uint8_t)code[1];
        } else {
            codes[at * 16 + c / 2] = (uint8_t)(code[0] | code[1] << 4);
        }
    }
}

template <int VT>
__global__ void dequantize_kernel(const uint8_t* codes, const uint8_t* scales, int format, int64_t N, int din, int nb, value_store_t<VT>* X)
{
    const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (at >= N * din) return;
    const int64_t row = at / din;
    const int col = (int)(at % din);
    const float x = format == MAXK_MX_8 ? mx_value<MAXK_MX_8>(codes, scales, row, col, nb) : mx_value<MAXK_MX_4>(codes, scales, row, col, nb);
    X[at] = narrow_value<VT>(x);
}

}  // namespace

maxk_status launch_mx_quantize(const void* X, int value_type, int64_t N, int din, int format, uint8_t* codes, uint8_t* scales, hipStream_t s)
{
    const int nb = mx_blocks(din);
    const int64_t grid = (N * nb + 255) / 256;
    if (grid > 0x7FFFFFFF) return MAXK_UNSUPPORTED;
#define MAXK_QUANTIZE(VT) \
    hipLaunchKernelGGL((quantize_kernel<VT>), dim3((unsigned)grid), dim3(256), 0, s, (const value_store_t<VT>*)X, N, din, nb, format, codes, scales)
    if (value_type == MAXK_VALUE_F32) MAXK_QUANTIZE(MAXK_VALUE_F32);
    else if (value_type == MAXK_VALUE_BF16) MAXK_QUANTIZE(MAXK_VALUE_BF16);
    else MAXK_QUANTIZE(MAXK_VALUE_F16);
#undef MAXK_QUANTIZE
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

maxk_status launch_mx_dequantize(const MxMatrix& A, int64_t N, int din, void* X, int value_type, hipStream_t s)
{
    const int64_t grid = (N * din + 255) / 256;
    if (grid > 0x7FFFFFFF) return MAXK_UNSUPPORTED;
#define MAXK_DEQUANTIZE(VT)                                                                                                               \
    hipLaunchKernelGGL((dequantize_kernel<VT>), dim3((unsigned)grid), dim3(256), 0, s, A.codes, A.scales, A.format, N, din, mx_blocks(din), \
                       (value_store_t<VT>*)X)
    if (value_type == MAXK_VALUE_F32) MAXK_DEQUANTIZE(MAXK_VALUE_F32);
    else if (value_type == MAXK_VALUE_BF16) MAXK_DEQUANTIZE(MAXK_VALUE_BF16);
    else MAXK_DEQUANTIZE(MAXK_VALUE_F16);
#undef MAXK_DEQUANTIZE
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

}  // namespace maxk
