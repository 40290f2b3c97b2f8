// Microscaled storage (include/maxk.h): blocks of 32 columns with one power-of-two scale, 8-bit integers or 4-bit floating point.
#pragma once

#include "common.hpp"

namespace maxk {

constexpr int kMxBlock = 32;  // columns that share a scale

__host__ __device__ constexpr int mx_blocks(int dim) { return (dim + kMxBlock - 1) / kMxBlock; }

// 2^(s - 127), s = 255: NaN.  (the subnormal 2^-127 for s = 0)
__device__ __forceinline__ float mx_scale(uint32_t s)
{
    return __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7FC00000u : s << 23);
}

// 2^(s - 133), what a whole step of an 8-bit code is worth (subnormal below s = 7); s = 255: NaN
__device__ __forceinline__ float mx8_unit(uint32_t s)
{
    return __uint_as_float(s >= 7 ? (s == 255 ? 0x7FC00000u : (s - 6) << 23) : 0x00800000u >> (7 - s));
}

// A gradient [N x dout]: dense (sp_index null), or k values a row at distinct columns
struct MxGrad {
    const void* values;
    int value_type;
    const void* sp_index;
    int index_bytes;
    int k;
};

struct MxMatrix {
    const uint8_t* codes;
    const uint8_t* scales;
    int format;
};

maxk_status launch_mx_quantize(const void* X, int value_type, int64_t N, int din, int format, uint8_t* codes, uint8_t* scales,
                               hipStream_t s);
maxk_status launch_mx_dequantize(const MxMatrix& A, int64_t N, int din, void* X, int value_type, hipStream_t s);
maxk_status launch_mx_linear(const MxMatrix& X, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int value_type,
                             hipStream_t s);
int64_t mx_weight_grad_workspace(int64_t N, int din, int dout);
maxk_status launch_mx_weight_grad(const MxMatrix& X, int64_t N, int din, int dout, const MxGrad& G, float* dW, float* db, float* workspace,
                                  hipStream_t s);
maxk_status launch_mx_input_grad(const MxGrad& G, int64_t N, const MxMatrix& W, int din, int dout, void* dX, int value_type,
                                 hipStream_t s);

}  // namespace maxk
