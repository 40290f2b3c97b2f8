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

// the largest of four neighbouring lanes
__device__ __forceinline__ uint32_t max_of_four(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));   // quad_perm [1,0,3,2]
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));  // quad_perm [2,3,0,1]
}

// A lane's 8 columns of a block that four neighbouring lanes share: their codes to `codes` (8 or 4 bytes); returns the block's scale byte
template <int FMT>
__device__ __forceinline__ uint32_t encode_unit(const float (&x)[8], uint8_t* codes)
{
    uint32_t top = 0;  // patterns of magnitudes are in the magnitudes' order, Inf and NaN above all others
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
    uint32_t s = max_of_four(top) >> 23;
    const bool finite = s != 255u;
    if constexpr (FMT == MAXK_MX_8) {
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // adding 1.5 * 2^23 rounds to a whole number, halfway cases to even, and leaves it in the low byte
                const float y = __builtin_amdgcn_ldexpf(x[4 * h + j], 133 - (int)s);
                q[j] = __float_as_uint(__builtin_amdgcn_fmed3f(y, -127.f, 127.f) + 0x1.8p23f);
            }
            const uint32_t low = __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u), high = __builtin_amdgcn_perm(q[3], q[2], 0x04000C0Cu);
            w[h] = finite ? low | high : 0u;
        }
        *reinterpret_cast<uint2*>(codes) = make_uint2(w[0], w[1]);
    } else {
        if (finite) s = s > 2u ? s - 2u : 0u;
        const float scale = mx_scale(s);
        uint32_t w = 0;  // the conversion divides by the scale, rounds to nearest even and saturates
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
        *reinterpret_cast<uint32_t*>(codes) = finite ? w : 0u;
    }
    return s;
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
maxk_status launch_mx_matvec(const void* X, int value_type, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int y_type,
                             hipStream_t s);
int64_t mx_weight_grad_workspace(int64_t N, int din, int dout);
maxk_status launch_mx_weight_grad(const MxMatrix& X, int64_t N, int din, int dout, const MxGrad& G, float* dW, float* db, float* workspace,
                                  hipStream_t s);
maxk_status launch_mx_input_grad(const MxGrad& G, int64_t N, const MxMatrix& W, int din, int dout, void* dX, int value_type,
                                 hipStream_t s);

}  // namespace maxk
