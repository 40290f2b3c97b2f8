// Y = X W^T + b for few rows of X in 32 or 16 bits and W in 4 (include/maxk.h): one node's or token's features through a layer.
//
// Bound by the reading of W, 17 bytes for 32 columns of a row; the matrix instructions take W as it decodes, exact in bf16, and X in bf16 parts that
// add up to it (three of fp32, two of fp16), so that products are exact, and 1 to 16 rows of X cost the same instructions.  A wavefront has 16 TILES rows of W and 512
// columns at a time: a lane has whole blocks of one row (its 16 bytes are one load), and the columns that a matrix instruction adds up are dealt to lanes in
// the same order on both sides.  The wavefronts of a workgroup share out the columns and are joined in LDS.
#include "mx_parts.hpp"
#include "rows.hpp"

namespace maxk {
namespace {

typedef float f32x4v __attribute__((ext_vector_type(4)));

constexpr int kRows = 16;      // of X a pass
constexpr int kBlocks = 16;    // blocks of a row of W that a wavefront has at a time: four a lane, four lanes a row
constexpr int kMostWaves = 8;  // of a workgroup, each with a share of the columns

template <int VT> constexpr int kParts = VT == MAXK_VALUE_F32 ? 3 : VT == MAXK_VALUE_BF16 ? 1 : 2;

// 8 columns of X in bf16 parts
template <int VT>
__device__ __forceinline__ void x_parts(const float (&x)[kRowUnit], bf16x8 (&part)[kParts<VT>])
{
    float cut[kRowUnit][kParts<VT>];
#pragma unroll
    for (int j = 0; j < kRowUnit; ++j) split<kParts<VT>>(x[j], cut[j]);
#pragma unroll
    for (int p = 0; p < kParts<VT>; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = uppers(cut[2 * j][p], cut[2 * j + 1][p]);
        part[p] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
    }
}

template <int VT, int TILES>
__global__ void __launch_bounds__(kMostWaves* kWave) matvec_kernel(const value_store_t<VT>* X, int64_t N, const uint8_t* codes, const uint8_t* scales, int din,
                                                                   int dout, const float* bias, void* Y, int y_type)
{
    __shared__ f32x4v sums[kMostWaves - 1][TILES][kWave];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    const int nb = mx_blocks(din), row16 = lane & 15, quarter = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.y * kRows;
    const int64_t n = min(n0 + row16, N - 1);  // (lanes behind the last row of X repeat it: what they add up is not stored)
    const int64_t o0 = (int64_t)blockIdx.x * (16 * TILES);
    const value_store_t<VT>*x = X + n * din, *x_end = X + N * din;
    f32x4v sum[TILES];
    const uint8_t *c[TILES], *s[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        sum[t] = f32x4v{0.f, 0.f, 0.f, 0.f};
        const int64_t o = min(o0 + t * 16 + row16, (int64_t)dout - 1);
        c[t] = codes + o * nb * 16;
        s[t] = scales + o * nb;
    }
    for (int b0 = wave * kBlocks; b0 < nb; b0 += waves * kBlocks) {
        uint4 code[TILES][4];
        float unit[TILES][4];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int b = b0 + i * 4 + quarter;
                code[t][i] = make_uint4(0, 0, 0, 0);
                unit[t][i] = 1.f;
                if (b < nb) {
                    code[t][i] = *reinterpret_cast<const uint4*>(c[t] + b * 16);
                    unit[t][i] = mx_scale(s[t][b]);
                }
            }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int col = (b0 + i * 4 + quarter) * kMxBlock + q * kRowUnit;
                float v[kRowUnit];
                load_row_unit<VT>(x + col, din - col, x_end, 0.f, v);
                bf16x8 part[kParts<VT>];
                x_parts<VT>(v, part);
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    const uint32_t w[4] = {code[t][i].x, code[t][i].y, code[t][i].z, code[t][i].w};
                    uint4 a;
                    a.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[q], unit[t][i], 0));
                    a.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[q], unit[t][i], 1));
                    a.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[q], unit[t][i], 2));
                    a.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[q], unit[t][i], 3));
#pragma unroll
                    for (int p = 0; p < kParts<VT>; ++p)
                        sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), part[p], sum[t], 0, 0, 0);
                }
            }
    }
    if (wave > 0) {
#pragma unroll
        for (int t = 0; t < TILES; ++t) sums[wave - 1][t][lane] = sum[t];
    }
    __syncthreads();
    if (wave > 0 || n0 + row16 >= N) return;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        for (int w = 1; w < waves; ++w) sum[t] += sums[w - 1][t][lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t o = o0 + t * 16 + quarter * 4 + j;
            if (o >= dout) continue;
            const float y = sum[t][j] + (bias ? bias[o] : 0.f);
            const int64_t at = (n0 + row16) * dout + o;
            if (y_type == MAXK_VALUE_F32) ((float*)Y)[at] = y;
            else if (y_type == MAXK_VALUE_BF16) ((uint16_t*)Y)[at] = round_value<MAXK_VALUE_BF16>(y);
            else ((uint16_t*)Y)[at] = round_value<MAXK_VALUE_F16>(y);
        }
    }
}

template <int VT, int TILES>
maxk_status matvec(const void* X, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int y_type, hipStream_t s)
{
    const int64_t passes = (N + kRows - 1) / kRows;
    if (passes > 65535) return MAXK_UNSUPPORTED;
    const int shares = (mx_blocks(din) + kBlocks - 1) / kBlocks, waves = std::min(shares, kMostWaves);
    hipLaunchKernelGGL((matvec_kernel<VT, TILES>), dim3((unsigned)((dout + 16 * TILES - 1) / (16 * TILES)), (unsigned)passes), dim3(waves * kWave), 0, s,
                       (const value_store_t<VT>*)X, N, W.codes, W.scales, din, dout, bias, Y, y_type);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

}  // namespace

maxk_status launch_mx_matvec(const void* X, int value_type, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int y_type,
                             hipStream_t s)
{
    if (value_type == MAXK_VALUE_F32) return matvec<MAXK_VALUE_F32, 1>(X, N, W, din, dout, bias, Y, y_type, s);
    if (value_type == MAXK_VALUE_BF16) return matvec<MAXK_VALUE_BF16, 1>(X, N, W, din, dout, bias, Y, y_type, s);
    return matvec<MAXK_VALUE_F16, 1>(X, N, W, din, dout, bias, Y, y_type, s);
}

}  // namespace maxk
