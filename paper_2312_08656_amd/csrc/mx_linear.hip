// Y = X W^T + b of 4-bit operands (include/maxk.h).
#include "mx.hpp"

namespace maxk {
namespace {

// one thread an output
template <int VT>
__global__ void linear_kernel(MxMatrix X, int64_t N, MxMatrix W, int din, int dout, const float* bias, value_store_t<VT>* Y)
{
    const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (at >= N * dout) return;
    const int64_t row = at / dout;
    const int o = (int)(at % dout), nb = mx_blocks(din);
    float sum = 0.f;
    for (int i = 0; i < din; ++i)
        sum += mx_value<MAXK_MX_4>(X.codes, X.scales, row, i, nb) * mx_value<MAXK_MX_4>(W.codes, W.scales, o, i, nb);
    Y[at] = narrow_value<VT>(bias ? sum + bias[o] : sum);
}

}  // namespace

maxk_status launch_mx_linear(const MxMatrix& X, int64_t N, const MxMatrix& W, int din, int dout, const float* bias, void* Y, int value_type,
                             hipStream_t s)
{
    const int64_t grid = (N * dout + 255) / 256;
    if (grid > 0x7FFFFFFF) return MAXK_UNSUPPORTED;
#define MAXK_LINEAR(VT) \
    hipLaunchKernelGGL((linear_kernel<VT>), dim3((unsigned)grid), dim3(256), 0, s, X, N, W, din, dout, bias, (value_store_t<VT>*)Y)
    if (value_type == MAXK_VALUE_F32) MAXK_LINEAR(MAXK_VALUE_F32);
    else if (value_type == MAXK_VALUE_BF16) MAXK_LINEAR(MAXK_VALUE_BF16);
    else MAXK_LINEAR(MAXK_VALUE_F16);
#undef MAXK_LINEAR
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

}  // namespace maxk
