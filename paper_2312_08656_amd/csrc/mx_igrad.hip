// Input gradient of the linear map with 4-bit weights (include/maxk.h): dX = dH W.
#include <algorithm>

#include "mx.hpp"

namespace maxk {
namespace {

__device__ __forceinline__ int grad_column(const MxGrad& G, int64_t row, int t)
{
    if (!G.k) return t;
    const int64_t at = row * G.k + t;
    return G.index_bytes == 1 ? ((const uint8_t*)G.sp_index)[at] : G.index_bytes == 2 ? ((const uint16_t*)G.sp_index)[at] : ((const int32_t*)G.sp_index)[at];
}

__device__ __forceinline__ float grad_value(const MxGrad& G, int64_t row, int t, int width)
{
    const int64_t at = row * width + t;
    if (G.value_type == MAXK_VALUE_F32) return ((const float*)G.values)[at];
    return G.value_type == MAXK_VALUE_BF16 ? widen_value<MAXK_VALUE_BF16>(((const uint16_t*)G.values)[at]) : widen_value<MAXK_VALUE_F16>(((const uint16_t*)G.values)[at]);
}

template <int VT>
__global__ void input_grad_kernel(MxGrad G, int64_t N, MxMatrix W, int din, int dout, value_store_t<VT>* dX)
{
    const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (at >= N * din) return;
    const int64_t row = at / din;
    const int i = (int)(at % din), nb = mx_blocks(din), width = G.k ? G.k : dout;
    float sum = 0.f;
    for (int t = 0; t < width; ++t) {
        const int o = grad_column(G, row, t);
        if ((uint32_t)o < (uint32_t)dout) sum += grad_value(G, row, t, width) * mx_value<MAXK_MX_4>(W.codes, W.scales, o, i, nb);
    }
    dX[at] = narrow_value<VT>(sum);
}

}  // namespace

maxk_status launch_mx_input_grad(const MxGrad& G, int64_t N, const MxMatrix& W, int din, int dout, void* dX, int value_type, hipStream_t s)
{
    const int64_t grid = (N * din + 255) / 256;
    if (grid > 0x7FFFFFFF) return MAXK_UNSUPPORTED;
#define MAXK_INPUT_GRAD(VT) \
    hipLaunchKernelGGL((input_grad_kernel<VT>), dim3((unsigned)grid), dim3(256), 0, s, G, N, W, din, dout, (value_store_t<VT>*)dX)
    if (value_type == MAXK_VALUE_F32) MAXK_INPUT_GRAD(MAXK_VALUE_F32);
    else if (value_type == MAXK_VALUE_BF16) MAXK_INPUT_GRAD(MAXK_VALUE_BF16);
    else MAXK_INPUT_GRAD(MAXK_VALUE_F16);
#undef MAXK_INPUT_GRAD
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

}  // namespace maxk
