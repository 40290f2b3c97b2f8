// Gradients of the linear map on microscaled storage (include/maxk.h): dW = dH^T X, db, dX = dH W.
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

// Rows are cut into ranges; thread i of a range's workgroup owns column i of the range's sums, and db is column din.
constexpr int kRangeRows = 1024;
__host__ __device__ constexpr int64_t ranges(int64_t N) { return N / kRangeRows < 1 ? 1 : N / kRangeRows > 256 ? 256 : N / kRangeRows; }

__global__ void weight_grad_kernel(MxMatrix X, int64_t N, int din, int dout, MxGrad G, float* sums)
{
    const int i = blockIdx.y * blockDim.x + threadIdx.x, nb = mx_blocks(din), width = G.k ? G.k : dout;
    if (i > din) return;
    float* mine = sums + (int64_t)blockIdx.x * dout * (din + 1);
    for (int o = 0; o < dout; ++o) mine[(int64_t)o * (din + 1) + i] = 0.f;
    const int64_t first = N * blockIdx.x / gridDim.x, last = N * (blockIdx.x + 1) / gridDim.x;
    for (int64_t n = first; n < last; ++n) {
        const float x = i == din ? 1.f : X.format == MAXK_MX_8 ? mx_value<MAXK_MX_8>(X.codes, X.scales, n, i, nb) : mx_value<MAXK_MX_4>(X.codes, X.scales, n, i, nb);
        for (int t = 0; t < width; ++t) {
            const int o = grad_column(G, n, t);
            if ((uint32_t)o < (uint32_t)dout) mine[(int64_t)o * (din + 1) + i] += grad_value(G, n, t, width) * x;
        }
    }
}

__global__ void add_ranges_kernel(const float* sums, int64_t n_ranges, int din, int dout, float* dW, float* db)
{
    const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, all = (int64_t)dout * (din + 1);
    if (at >= all) return;
    float sum = 0.f;
    for (int64_t r = 0; r < n_ranges; ++r) sum += sums[r * all + at];
    const int64_t o = at / (din + 1);
    const int i = (int)(at % (din + 1));
    if (i < din) dW[o * din + i] = sum;
    else if (db) db[o] = sum;
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

int64_t mx_weight_grad_workspace(int64_t N, int din, int dout) { return ranges(N) * dout * (din + 1ll) * (int64_t)sizeof(float); }

maxk_status launch_mx_weight_grad(const MxMatrix& X, int64_t N, int din, int dout, const MxGrad& G, float* dW, float* db, float* workspace,
                                  hipStream_t s)
{
    const unsigned n = (unsigned)ranges(N);
    hipLaunchKernelGGL(weight_grad_kernel, dim3(n, (din + 64) / 64), dim3(64), 0, s, X, N, din, dout, G, workspace);
    MAXK_LAUNCH_CHECK();
    const int64_t all = (int64_t)dout * (din + 1);
    hipLaunchKernelGGL(add_ranges_kernel, dim3((unsigned)((all + 255) / 256)), dim3(256), 0, s, workspace, (int64_t)n, din, dout, dW, db);
    MAXK_LAUNCH_CHECK();
    return MAXK_OK;
}

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
