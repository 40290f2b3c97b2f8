// Entry points of the microscaled operators: checks of their arguments (include/maxk.h).
#include "mx.hpp"

namespace {

using namespace maxk;

bool bad_type(int t) { return t < MAXK_VALUE_F32 || t > MAXK_VALUE_F16; }
bool bad_format(int f) { return f != MAXK_MX_8 && f != MAXK_MX_4; }
size_t bytes_of(int t) { return t == MAXK_VALUE_F32 ? 4 : 2; }

maxk_status bad_sizes(int64_t N, int64_t a, int64_t b)
{
    if (N < 0 || N > 0x7FFFFFF0ll || a < 1 || b < 1) return MAXK_INVALID_ARGUMENT;
    return a > MAXK_MX_MAX_DIM || b > MAXK_MX_MAX_DIM ? MAXK_UNSUPPORTED : MAXK_OK;
}

bool bad_index(int index_bytes, int dout, int k)
{
    if (index_bytes != 1 && index_bytes != 2 && index_bytes != 4) return true;
    return k < 1 || k > dout || (index_bytes == 1 && dout > 256) || (index_bytes == 2 && dout > 65536);
}

bool bad_codes(const void* codes, const void* scales) { return !codes || !scales || !aligned(codes, 16); }

// the matrices a gradient call reads and writes besides the weights
bool bad_gradient(const MxGrad& G)
{
    if (!G.values || !aligned(G.values, bytes_of(G.value_type))) return true;
    return G.k && (!G.sp_index || !aligned(G.sp_index, (size_t)G.index_bytes));
}

maxk_status weight_grad(const MxMatrix& X, int64_t N, int din, int dout, const MxGrad& G, float* dW, float* db, void* workspace, int64_t bytes,
                        void* stream)
{
    if (bad_format(X.format) || bad_type(G.value_type)) return MAXK_INVALID_ARGUMENT;
    if (const maxk_status st = bad_sizes(N, din, dout)) return st;
    if (!dW || !aligned(dW, 4) || !aligned(db, 4)) return MAXK_INVALID_ARGUMENT;
    if (N > 0 && (bad_codes(X.codes, X.scales) || bad_gradient(G))) return MAXK_INVALID_ARGUMENT;
    if (!workspace || !aligned(workspace, 16)) return MAXK_INVALID_ARGUMENT;
    if (bytes < mx_weight_grad_workspace(N, din, dout)) return MAXK_SCRATCH_TOO_SMALL;
    return launch_mx_weight_grad(X, N, din, dout, G, dW, db, (float*)workspace, (hipStream_t)stream);
}

maxk_status input_grad(const MxGrad& G, int64_t N, const MxMatrix& W, int din, int dout, void* dX, int type, void* stream)
{
    if (bad_type(G.value_type) || bad_type(type)) return MAXK_INVALID_ARGUMENT;
    if (const maxk_status st = bad_sizes(N, din, dout)) return st;
    if (N == 0) return MAXK_OK;
    if (bad_gradient(G) || bad_codes(W.codes, W.scales) || !dX || !aligned(dX, bytes_of(type))) return MAXK_INVALID_ARGUMENT;
    return launch_mx_input_grad(G, N, W, din, dout, dX, type, (hipStream_t)stream);
}

}  // namespace

extern "C" {

MAXK_API maxk_status maxk_mx_quantize(const void* d_X, int32_t value_type, int64_t N, int32_t din, int32_t format, void* d_codes,
                                      uint8_t* d_scales, void* stream)
{
    if (bad_type(value_type) || bad_format(format)) return MAXK_INVALID_ARGUMENT;
    if (const maxk_status st = bad_sizes(N, din, 1)) return st;
    if (N == 0) return MAXK_OK;
    if (!d_X || !aligned(d_X, bytes_of(value_type)) || bad_codes(d_codes, d_scales)) return MAXK_INVALID_ARGUMENT;
    return launch_mx_quantize(d_X, value_type, N, din, format, (uint8_t*)d_codes, d_scales, (hipStream_t)stream);
}

MAXK_API maxk_status maxk_mx_dequantize(const void* d_codes, const uint8_t* d_scales, int32_t format, int64_t N, int32_t din, void* d_X,
                                        int32_t value_type, void* stream)
{
    if (bad_type(value_type) || bad_format(format)) return MAXK_INVALID_ARGUMENT;
    if (const maxk_status st = bad_sizes(N, din, 1)) return st;
    if (N == 0) return MAXK_OK;
    if (!d_X || !aligned(d_X, bytes_of(value_type)) || bad_codes(d_codes, d_scales)) return MAXK_INVALID_ARGUMENT;
    return launch_mx_dequantize({(const uint8_t*)d_codes, d_scales, format}, N, din, d_X, value_type, (hipStream_t)stream);
}

MAXK_API maxk_status maxk_mx_linear(const uint8_t* d_x_codes, const uint8_t* d_x_scales, int64_t N, const uint8_t* d_w_codes,
                                    const uint8_t* d_w_scales, int32_t din, int32_t dout, const float* d_bias, void* d_Y,
                                    int32_t value_type, void* stream)
{
    if (bad_type(value_type)) return MAXK_INVALID_ARGUMENT;
    if (const maxk_status st = bad_sizes(N, din, dout)) return st;
    if (N == 0) return MAXK_OK;
    if (bad_codes(d_x_codes, d_x_scales) || bad_codes(d_w_codes, d_w_scales) || !d_Y || !aligned(d_Y, bytes_of(value_type)) ||
        !aligned(d_bias, 4))
        return MAXK_INVALID_ARGUMENT;
    return launch_mx_linear({d_x_codes, d_x_scales, MAXK_MX_4}, N, {d_w_codes, d_w_scales, MAXK_MX_4}, din, dout, d_bias, d_Y, value_type,
                            (hipStream_t)stream);
}

MAXK_API maxk_status maxk_mx_matvec(const void* d_X, int32_t value_type, int64_t N, const uint8_t* d_w_codes, const uint8_t* d_w_scales, int32_t din,
                                    int32_t dout, const float* d_bias, void* d_Y, int32_t y_value_type, void* stream)
{
    if (bad_type(value_type) || bad_type(y_value_type)) return MAXK_INVALID_ARGUMENT;
    if (N < 0 || din < 1 || dout < 1) return MAXK_INVALID_ARGUMENT;
    if (din > MAXK_MX_MAX_DIM || dout > MAXK_MAX_CLASSES || N > MAXK_MX_MATVEC_MAX_ROWS) return MAXK_UNSUPPORTED;
    if (N == 0) return MAXK_OK;
    if (!d_X || !aligned(d_X, bytes_of(value_type)) || bad_codes(d_w_codes, d_w_scales) || !d_Y || !aligned(d_Y, bytes_of(y_value_type)) || !aligned(d_bias, 4))
        return MAXK_INVALID_ARGUMENT;
    return launch_mx_matvec(d_X, value_type, N, {d_w_codes, d_w_scales, MAXK_MX_4}, din, dout, d_bias, d_Y, y_value_type, (hipStream_t)stream);
}

MAXK_API int64_t maxk_mx_weight_grad_workspace(int64_t N, int32_t din, int32_t dout)
{
    if (const maxk_status st = bad_sizes(N, din, dout)) return st;
    return mx_weight_grad_workspace(N, din, dout);
}

MAXK_API maxk_status maxk_mx_weight_grad(const void* d_codes, const uint8_t* d_scales, int32_t format, int64_t N, int32_t din, int32_t dout,
                                         const void* d_dH, int32_t value_type, float* d_dW, float* d_db, void* d_workspace,
                                         int64_t workspace_bytes, void* stream)
{
    return weight_grad({(const uint8_t*)d_codes, d_scales, format}, N, din, dout, {d_dH, value_type, nullptr, 0, 0}, d_dW, d_db, d_workspace,
                       workspace_bytes, stream);
}

MAXK_API maxk_status maxk_mx_weight_grad_cbsr(const void* d_codes, const uint8_t* d_scales, int32_t format, int64_t N, int32_t din,
                                              int32_t dout, const float* d_dXs, const void* d_sp_index, int32_t index_bytes, int32_t k,
                                              float* d_dW, float* d_db, void* d_workspace, int64_t workspace_bytes, void* stream)
{
    if (bad_index(index_bytes, dout, k)) return MAXK_INVALID_ARGUMENT;
    return weight_grad({(const uint8_t*)d_codes, d_scales, format}, N, din, dout, {d_dXs, MAXK_VALUE_F32, d_sp_index, index_bytes, k}, d_dW,
                       d_db, d_workspace, workspace_bytes, stream);
}

MAXK_API maxk_status maxk_mx_input_grad(const void* d_dH, int32_t value_type, int64_t N, const uint8_t* d_w_codes, const uint8_t* d_w_scales,
                                        int32_t din, int32_t dout, void* d_dX, int32_t dx_value_type, void* stream)
{
    return input_grad({d_dH, value_type, nullptr, 0, 0}, N, {d_w_codes, d_w_scales, MAXK_MX_4}, din, dout, d_dX, dx_value_type, stream);
}

MAXK_API maxk_status maxk_mx_input_grad_cbsr(const float* d_dXs, const void* d_sp_index, int32_t index_bytes, int32_t k, int64_t N,
                                             const uint8_t* d_w_codes, const uint8_t* d_w_scales, int32_t din, int32_t dout, void* d_dX,
                                             int32_t dx_value_type, void* stream)
{
    if (bad_index(index_bytes, dout, k)) return MAXK_INVALID_ARGUMENT;
    return input_grad({d_dXs, MAXK_VALUE_F32, d_sp_index, index_bytes, k}, N, {d_w_codes, d_w_scales, MAXK_MX_4}, din, dout, d_dX,
                      dx_value_type, stream);
}

}  // extern "C"
