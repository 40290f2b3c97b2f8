// Entry points of the norm, the log probabilities and distillation: checks of their arguments (include/maxk.h).
#include <math.h>

#include "heads.hpp"

namespace {

using namespace maxk;

bool bad_type(int t) { return t < MAXK_VALUE_F32 || t > MAXK_VALUE_F16; }
size_t bytes_of(int t) { return t == MAXK_VALUE_F32 ? 4 : 2; }
bool bad_values(const void* p, int t) { return !p || !aligned(p, bytes_of(t)); }
bool bad_floats(const void* p) { return !aligned(p, 4); }  // (null is none)

maxk_status bad_rows(int64_t N, int64_t dim, int64_t most)
{
    if (N < 0 || N > 0x7FFFFFF0ll || dim < 1) return MAXK_INVALID_ARGUMENT;
    return dim > most ? MAXK_UNSUPPORTED : MAXK_OK;
}

bool bad_index(const void* p, int bytes, int V)
{
    if (bytes != 1 && bytes != 2 && bytes != 4) return true;
    return !p || !aligned(p, (size_t)bytes) || (bytes == 1 && V > 256) || (bytes == 2 && V > 65536);
}

bool bad_labels(const void* p, int bytes) { return p && ((bytes != 4 && bytes != 8) || !aligned(p, (size_t)bytes)); }

// Logits are taken times log2 e / temperature in fp32: a factor of Inf makes a NaN of the largest one's difference, 0
bool good_temperature(double t) { return t > 0.0 && isfinite((float)t) && isfinite((float)(1.0 / t) * kLog2e); }

// r is fp32, and 1 / sqrt(eps) of a row of zeros: Inf there makes NaN of it
bool good_eps(double eps) { return eps > 0.0 && isfinite(eps) && isfinite((float)(1.0 / sqrt(eps))); }

maxk_status classes(const ClassCall& C, int value_type, void* workspace, int64_t bytes, void* stream)
{
    if (bad_values(C.logits, value_type) || (C.dlogits && bad_values(C.dlogits, value_type))) return MAXK_INVALID_ARGUMENT;
    const int64_t need = classes_workspace(C.N, C.V, C.top_k);
    if (need > 0 && (!workspace || !aligned(workspace, 16))) return MAXK_INVALID_ARGUMENT;
    if (bytes < need) return MAXK_SCRATCH_TOO_SMALL;
    return launch_classes(C, value_type, workspace, (hipStream_t)stream);
}

maxk_status logprobs(ClassCall C, int value_type, void* workspace, int64_t bytes, void* stream)
{
    if (bad_type(value_type)) return MAXK_INVALID_ARGUMENT;
    if (const maxk_status st = bad_rows(C.N, C.V, MAXK_MAX_CLASSES)) return st;
    if (C.top_k < 0 || C.top_k > C.V || C.top_k > MAXK_MAX_ALTERNATIVES) return MAXK_INVALID_ARGUMENT;
    if (C.N == 0) return MAXK_OK;
    if (bad_labels(C.labels, C.label_bytes) || ((C.logprob || C.dlogprob) && !C.labels)) return MAXK_INVALID_ARGUMENT;
    if (bad_floats(C.logprob) || bad_floats(C.entropy) || bad_floats(C.dlogprob) || bad_floats(C.dentropy)) return MAXK_INVALID_ARGUMENT;
    if (C.top_k ? !C.top_data || bad_floats(C.top_data) || bad_index(C.top_index, C.top_index_bytes, C.V) : C.top_data || C.top_index)
        return MAXK_INVALID_ARGUMENT;
    return classes(C, value_type, workspace, bytes, stream);
}

maxk_status distill(ClassCall C, int value_type, double temperature, void* workspace, int64_t bytes, void* stream)
{
    if (bad_type(value_type) || bad_type(C.data_type) || !good_temperature(temperature)) return MAXK_INVALID_ARGUMENT;
    if (const maxk_status st = bad_rows(C.N, C.V, MAXK_MAX_CLASSES)) return st;
    if (C.k < 1 || C.k > C.V) return MAXK_INVALID_ARGUMENT;
    if (C.k > MAXK_DISTILL_MAX_K) return MAXK_UNSUPPORTED;
    if (C.N == 0) return MAXK_OK;
    if (bad_values(C.data, C.data_type) || bad_index(C.index, C.index_bytes, C.V) || bad_floats(C.loss) || bad_floats(C.dloss)) return MAXK_INVALID_ARGUMENT;
    C.scale = (float)(1.0 / temperature);
    return classes(C, value_type, workspace, bytes, stream);
}

}  // namespace

extern "C" {

MAXK_API maxk_status maxk_rms_norm(const void* d_X, const void* d_residual, int32_t value_type, int64_t N, int32_t dim, const float* d_gamma, double eps,
                                   void* d_H, void* d_Y, int32_t format, void* d_codes, uint8_t* d_scales, float* d_rstd, void* stream)
{
    if (bad_type(value_type) || !good_eps(eps)) return MAXK_INVALID_ARGUMENT;
    if (const maxk_status st = bad_rows(N, dim, MAXK_NORM_MAX_DIM)) return st;
    if (N == 0) return MAXK_OK;
    if (!d_residual != !d_H || !d_codes != !d_scales || (!d_Y && !d_codes)) return MAXK_INVALID_ARGUMENT;
    if (d_codes && ((format != MAXK_MX_8 && format != MAXK_MX_4) || !aligned(d_codes, 16))) return MAXK_INVALID_ARGUMENT;
    if (bad_values(d_X, value_type) || (d_residual && (bad_values(d_residual, value_type) || bad_values(d_H, value_type))) ||
        (d_Y && bad_values(d_Y, value_type)) || (d_Y && d_Y == d_H) || !d_gamma || bad_floats(d_gamma) || bad_floats(d_rstd))
        return MAXK_INVALID_ARGUMENT;
    return launch_rms_norm({d_X, d_residual, d_gamma, eps, d_H, d_Y, format, (uint8_t*)d_codes, d_scales, d_rstd}, value_type, N, dim, (hipStream_t)stream);
}

MAXK_API int64_t maxk_rms_norm_grad_workspace(int64_t N, int32_t dim)
{
    if (const maxk_status st = bad_rows(N, dim, MAXK_NORM_MAX_DIM)) return st;
    return rms_norm_grad_workspace(N, dim);
}

MAXK_API maxk_status maxk_rms_norm_grad(const void* d_dY, const void* d_H, const void* d_dH, int32_t value_type, int64_t N, int32_t dim,
                                        const float* d_gamma, const float* d_rstd, void* d_dX, float* d_dgamma, void* d_workspace,
                                        int64_t workspace_bytes, void* stream)
{
    if (bad_type(value_type)) return MAXK_INVALID_ARGUMENT;
    if (const maxk_status st = bad_rows(N, dim, MAXK_NORM_MAX_DIM)) return st;
    if (bad_floats(d_dgamma)) return MAXK_INVALID_ARGUMENT;
    if (N > 0 && (bad_values(d_dY, value_type) || bad_values(d_H, value_type) || (d_dH && bad_values(d_dH, value_type)) || !d_gamma || bad_floats(d_gamma) ||
                  !d_rstd || bad_floats(d_rstd) || bad_values(d_dX, value_type)))
        return MAXK_INVALID_ARGUMENT;
    if (d_dgamma && N > 0) {
        if (!d_workspace || !aligned(d_workspace, 16)) return MAXK_INVALID_ARGUMENT;
        if (workspace_bytes < rms_norm_grad_workspace(N, dim)) return MAXK_SCRATCH_TOO_SMALL;
    }
    return launch_rms_norm_grad({d_dY, d_H, d_dH, d_gamma, d_rstd, d_dX, d_dgamma, (float*)d_workspace}, value_type, N, dim, (hipStream_t)stream);
}

MAXK_API int64_t maxk_classes_workspace(int64_t N, int32_t V, int32_t k)
{
    if (const maxk_status st = bad_rows(N, V, MAXK_MAX_CLASSES)) return st;
    if (k < 0 || k > V || k > MAXK_MAX_ALTERNATIVES) return MAXK_INVALID_ARGUMENT;
    return classes_workspace(N, V, k);
}

MAXK_API maxk_status maxk_logprobs(const void* d_logits, int32_t value_type, int64_t N, int32_t V, const void* d_labels, int32_t label_bytes,
                                   float* d_logprob, float* d_entropy, float* d_top_data, void* d_top_index, int32_t index_bytes, int32_t k,
                                   void* d_workspace, int64_t workspace_bytes, void* stream)
{
    ClassCall C = {};
    C.logits = d_logits, C.N = N, C.V = V, C.scale = 1.f;
    C.labels = d_labels, C.label_bytes = label_bytes;
    C.logprob = d_logprob, C.entropy = d_entropy;
    C.top_data = d_top_data, C.top_index = d_top_index, C.top_index_bytes = index_bytes, C.top_k = k;
    if (!d_logprob && !d_entropy && !d_top_data && N > 0) return MAXK_INVALID_ARGUMENT;
    return logprobs(C, value_type, d_workspace, workspace_bytes, stream);
}

MAXK_API maxk_status maxk_logprobs_grad(const void* d_logits, int32_t value_type, int64_t N, int32_t V, const void* d_labels, int32_t label_bytes,
                                        const float* d_dlogprob, const float* d_dentropy, float* d_logprob, float* d_entropy, void* d_dlogits,
                                        void* d_workspace, int64_t workspace_bytes, void* stream)
{
    ClassCall C = {};
    C.logits = d_logits, C.N = N, C.V = V, C.scale = 1.f;
    C.labels = d_labels, C.label_bytes = label_bytes;
    C.dlogprob = d_dlogprob, C.dentropy = d_dentropy;
    C.logprob = d_logprob, C.entropy = d_entropy, C.dlogits = d_dlogits;
    if ((!d_dlogits || (!d_dlogprob && !d_dentropy)) && N > 0) return MAXK_INVALID_ARGUMENT;
    return logprobs(C, value_type, d_workspace, workspace_bytes, stream);
}

MAXK_API maxk_status maxk_distill(const void* d_logits, int32_t value_type, int64_t N, int32_t V, const void* d_top_data, int32_t top_value_type,
                                  const void* d_top_index, int32_t index_bytes, int32_t k, double temperature, float* d_loss, void* d_workspace,
                                  int64_t workspace_bytes, void* stream)
{
    ClassCall C = {};
    C.logits = d_logits, C.N = N, C.V = V;
    C.data = d_top_data, C.data_type = top_value_type, C.index = d_top_index, C.index_bytes = index_bytes, C.k = k;
    C.loss = d_loss;
    if (!d_loss && N > 0) return MAXK_INVALID_ARGUMENT;
    return distill(C, value_type, temperature, d_workspace, workspace_bytes, stream);
}

MAXK_API maxk_status maxk_distill_grad(const void* d_logits, int32_t value_type, int64_t N, int32_t V, const void* d_top_data, int32_t top_value_type,
                                       const void* d_top_index, int32_t index_bytes, int32_t k, double temperature, const float* d_dloss, float* d_loss,
                                       void* d_dlogits, void* d_workspace, int64_t workspace_bytes, void* stream)
{
    ClassCall C = {};
    C.logits = d_logits, C.N = N, C.V = V;
    C.data = d_top_data, C.data_type = top_value_type, C.index = d_top_index, C.index_bytes = index_bytes, C.k = k;
    C.dloss = d_dloss, C.loss = d_loss, C.dlogits = d_dlogits;
    if ((!d_dlogits || !d_dloss) && N > 0) return MAXK_INVALID_ARGUMENT;
    return distill(C, value_type, temperature, d_workspace, workspace_bytes, stream);
}

}  // extern "C"
