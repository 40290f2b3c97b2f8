// Both ends of a classifier (include/maxk.h): the norm in front of a layer, class probabilities and their losses behind the last one.
#pragma once

#include "common.hpp"

namespace maxk {

constexpr float kLog2e = 1.44269504088896341f;

struct NormCall {
    const void *X, *residual;  // residual: may be null, and H with it
    const float* gamma;
    double eps;
    void *H, *Y;               // Y: may be null
    int format;                // of codes
    uint8_t *codes, *scales;   // may be null
    float* rstd;               // may be null
};
maxk_status launch_rms_norm(const NormCall& C, int value_type, int64_t N, int dim, hipStream_t s);

struct NormGradCall {
    const void *dY, *H, *dH;   // dH: may be null
    const float *gamma, *rstd;
    void* dX;
    float* dgamma;             // may be null
    float* workspace;
};
int64_t rms_norm_grad_workspace(int64_t N, int dim);
maxk_status launch_rms_norm_grad(const NormGradCall& C, int value_type, int64_t N, int dim, hipStream_t s);

// Rows of logits [N x V] and what is made of them.  Log probabilities (index null): of the given classes, entropies, the likeliest classes, or (dlogits) the
// gradient.  Distillation (index): the divergence from the k entries a row that a teacher passed on, and (dlogits) the gradient.
struct ClassCall {
    const void* logits;
    int64_t N;
    int32_t V;
    float scale;                        // logits are taken times this
    // given
    const void* labels;                 // may be null
    const void *data, *index;           // the teacher's entries
    int32_t label_bytes, data_type, index_bytes, k;
    const float *dlogprob, *dentropy, *dloss;  // the first two may be null
    // results
    float *logprob, *entropy, *loss;    // may be null
    float* top_data;                    // may be null, and top_index with it
    void* top_index;
    int32_t top_index_bytes, top_k;
    void* dlogits;                      // may be null
};
int64_t classes_workspace(int64_t N, int32_t V, int32_t top_k);  // 0: none is needed
maxk_status launch_classes(const ClassCall& C, int value_type, void* workspace, hipStream_t s);

}  // namespace maxk
