"""MaxK-GNN aggregation hot path on AMD MI355X: thin Python binding of libmaxk.

Argument marshalling only -- every step (top-k/CBSR, forward SpGEMM, backward
SSpMM, dense SpMM baseline, graph preprocessing) runs in the HIP kernels behind
the C ABI declared in ``include/maxk.h``.  PyTorch supplies device memory and
the stream, nothing else.  There is no CPU or eager fallback: if ``libmaxk.so``
is missing or a call fails, an exception is raised.
"""
from .binding import (  # noqa: F401
    BWD_AUTO,
    BWD_EXPAND_REDUCE,
    BWD_PULL_CSC,
    BWD_PUSH_CSR,
    BWD_SLAB_PULL,
    BWD_TILED,
    VALUE_BF16,
    VALUE_F16,
    VALUE_F32,
    MaxKError,
    MaxKGraph,
    index_dtype,
    lib_path,
    load_library,
    maxk_cbsr_scatter,
    maxk_graph_create,
    maxk_graph_destroy,
    maxk_spgemm_fwd,
    maxk_spgemm_fwd_narrow,
    maxk_spgemm_fwd_noalloc,
    maxk_sspmm_bwd,
    maxk_sspmm_bwd_narrow,
    maxk_topk_cbsr,
    maxk_topk_cbsr_narrow,
    spmm_baseline,
)
from .mx import (  # noqa: E402,F401
    MX_4,
    MX_8,
    maxk_mx_dequantize,
    maxk_mx_input_grad,
    maxk_mx_input_grad_cbsr,
    maxk_mx_linear,
    maxk_mx_matvec,
    maxk_mx_quantize,
    maxk_mx_weight_grad,
    maxk_mx_weight_grad_cbsr,
    mx_blocks,
    mx_empty,
    mx_weight_grad_workspace,
)
from .heads import (  # noqa: E402,F401
    classes_workspace,
    maxk_distill,
    maxk_distill_grad,
    maxk_logprobs,
    maxk_logprobs_grad,
    maxk_rms_norm,
    maxk_rms_norm_grad,
    rms_norm_grad_workspace,
)
from .autograd import (  # noqa: E402,F401
    MaxKAggregate,
    MaxKDistill,
    MaxKLayer,
    MaxKLogprobs,
    MaxKNormLayer,
    MaxKRMSNorm,
    maxk_aggregate,
    maxk_class_logprobs,
    maxk_distill_loss,
    maxk_layer,
    maxk_norm_layer,
    maxk_residual_norm,
)
