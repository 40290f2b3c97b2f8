// Marshalling of torch tensors for the calls of a pass: what binding.py does with ctypes, and the two halves of one aggregation with
// their buffers.  Host code only; the calls themselves are libmaxk's, whose addresses come from binding.py.
//
// Bound by the host on small graphs: a call took 4.8 to 5.1 us from Python, 1.2 of them checks and 0.8 ctypes, an empty tensor 1.5, and
// the backward half of a pass runs in a thread of its own, where the same Python is slower still.
//
// Every function returns false (None) on anything but plain device tensors of the shapes and types that the call takes; binding.py then makes
// the call itself, which raises what is to be raised.  A call that was made and failed is not made again: its status goes to binding.py's check.
#include <c10/hip/HIPStream.h>
#include <torch/extension.h>

#include <utility>

#include "../../include/maxk.h"

namespace {

decltype(&maxk_topk_cbsr_narrow) topk_call;
decltype(&maxk_spgemm_fwd_narrow) forward_call;
decltype(&maxk_spgemm_fwd_noalloc) forward_noalloc_call;
decltype(&maxk_sspmm_bwd_narrow) backward_call;
decltype(&maxk_cbsr_scatter) scatter_call;
decltype(&maxk_mx_quantize) quantize_call;
decltype(&maxk_mx_dequantize) dequantize_call;
decltype(&maxk_mx_linear) linear_call;
decltype(&maxk_mx_weight_grad_workspace) weight_grad_workspace_call;
decltype(&maxk_mx_weight_grad) weight_grad_call;
decltype(&maxk_mx_weight_grad_cbsr) weight_grad_cbsr_call;
decltype(&maxk_mx_input_grad) input_grad_call;
decltype(&maxk_mx_input_grad_cbsr) input_grad_cbsr_call;

decltype(&maxk_mx_matvec) matvec_call;
decltype(&maxk_rms_norm) rms_norm_call;
decltype(&maxk_rms_norm_grad_workspace) rms_norm_grad_workspace_call;
decltype(&maxk_rms_norm_grad) rms_norm_grad_call;
decltype(&maxk_classes_workspace) classes_workspace_call;
decltype(&maxk_logprobs) logprobs_call;
decltype(&maxk_logprobs_grad) logprobs_grad_call;
decltype(&maxk_distill) distill_call;
decltype(&maxk_distill_grad) distill_grad_call;

PyObject* check;  // (status, name of the call): raises; held for good

void bind(const std::vector<uintptr_t>& at, const py::function& raise)
{
    TORCH_CHECK(at.size() == 22, "twenty-two addresses");
    topk_call = reinterpret_cast<decltype(topk_call)>(at[0]);
    forward_call = reinterpret_cast<decltype(forward_call)>(at[1]);
    forward_noalloc_call = reinterpret_cast<decltype(forward_noalloc_call)>(at[2]);
    backward_call = reinterpret_cast<decltype(backward_call)>(at[3]);
    scatter_call = reinterpret_cast<decltype(scatter_call)>(at[4]);
    quantize_call = reinterpret_cast<decltype(quantize_call)>(at[5]);
    dequantize_call = reinterpret_cast<decltype(dequantize_call)>(at[6]);
    linear_call = reinterpret_cast<decltype(linear_call)>(at[7]);
    weight_grad_workspace_call = reinterpret_cast<decltype(weight_grad_workspace_call)>(at[8]);
    weight_grad_call = reinterpret_cast<decltype(weight_grad_call)>(at[9]);
    weight_grad_cbsr_call = reinterpret_cast<decltype(weight_grad_cbsr_call)>(at[10]);
    input_grad_call = reinterpret_cast<decltype(input_grad_call)>(at[11]);
    input_grad_cbsr_call = reinterpret_cast<decltype(input_grad_cbsr_call)>(at[12]);
    matvec_call = reinterpret_cast<decltype(matvec_call)>(at[13]);
    rms_norm_call = reinterpret_cast<decltype(rms_norm_call)>(at[14]);
    rms_norm_grad_workspace_call = reinterpret_cast<decltype(rms_norm_grad_workspace_call)>(at[15]);
    rms_norm_grad_call = reinterpret_cast<decltype(rms_norm_grad_call)>(at[16]);
    classes_workspace_call = reinterpret_cast<decltype(classes_workspace_call)>(at[17]);
    logprobs_call = reinterpret_cast<decltype(logprobs_call)>(at[18]);
    logprobs_grad_call = reinterpret_cast<decltype(logprobs_grad_call)>(at[19]);
    distill_call = reinterpret_cast<decltype(distill_call)>(at[20]);
    distill_grad_call = reinterpret_cast<decltype(distill_grad_call)>(at[21]);
    Py_XDECREF(std::exchange(check, py::function(raise).release().ptr()));
}

// The tensor in `x`, where it is a plain one in device memory: no subclass with a dispatch of its own, no functorch wrapper
const at::Tensor* plain(const py::handle& x)
{
    if (!THPVariable_Check(x.ptr())) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(x.ptr());
    if (!t.defined() || !t.is_cuda() || !t.has_storage() || t.layout() != at::kStrided) return nullptr;
    const auto keys = t.key_set();
    if (keys.has_any(c10::DispatchKeySet({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::FuncTorchBatched,
                                          c10::DispatchKey::Functionalize})))
        return nullptr;
    return &t;
}

const at::Tensor* matrix(const py::handle& x, int64_t rows, int64_t cols)  // contiguous; -1: any
{
    const at::Tensor* t = plain(x);
    if (!t || t->dim() != 2 || !t->is_contiguous()) return nullptr;
    return (rows < 0 || t->size(0) == rows) && (cols < 0 || t->size(1) == cols) ? t : nullptr;
}

int index_bytes(const at::Tensor& t)
{
    switch (t.scalar_type()) {
        case at::kByte: return 1;
        case at::kUInt16:
        case at::kShort: return 2;
        case at::kInt: return 4;
        default: return 0;
    }
}

int value_type(const at::Tensor& t)
{
    return t.scalar_type() == at::kFloat ? MAXK_VALUE_F32 : t.scalar_type() == at::kBFloat16 ? MAXK_VALUE_BF16 : t.scalar_type() == at::kHalf ? MAXK_VALUE_F16 : -1;
}

bool takes(const at::Tensor& t, bool narrow) { return narrow ? value_type(t) >= 0 : t.scalar_type() == at::kFloat; }

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

maxk_graph* graph(uintptr_t g) { return reinterpret_cast<maxk_graph*>(g); }

template <typename F>
bool made(const char* what, F&& call)  // call() may change `what` to the call that failed
{
    maxk_status st;
    {
        py::gil_scoped_release released;  // a first call may build tables
        st = call(what);
    }
    if (st != MAXK_OK) py::reinterpret_borrow<py::function>(check)(st, what);
    return true;
}

bool topk(const py::handle& H_, int64_t k, const py::handle& data_, const py::handle& index_, bool narrow)
{
    const at::Tensor* H = matrix(H_, -1, -1);
    if (!H || H->scalar_type() != at::kFloat) return false;
    const int64_t N = H->size(0), dim = H->size(1);
    const at::Tensor *data = matrix(data_, N, k), *index = matrix(index_, N, k);
    if (!data || !index || !takes(*data, narrow) || !index_bytes(*index)) return false;
    return made(narrow ? "maxk_topk_cbsr_narrow" : "maxk_topk_cbsr", [&, s = stream()](const char*) {
        return topk_call(static_cast<const float*>(H->data_ptr()), N, (int32_t)dim, (int32_t)k, data->data_ptr(), value_type(*data), index->data_ptr(),
                         index_bytes(*index), s);
    });
}

bool forward(uintptr_t g, int64_t N, const py::handle& data_, const py::handle& index_, int64_t dim, const py::handle& Y_, bool narrow)
{
    const at::Tensor *data = matrix(data_, N, -1), *Y = matrix(Y_, N, dim);
    if (!g || !data || !Y || !takes(*data, narrow) || Y->scalar_type() != at::kFloat) return false;
    const int64_t k = data->size(1);
    const at::Tensor* index = matrix(index_, N, k);
    if (!index || !index_bytes(*index)) return false;
    return made(narrow ? "maxk_spgemm_fwd_narrow" : "maxk_spgemm_fwd", [&, s = stream()](const char*) {
        return forward_call(graph(g), data->data_ptr(), value_type(*data), index->data_ptr(), index_bytes(*index), (int32_t)dim, (int32_t)k,
                            static_cast<float*>(Y->data_ptr()), s);
    });
}

bool forward_noalloc(uintptr_t g, int64_t N, const py::handle& data_, const py::handle& index_, int64_t dim, const py::handle& Y_)
{
    const at::Tensor *data = matrix(data_, N, -1), *Y = matrix(Y_, N, dim);
    if (!g || !data || !Y || data->scalar_type() != at::kFloat || Y->scalar_type() != at::kFloat) return false;
    const int64_t k = data->size(1);
    const at::Tensor* index = matrix(index_, N, k);
    if (!index || !index_bytes(*index)) return false;
    return made("maxk_spgemm_fwd_noalloc", [&, s = stream()](const char*) {
        return forward_noalloc_call(graph(g), static_cast<const float*>(data->data_ptr()), index->data_ptr(), index_bytes(*index), (int32_t)dim,
                                    (int32_t)k, static_cast<float*>(Y->data_ptr()), s);
    });
}

bool backward(uintptr_t g, int64_t N, const py::handle& dY_, const py::handle& index_, const py::handle& dXs_, bool narrow)
{
    const at::Tensor *dY = matrix(dY_, N, -1), *index = matrix(index_, N, -1);
    if (!g || !dY || !index || !takes(*dY, narrow) || !index_bytes(*index)) return false;
    const int64_t k = index->size(1);
    const at::Tensor* dXs = matrix(dXs_, N, k);
    if (!dXs || dXs->scalar_type() != at::kFloat) return false;
    return made(narrow ? "maxk_sspmm_bwd_narrow" : "maxk_sspmm_bwd", [&, s = stream()](const char*) {
        return backward_call(graph(g), dY->data_ptr(), value_type(*dY), index->data_ptr(), index_bytes(*index), (int32_t)dY->size(1), (int32_t)k,
                             static_cast<float*>(dXs->data_ptr()), s);
    });
}

bool scatter(const py::handle& values_, const py::handle& index_, const py::handle& dense_)
{
    const at::Tensor* values = matrix(values_, -1, -1);
    if (!values || values->scalar_type() != at::kFloat) return false;
    const int64_t N = values->size(0), k = values->size(1);
    const at::Tensor *index = matrix(index_, N, k), *dense = matrix(dense_, N, -1);
    if (!index || !dense || !index_bytes(*index) || dense->scalar_type() != at::kFloat) return false;
    return made("maxk_cbsr_scatter", [&, s = stream()](const char*) {
        return scatter_call(static_cast<const float*>(values->data_ptr()), index->data_ptr(), index_bytes(*index), N, (int32_t)dense->size(1), (int32_t)k,
                            static_cast<float*>(dense->data_ptr()), s);
    });
}

at::ScalarType index_type(int ib) { return ib == 1 ? at::kByte : ib == 2 ? at::kUInt16 : at::kInt; }

// (Y, sp_index) of one aggregation: top-k, then the forward pass
py::object aggregate_forward(uintptr_t g, int64_t N, const py::handle& H_, int64_t k, int ib)
{
    const at::Tensor* H = matrix(H_, N, -1);
    if (!g || !H || H->scalar_type() != at::kFloat || k < 1 || (ib != 1 && ib != 2 && ib != 4)) return py::none();
    const int64_t dim = H->size(1);
    if (k > dim) return py::none();
    at::Tensor data, index, Y;
    try {
        data = at::empty({N, k}, H->options());
        index = at::empty({N, k}, H->options().dtype(index_type(ib)));
        Y = at::empty({N, dim}, H->options());
    } catch (const c10::Error&) {  // no memory: said by the calls from Python
        return py::none();
    }
    made("maxk_topk_cbsr", [&, s = stream()](const char*& what) {
        const maxk_status st = topk_call(static_cast<const float*>(H->data_ptr()), N, (int32_t)dim, (int32_t)k, data.data_ptr(), MAXK_VALUE_F32,
                                         index.data_ptr(), ib, s);
        if (st != MAXK_OK) return st;
        what = "maxk_spgemm_fwd";
        return forward_call(graph(g), data.data_ptr(), MAXK_VALUE_F32, index.data_ptr(), ib, (int32_t)dim, (int32_t)k, static_cast<float*>(Y.data_ptr()), s);
    });
    return py::make_tuple(Y, index);
}

// dH of one aggregation: the backward pass at the columns kept, then back to dense rows
py::object aggregate_backward(uintptr_t g, int64_t N, const py::handle& dY_, const py::handle& index_, int64_t dim, int64_t k)
{
    const at::Tensor *dY = matrix(dY_, N, dim), *index = matrix(index_, N, k);
    if (!g || !dY || !index || dY->scalar_type() != at::kFloat || !index_bytes(*index)) return py::none();
    const int ib = index_bytes(*index);
    at::Tensor dXs, dH;
    try {
        dXs = at::empty({N, k}, dY->options());
        dH = at::empty({N, dim}, dY->options());
    } catch (const c10::Error&) {
        return py::none();
    }
    made("maxk_sspmm_bwd", [&, s = stream()](const char*& what) {
        const maxk_status st = backward_call(graph(g), dY->data_ptr(), MAXK_VALUE_F32, index->data_ptr(), ib, (int32_t)dim, (int32_t)k,
                                             static_cast<float*>(dXs.data_ptr()), s);
        if (st != MAXK_OK) return st;
        what = "maxk_cbsr_scatter";
        return scatter_call(static_cast<const float*>(dXs.data_ptr()), index->data_ptr(), ib, N, (int32_t)dim, (int32_t)k, static_cast<float*>(dH.data_ptr()), s);
    });
    return py::cast(dH);
}

// ---- microscaled storage ----

// matrix() of a width that the calls take, and 32 bits hold
const at::Tensor* sized(const py::handle& x, int64_t rows, int64_t cols)
{
    const at::Tensor* t = matrix(x, rows, cols);
    return t && t->size(1) <= MAXK_MX_MAX_DIM ? t : nullptr;
}

// A stored matrix [rows, din]: its codes and scales, or nulls.  din < 0: as many whole blocks as there are
struct Stored {
    const at::Tensor *codes, *scales;
    int format;
    int64_t din;
    explicit operator bool() const { return codes != nullptr; }
    uint8_t* code() const { return static_cast<uint8_t*>(codes->data_ptr()); }
    uint8_t* scale() const { return static_cast<uint8_t*>(scales->data_ptr()); }
};

Stored stored(const py::handle& codes_, const py::handle& scales_, int64_t rows, int64_t din, bool only4)
{
    const at::Tensor *scales = matrix(scales_, rows, din < 0 ? -1 : (din + 31) / 32), *codes = matrix(codes_, rows, -1);
    if (!scales || !codes || scales->scalar_type() != at::kByte) return {};
    const bool four = codes->scalar_type() == at::kByte;
    if (!four && (only4 || codes->scalar_type() != at::kChar)) return {};
    if (codes->size(1) != scales->size(1) * (four ? 16 : 32) || (din < 0 && scales->size(1) > MAXK_MX_MAX_DIM / 32)) return {};
    return {codes, scales, four ? MAXK_MX_4 : MAXK_MX_8, din < 0 ? scales->size(1) * 32 : din};
}

const at::Tensor* vector(const py::handle& x, int64_t length)
{
    const at::Tensor* t = plain(x);
    return t && t->dim() == 1 && t->is_contiguous() && t->size(0) == length && t->scalar_type() == at::kFloat ? t : nullptr;
}

bool mx_quantize(const py::handle& X_, const py::handle& codes_, const py::handle& scales_)
{
    const at::Tensor* X = sized(X_, -1, -1);
    if (!X || value_type(*X) < 0) return false;
    const Stored to = stored(codes_, scales_, X->size(0), X->size(1), false);
    if (!to) return false;
    return made("maxk_mx_quantize", [&, s = stream()](const char*) {
        return quantize_call(X->data_ptr(), value_type(*X), X->size(0), (int32_t)X->size(1), to.format, to.code(), to.scale(), s);
    });
}

bool mx_dequantize(const py::handle& codes_, const py::handle& scales_, const py::handle& X_)
{
    const at::Tensor* X = sized(X_, -1, -1);
    if (!X || value_type(*X) < 0) return false;
    const Stored from = stored(codes_, scales_, X->size(0), X->size(1), false);
    if (!from) return false;
    return made("maxk_mx_dequantize", [&, s = stream()](const char*) {
        return dequantize_call(from.code(), from.scale(), from.format, X->size(0), (int32_t)X->size(1), X->data_ptr(), value_type(*X), s);
    });
}

bool mx_linear(const py::handle& xc, const py::handle& xs, const py::handle& wc, const py::handle& ws, const py::handle& Y_, const py::handle& bias_)
{
    const at::Tensor* Y = sized(Y_, -1, -1);
    if (!Y || value_type(*Y) < 0) return false;
    const Stored X = stored(xc, xs, Y->size(0), -1, true), W = stored(wc, ws, Y->size(1), -1, true);
    const at::Tensor* bias = bias_.is_none() ? nullptr : vector(bias_, Y->size(1));
    if (!X || !W || X.din != W.din || (!bias && !bias_.is_none())) return false;
    return made("maxk_mx_linear", [&, s = stream()](const char*) {
        return linear_call(X.code(), X.scale(), Y->size(0), W.code(), W.scale(), (int32_t)X.din, (int32_t)Y->size(1),
                           bias ? static_cast<const float*>(bias->data_ptr()) : nullptr, Y->data_ptr(), value_type(*Y), s);
    });
}

// The gradient of a call: dense (index_ None) or CBSR
struct Gradient {
    const at::Tensor *values, *index;
    explicit operator bool() const { return values != nullptr; }
};

Gradient gradient(const py::handle& values_, const py::handle& index_)
{
    const at::Tensor* values = sized(values_, -1, -1);
    if (!values || value_type(*values) < 0) return {};
    if (index_.is_none()) return {values, nullptr};
    const at::Tensor* index = matrix(index_, values->size(0), values->size(1));
    if (!index || !index_bytes(*index) || values->scalar_type() != at::kFloat) return {};
    return {values, index};
}

bool mx_weight_grad(const py::handle& codes_, const py::handle& scales_, const py::handle& values_, const py::handle& index_, const py::handle& dW_,
                    const py::handle& db_, const py::handle& workspace_)
{
    const Gradient G = gradient(values_, index_);
    const at::Tensor* dW = sized(dW_, -1, -1);
    if (!G || !dW || dW->scalar_type() != at::kFloat) return false;
    const int64_t N = G.values->size(0), dout = dW->size(0), din = dW->size(1);
    if (!G.index && G.values->size(1) != dout) return false;
    const Stored X = stored(codes_, scales_, N, din, false);
    const at::Tensor* db = db_.is_none() ? nullptr : vector(db_, dout);
    if (!X || (!db && !db_.is_none()) || dout > MAXK_MX_MAX_DIM) return false;
    at::Tensor own;
    const at::Tensor* workspace = &own;
    if (workspace_.is_none()) {
        const int64_t need = weight_grad_workspace_call(N, (int32_t)din, (int32_t)dout);
        if (need < 0) return false;
        try {
            own = at::empty({need}, dW->options().dtype(at::kByte));
        } catch (const c10::Error&) {  // no memory: said by the call from Python
            return false;
        }
    } else {
        workspace = plain(workspace_);
        if (!workspace || !workspace->is_contiguous() || workspace->scalar_type() != at::kByte) return false;
    }
    float *w = static_cast<float*>(dW->data_ptr()), *b = db ? static_cast<float*>(db->data_ptr()) : nullptr;
    return made(G.index ? "maxk_mx_weight_grad_cbsr" : "maxk_mx_weight_grad", [&, s = stream()](const char*) {
        if (G.index)
            return weight_grad_cbsr_call(X.code(), X.scale(), X.format, N, (int32_t)din, (int32_t)dout, static_cast<const float*>(G.values->data_ptr()),
                                         G.index->data_ptr(), index_bytes(*G.index), (int32_t)G.values->size(1), w, b, workspace->data_ptr(),
                                         workspace->numel(), s);
        return weight_grad_call(X.code(), X.scale(), X.format, N, (int32_t)din, (int32_t)dout, G.values->data_ptr(), value_type(*G.values), w, b,
                                workspace->data_ptr(), workspace->numel(), s);
    });
}

bool mx_input_grad(const py::handle& values_, const py::handle& index_, const py::handle& wc, const py::handle& ws, const py::handle& dX_)
{
    const Gradient G = gradient(values_, index_);
    const at::Tensor* dX = sized(dX_, -1, -1);
    if (!G || !dX || value_type(*dX) < 0 || dX->size(0) != G.values->size(0)) return false;
    const int64_t N = dX->size(0), din = dX->size(1);
    const Stored W = stored(wc, ws, G.index ? -1 : G.values->size(1), din, true);
    if (!W || W.codes->size(0) != W.scales->size(0)) return false;
    const int64_t dout = W.codes->size(0);
    if (dout > MAXK_MX_MAX_DIM) return false;
    return made(G.index ? "maxk_mx_input_grad_cbsr" : "maxk_mx_input_grad", [&, s = stream()](const char*) {
        if (G.index)
            return input_grad_cbsr_call(static_cast<const float*>(G.values->data_ptr()), G.index->data_ptr(), index_bytes(*G.index),
                                        (int32_t)G.values->size(1), N, W.code(), W.scale(), (int32_t)din, (int32_t)dout, dX->data_ptr(), value_type(*dX), s);
        return input_grad_call(G.values->data_ptr(), value_type(*G.values), N, W.code(), W.scale(), (int32_t)din, (int32_t)dout, dX->data_ptr(),
                               value_type(*dX), s);
    });
}

// ---- both ends of a classifier ----

// Whether tensors (null: none) are the current device's, whose stream a call takes
template <typename... T>
bool here(const T*... tensors)
{
    const c10::DeviceIndex device = c10::hip::current_device();
    return ((!tensors || tensors->device().index() == device) && ...);
}

const void* address(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
void* place(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
float* floats(const at::Tensor* t) { return t ? static_cast<float*>(t->data_ptr()) : nullptr; }

// Arguments that may be None; `good` turns false where one is something else than the call takes
struct Optionals {
    bool good = true;
    const at::Tensor* like(const py::handle& x, const at::Tensor& X)  // a matrix of X's shape and type
    {
        if (x.is_none()) return nullptr;
        const at::Tensor* t = matrix(x, X.size(0), X.size(1));
        good &= t && t->scalar_type() == X.scalar_type();
        return t;
    }
    const at::Tensor* floats(const py::handle& x, int64_t n)
    {
        if (x.is_none()) return nullptr;
        const at::Tensor* t = vector(x, n);
        good &= t != nullptr;
        return t;
    }
    const at::Tensor* labels(const py::handle& x, int64_t n)
    {
        if (x.is_none()) return nullptr;
        const at::Tensor* t = plain(x);
        if (t && (t->dim() != 1 || !t->is_contiguous() || t->size(0) != n || (t->scalar_type() != at::kInt && t->scalar_type() != at::kLong))) t = nullptr;
        good &= t != nullptr;
        return t;
    }
};

int label_bytes(const at::Tensor* t) { return !t ? 0 : t->scalar_type() == at::kLong ? 8 : 4; }

// The workspace of a call that needs `need` bytes: the one that is given, or `own`, made here
bool workspace_for(const py::handle& given, int64_t need, const at::Tensor& X, at::Tensor& own, const at::Tensor*& workspace)
{
    workspace = nullptr;
    if (need < 0) return false;
    if (!given.is_none()) {
        workspace = plain(given);
        return workspace && workspace->is_contiguous() && workspace->scalar_type() == at::kByte && here(workspace);
    }
    if (need == 0) return true;
    try {
        own = at::empty({need}, X.options().dtype(at::kByte));
    } catch (const c10::Error&) {  // no memory: said by the call from Python
        return false;
    }
    workspace = &own;
    return true;
}
int64_t room(const at::Tensor* workspace) { return workspace ? workspace->numel() : 0; }

const at::Tensor* rows(const py::handle& x, int64_t most)  // a matrix of values of a width that the call takes
{
    const at::Tensor* t = matrix(x, -1, -1);
    return t && value_type(*t) >= 0 && t->size(1) <= most ? t : nullptr;
}

bool mx_matvec(const py::handle& X_, const py::handle& wc, const py::handle& ws, const py::handle& Y_, const py::handle& bias_)
{
    const at::Tensor *X = rows(X_, MAXK_MX_MAX_DIM), *Y = rows(Y_, MAXK_MAX_CLASSES);
    if (!X || !Y || Y->size(0) != X->size(0)) return false;
    const Stored W = stored(wc, ws, Y->size(1), X->size(1), true);
    Optionals given;
    const at::Tensor* bias = given.floats(bias_, Y->size(1));
    if (!W || !given.good || !here(X, Y, W.codes, W.scales, bias)) return false;
    return made("maxk_mx_matvec", [&, s = stream()](const char*) {
        return matvec_call(X->data_ptr(), value_type(*X), X->size(0), W.code(), W.scale(), (int32_t)X->size(1), (int32_t)Y->size(1), floats(bias), Y->data_ptr(),
                           value_type(*Y), s);
    });
}

bool rms_norm(const py::handle& X_, const py::handle& gamma_, const py::handle& Y_, const py::handle& codes_, const py::handle& scales_,
              const py::handle& residual_, const py::handle& H_, const py::handle& rstd_, double eps)
{
    const at::Tensor* X = rows(X_, MAXK_NORM_MAX_DIM);
    if (!X) return false;
    const int64_t N = X->size(0), dim = X->size(1);
    Optionals given;
    const at::Tensor *gamma = vector(gamma_, dim), *Y = given.like(Y_, *X), *residual = given.like(residual_, *X), *H = given.like(H_, *X),
                     *rstd = given.floats(rstd_, N);
    Stored to = {};
    if (!codes_.is_none()) {
        to = stored(codes_, scales_, N, dim, false);
        given.good &= (bool)to;
    } else {
        given.good &= scales_.is_none();
    }
    if (!given.good || !gamma || !residual != !H || (!Y && !to) || !here(X, gamma, Y, to.codes, to.scales, residual, H, rstd)) return false;
    return made("maxk_rms_norm", [&, s = stream()](const char*) {
        return rms_norm_call(X->data_ptr(), address(residual), value_type(*X), N, (int32_t)dim, floats(gamma), eps, place(H), place(Y), to ? to.format : 0,
                             place(to.codes), static_cast<uint8_t*>(place(to.scales)), floats(rstd), s);
    });
}

bool rms_norm_grad(const py::handle& dY_, const py::handle& H_, const py::handle& gamma_, const py::handle& rstd_, const py::handle& dX_,
                   const py::handle& dgamma_, const py::handle& dH_, const py::handle& workspace_)
{
    const at::Tensor* H = rows(H_, MAXK_NORM_MAX_DIM);
    if (!H) return false;
    const int64_t N = H->size(0), dim = H->size(1);
    Optionals given;
    const at::Tensor *dY = given.like(dY_, *H), *dX = given.like(dX_, *H), *dH = given.like(dH_, *H), *dgamma = given.floats(dgamma_, dim),
                     *gamma = vector(gamma_, dim), *rstd = vector(rstd_, N), *workspace;
    if (!given.good || !dY || !dX || !gamma || !rstd || !here(H, dY, dX, dH, dgamma, gamma, rstd)) return false;
    at::Tensor own;
    if (!workspace_for(workspace_, dgamma ? rms_norm_grad_workspace_call(N, (int32_t)dim) : 0, *H, own, workspace)) return false;
    return made("maxk_rms_norm_grad", [&, s = stream()](const char*) {
        return rms_norm_grad_call(dY->data_ptr(), H->data_ptr(), address(dH), value_type(*H), N, (int32_t)dim, floats(gamma), floats(rstd), dX->data_ptr(),
                                  floats(dgamma), place(workspace), room(workspace), s);
    });
}

bool logprobs(const py::handle& logits_, const py::handle& labels_, const py::handle& logprob_, const py::handle& entropy_, const py::handle& data_,
              const py::handle& index_, const py::handle& workspace_)
{
    const at::Tensor* logits = rows(logits_, MAXK_MAX_CLASSES);
    if (!logits) return false;
    const int64_t N = logits->size(0), V = logits->size(1);
    Optionals given;
    const at::Tensor *labels = given.labels(labels_, N), *logprob = given.floats(logprob_, N), *entropy = given.floats(entropy_, N), *data = nullptr,
                     *index = nullptr, *workspace;
    int64_t k = 0;
    if (!data_.is_none()) {
        data = matrix(data_, N, -1);
        if (!data || data->scalar_type() != at::kFloat) return false;
        k = data->size(1);
        index = matrix(index_, N, k);
        if (!index || !index_bytes(*index) || k < 1 || k > MAXK_MAX_ALTERNATIVES) return false;
    } else if (!index_.is_none()) {
        return false;
    }
    if (!given.good || (logprob && !labels) || (!logprob && !entropy && !data) || !here(logits, labels, logprob, entropy, data, index)) return false;
    at::Tensor own;
    if (!workspace_for(workspace_, classes_workspace_call(N, (int32_t)V, (int32_t)k), *logits, own, workspace)) return false;
    return made("maxk_logprobs", [&, s = stream()](const char*) {
        return logprobs_call(logits->data_ptr(), value_type(*logits), N, (int32_t)V, address(labels), label_bytes(labels), floats(logprob), floats(entropy),
                             floats(data), place(index), index ? index_bytes(*index) : 0, (int32_t)k, place(workspace), room(workspace), s);
    });
}

bool logprobs_grad(const py::handle& logits_, const py::handle& dlogits_, const py::handle& labels_, const py::handle& dlogprob_, const py::handle& dentropy_,
                   const py::handle& logprob_, const py::handle& entropy_, const py::handle& workspace_)
{
    const at::Tensor* logits = rows(logits_, MAXK_MAX_CLASSES);
    if (!logits) return false;
    const int64_t N = logits->size(0), V = logits->size(1);
    Optionals given;
    const at::Tensor *labels = given.labels(labels_, N), *dlogprob = given.floats(dlogprob_, N), *dentropy = given.floats(dentropy_, N),
                     *logprob = given.floats(logprob_, N), *entropy = given.floats(entropy_, N), *dlogits = given.like(dlogits_, *logits), *workspace;
    if (!given.good || !dlogits || (!dlogprob && !dentropy) || ((dlogprob || logprob) && !labels) ||
        !here(logits, dlogits, labels, dlogprob, dentropy, logprob, entropy))
        return false;
    at::Tensor own;
    if (!workspace_for(workspace_, classes_workspace_call(N, (int32_t)V, 0), *logits, own, workspace)) return false;
    return made("maxk_logprobs_grad", [&, s = stream()](const char*) {
        return logprobs_grad_call(logits->data_ptr(), value_type(*logits), N, (int32_t)V, address(labels), label_bytes(labels), floats(dlogprob), floats(dentropy),
                                  floats(logprob), floats(entropy), dlogits->data_ptr(), place(workspace), room(workspace), s);
    });
}

// the loss, or (dlogits_ not None) its gradient
bool distill(const py::handle& logits_, const py::handle& data_, const py::handle& index_, const py::handle& dloss_, const py::handle& dlogits_,
             double temperature, const py::handle& loss_, const py::handle& workspace_)
{
    const at::Tensor *logits = rows(logits_, MAXK_MAX_CLASSES), *data = rows(data_, MAXK_DISTILL_MAX_K);
    if (!logits || !data || data->size(0) != logits->size(0)) return false;
    const int64_t N = logits->size(0), V = logits->size(1), k = data->size(1);
    const at::Tensor* index = matrix(index_, N, k);
    if (!index || !index_bytes(*index)) return false;
    Optionals given;
    const at::Tensor *dloss = given.floats(dloss_, N), *loss = given.floats(loss_, N), *dlogits = given.like(dlogits_, *logits), *workspace;
    if (!given.good || (dlogits ? !dloss : !loss) || !here(logits, data, index, dloss, loss, dlogits)) return false;
    at::Tensor own;
    if (!workspace_for(workspace_, classes_workspace_call(N, (int32_t)V, 0), *logits, own, workspace)) return false;
    return made(dlogits ? "maxk_distill_grad" : "maxk_distill", [&, s = stream()](const char*) {
        const int32_t v = (int32_t)V, n = (int32_t)k;
        if (dlogits)
            return distill_grad_call(logits->data_ptr(), value_type(*logits), N, v, data->data_ptr(), value_type(*data), index->data_ptr(), index_bytes(*index), n,
                                     temperature, floats(dloss), floats(loss), dlogits->data_ptr(), place(workspace), room(workspace), s);
        return distill_call(logits->data_ptr(), value_type(*logits), N, v, data->data_ptr(), value_type(*data), index->data_ptr(), index_bytes(*index), n,
                            temperature, floats(loss), place(workspace), room(workspace), s);
    });
}

}  // namespace

PYBIND11_MODULE(_torch_calls, m)
{
    m.def("bind", &bind);
    m.def("topk", &topk);
    m.def("forward", &forward);
    m.def("forward_noalloc", &forward_noalloc);
    m.def("backward", &backward);
    m.def("scatter", &scatter);
    m.def("aggregate_forward", &aggregate_forward);
    m.def("aggregate_backward", &aggregate_backward);
    m.def("mx_quantize", &mx_quantize);
    m.def("mx_dequantize", &mx_dequantize);
    m.def("mx_linear", &mx_linear);
    m.def("mx_weight_grad", &mx_weight_grad);
    m.def("mx_input_grad", &mx_input_grad);
    m.def("mx_matvec", &mx_matvec);
    m.def("rms_norm", &rms_norm);
    m.def("rms_norm_grad", &rms_norm_grad);
    m.def("logprobs", &logprobs);
    m.def("logprobs_grad", &logprobs_grad);
    m.def("distill", &distill);
}
