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

PyObject* check;  // (status, name of the call): raises; held for good

void bind(const std::vector<uintptr_t>& at, const py::function& raise)
{
    TORCH_CHECK(at.size() == 13, "thirteen addresses");
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
}
