// What the sources of kla_binding.so that bind operators on rows share (kla_layer_binding.cpp, kla_attn_binding.cpp): tensors whose rows are evenly
// spaced, packed batches, new tensors, and a node's backward.
#pragma once
#include <c10/hip/HIPFunctions.h>

#include "kla_binding.hpp"

namespace kla_binding {
namespace {

template <typename F> bool address(PyObject* o, F* f)
{
    void* p = PyLong_AsVoidPtr(o);
    if (!p && !PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
    *f = reinterpret_cast<F>(p);
    return p != nullptr;
}

// ---- tensors ------------------------------------------------------------------------------------------------------------------------
// Rows (the last `inner` dimensions, contiguous) evenly spaced: *ld elements from one to the next; false: they are not.
bool row_stride(const at::Tensor& t, int inner, long* ld)
{
    const auto size = t.sizes(), stride = t.strides();
    const int dims = (int)size.size();
    int64_t row = 1, step = -1, count = 1;
    for (int i = dims - 1; i >= dims - inner; --i) {
        if (size[i] != 1 && stride[i] != row && t.numel()) return false;
        row *= size[i];
    }
    for (int i = dims - inner - 1; i >= 0; --i) {
        if (size[i] != 1) {
            if (step >= 0 && stride[i] != step * count && t.numel()) return false;
            if (step < 0) step = stride[i];
        }
        count *= size[i];
    }
    if (step < 0) step = row;
    if (step < row && t.numel()) return false;
    *ld = (long)(step > row ? step : row);
    return true;
}
// GPU tensor of this type and these extents whose rows are evenly spaced
template <typename O> const at::Tensor* rows(const O& o, at::ScalarType type, at::IntArrayRef shape, int inner, long* ld)
{
    const at::Tensor* t = plain(o);
    return t && t->is_cuda() && t->scalar_type() == type && t->sizes() == shape && row_stride(*t, inner, ld) ? t : nullptr;
}
// the same, or none (then *t stays null); false: neither
template <typename O> bool rows_or_none(const O& o, at::ScalarType type, at::IntArrayRef shape, int inner, long* ld, const at::Tensor** t)
{
    *t = nullptr;
    *ld = 0;
    if (is_none(o)) return true;
    *t = rows(o, type, shape, inner, ld);
    return *t != nullptr;
}
// all on the current device
bool together(std::initializer_list<const at::Tensor*> ts)
{
    const auto device = c10::hip::current_device();
    for (const at::Tensor* t : ts) if (t && t->device().index() != device) return false;
    return true;
}
bool wants(std::initializer_list<const at::Tensor*> ts)
{
    if (!c10::GradMode::is_enabled()) return false;
    for (const at::Tensor* t : ts) if (t && t->requires_grad()) return true;
    return false;
}
at::Tensor value(const at::Tensor* t) { return t ? *t : at::Tensor(); }
std::optional<at::Tensor> maybe(const at::Tensor* t) { return t ? std::optional<at::Tensor>(*t) : std::nullopt; }
at::Tensor fresh(const at::Tensor& like, at::IntArrayRef shape, at::ScalarType type) { return at::empty(shape, like.options().dtype(type).requires_grad(false)); }
at::Tensor fresh(const at::Tensor* like) { return like ? fresh(*like, like->sizes(), like->scalar_type()) : at::Tensor(); }
at::Tensor bytes(const at::Tensor& like, size_t n) { return n ? fresh(like, {(int64_t)n}, at::kByte) : at::Tensor(); }
void* at_of(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
float* f_of(const at::Tensor& t) { return static_cast<float*>(at_of(t)); }
size_t size_of(const at::Tensor& t) { return t.defined() ? t.nbytes() : 0; }
PyObject* wrap(const at::Tensor& t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}
PyObject* pair(const at::Tensor& a, const at::Tensor& b)
{
    PyObject* r = PyTuple_New(2);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, wrap(a));
    PyTuple_SET_ITEM(r, 1, wrap(b));
    return r;
}
struct Refused { int code; };                            // by the library: handed back as its status code
void check(int rc) { if (rc != KLA_OK) throw Refused{rc}; }

// In the backward of a node: what comes back from hooks on saved tensors, and the library's answer.
#define KLA_BACKWARD(name)                                                                                                         \
    TORCH_CHECK(!c10::GradMode::is_enabled(), name ": the gradients have no gradients of their own (create_graph)")
void taken(bool ok, const char* name) { TORCH_CHECK(ok, name, ": the saved tensors are not those of the forward"); }
template <typename F> void refused(const char* name, F&& f)
{
    try { f(); } catch (const Refused& e) { TORCH_CHECK(false, name, " failed with status ", e.code); }
}

// The offsets of a packed batch
struct Offsets {
    const at::Tensor* dev = nullptr;
    const int32_t* host = nullptr;
    int n_seq = 0;
    template <typename O> bool take(const O& cu_, const O& host_)
    {
        if (is_none(cu_)) return is_none(host_);
        dev = on_gpu(cu_);
        const at::Tensor* h = dense(host_);
        if (!dev || !h || !h->is_cpu() || dev->scalar_type() != at::kInt || h->scalar_type() != at::kInt || dev->dim() != 1 || h->dim() != 1 ||
            dev->numel() != h->numel() || dev->numel() < 2 || dev->numel() > INT_MAX)
            return false;
        host = static_cast<const int32_t*>(h->data_ptr());
        n_seq = (int)dev->numel() - 1;
        return true;
    }
    const int32_t* device() const { return static_cast<const int32_t*>(ptr(dev)); }
    // For the backward: a host copy of our own (the caller may fill its own anew), and the device's unchanged (an inference tensor does
    // not count its changes).
    void keep(torch::autograd::AutogradContext* ctx, const at::Tensor* host_tensor) const
    {
        if (!dev) return;
        const at::Tensor cu = dev->is_inference() ? dev->clone() : *dev;
        ctx->saved_data["cu"] = cu;
        ctx->saved_data["cu_version"] = (int64_t)cu._version();
        ctx->saved_data["cu_host"] = host_tensor->clone();
    }
    static void back(torch::autograd::AutogradContext* ctx, at::Tensor* dev, at::Tensor* host)
    {
        const auto cu = ctx->saved_data.find("cu");
        if (cu == ctx->saved_data.end()) return;
        *dev = cu->second.toTensor();
        *host = ctx->saved_data["cu_host"].toTensor();
        TORCH_CHECK((int64_t)dev->_version() == ctx->saved_data["cu_version"].toInt(),
                    "one of the variables needed for gradient computation has been modified by an inplace operation: cu_seqlens");
    }
};

}  // namespace
}  // namespace kla_binding
