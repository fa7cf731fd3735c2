// What the sources of kla_binding.so share: how a tensor is taken from a Python object, or from the autograd graph.
#pragma once
#include <Python.h>

#include <pybind11/pybind11.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <climits>
#include <initializer_list>
#include <optional>

#include "../../include/kla.h"

namespace kla_binding {

// A plain tensor: torch.Tensor or Parameter itself, strided, with memory of its own.  (What function transforms and fake modes pass
// around is not.)
inline const at::Tensor* plain(const at::Tensor& t)
{
    if (!t.defined() || t.layout() != at::kStrided) return nullptr;
    const c10::TensorImpl* impl = t.unsafeGetTensorImpl();
    const c10::DispatchKeySet ks = impl->key_set();
    if (!impl->has_storage() || impl->is_python_dispatch() || ks.has(c10::DispatchKey::FuncTorchBatched) ||
        ks.has(c10::DispatchKey::FuncTorchGradWrapper) || ks.has(c10::DispatchKey::Functionalize))
        return nullptr;
    return &t;
}
inline const at::Tensor* plain(PyObject* o) { return THPVariable_CheckExact(o) ? plain(THPVariable_Unpack(o)) : nullptr; }
// the same, contiguous
template <typename O> const at::Tensor* dense(const O& o)
{
    const at::Tensor* t = plain(o);
    return t && t->is_contiguous() ? t : nullptr;
}
template <typename O> const at::Tensor* on_gpu(const O& o)
{
    const at::Tensor* t = dense(o);
    return t && t->is_cuda() ? t : nullptr;
}
// GPU tensor of this element type and these extents
template <typename O> const at::Tensor* gpu(const O& o, at::ScalarType type, at::IntArrayRef shape)
{
    const at::Tensor* t = on_gpu(o);
    return t && t->scalar_type() == type && t->sizes() == shape ? t : nullptr;
}
inline bool is_none(PyObject* o) { return o == Py_None; }
inline bool is_none(const at::Tensor& t) { return !t.defined(); }
// the same, or None (then *t stays null); false: neither
template <typename O> bool gpu_or_none(const O& o, at::ScalarType type, at::IntArrayRef shape, const at::Tensor** t)
{
    *t = nullptr;
    if (is_none(o)) return true;
    *t = gpu(o, type, shape);
    return *t != nullptr;
}
// What a forward left behind for the backward of q: bytes on q's device, or none (then *t stays null); false: something else.
// (It comes back through the caller's hands, a hook on saved tensors, and goes to the kernels as a bare pointer.)
template <typename O> bool saved_or_none(const O& o, const at::Tensor& q, const at::Tensor** t)
{
    *t = nullptr;
    if (is_none(o)) return true;
    *t = on_gpu(o);
    return *t && (*t)->scalar_type() == at::kByte && (*t)->device() == q.device();
}
inline void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
inline float* fptr(const at::Tensor* t) { return static_cast<float*>(ptr(t)); }

// Tensors of the caller's that a call has written through their bare pointers (null: not given): what the graph saved of them has
// changed, and its backward has to find out.  (An inference tensor does not count its changes.)
inline void written(std::initializer_list<const at::Tensor*> ts)
{
    for (const at::Tensor* t : ts) if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

inline bool type_of(const at::Tensor& q, kla_dtype* dt)
{
    if (q.scalar_type() == at::kBFloat16) *dt = KLA_BF16;
    else if (q.scalar_type() == at::kFloat) *dt = KLA_F32;
    else return false;
    return true;
}
inline bool number(PyObject* o, double* x)
{
    *x = PyFloat_AsDouble(o);
    if (*x == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}
inline bool integer(PyObject* o, long lo, long hi, long* x)
{
    *x = PyLong_AsLong(o);
    if (*x == -1 && PyErr_Occurred()) { PyErr_Clear(); return false; }
    return *x >= lo && *x <= hi;
}
inline bool ints(std::initializer_list<int64_t> xs)
{
    for (const int64_t x : xs) if (x > INT_MAX) return false;
    return true;
}
inline void* stream() { return c10::hip::getCurrentHIPStream().stream(); }
// Other threads run while a call allocates and launches (and get their turn back if it throws).
struct NoGil {
    PyThreadState* state = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(state); }
};
inline PyObject* wrap(const std::optional<at::Tensor>& t)
{
    if (t) return THPVariable_Wrap(*t);
    Py_RETURN_NONE;
}

#define KLA_FASTCALL(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}

// The entry points of the operators around the recurrence (kla_layer_binding.cpp), ended by an entry without a name
extern PyMethodDef layer_methods[];
// and those of attention (kla_attn_binding.cpp)
extern PyMethodDef attn_methods[];

}  // namespace kla_binding
