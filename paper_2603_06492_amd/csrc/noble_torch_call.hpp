// Calls on torch tensors in native code, as the bindings of the attention and the decoding side make them: the checks of one
// call's arguments, its outputs and its scratch.  A binding includes it once.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "noble_attn.h"

namespace {

// Releases the GIL for its lifetime.
struct NoGil {
    PyThreadState* s = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(s); }
};

// An ordinary strided CUDA tensor, or nullptr (anything else).
const at::Tensor* plain(PyObject* o) {
    static const c10::DispatchKeySet special({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched,
                                              c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize,
                                              c10::DispatchKey::Conjugate, c10::DispatchKey::Negative,
                                              c10::DispatchKey::ZeroTensor});
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != c10::kStrided || !t.device().is_cuda() || !t.has_storage() ||
        t.key_set().has_any(special))
        return nullptr;
    return &t;
}

// The arguments of one call as they are checked; ok turns false at the first that the native path does not take.
struct Call {
    bool ok = !c10::impl::TorchDispatchModeTLS::any_modes_set();
    at::Device dev{c10::kCUDA};
    at::ScalarType sd = at::kBFloat16;
    int32_t dtype = NOBLE_BF16;

    const at::Tensor* tensor(PyObject* o) {
        const at::Tensor* t = ok ? plain(o) : nullptr;
        if (!t) ok = false;
        return t;
    }
    // The tensor that sets the call's device and storage type.
    const at::Tensor* first(PyObject* o) {
        const at::Tensor* t = tensor(o);
        if (!t) return nullptr;
        dev = t->device();
        sd = t->scalar_type();
        ok = sd == at::kBFloat16 || sd == at::kFloat;
        dtype = sd == at::kBFloat16 ? NOBLE_BF16 : NOBLE_F32;
        return ok ? t : nullptr;
    }
    // Data pointer of a dense argument of the given dtype and shape (None: NULL).
    void* dense(PyObject* o, at::ScalarType dt, std::initializer_list<int64_t> shape) {
        if (o == Py_None || !ok) return nullptr;
        const at::Tensor* t = tensor(o);
        if (!t || t->scalar_type() != dt || t->device() != dev || !t->is_contiguous() || !t->sizes().equals(shape)) {
            ok = false;
            return nullptr;
        }
        return t->data_ptr();
    }
    float* floats(PyObject* o, std::initializer_list<int64_t> shape) {
        return static_cast<float*>(dense(o, at::kFloat, shape));
    }
    int32_t* ints(PyObject* o, std::initializer_list<int64_t> shape) {
        return static_cast<int32_t*>(dense(o, at::kInt, shape));
    }
    // A [rows, heads, D] tensor of the storage type with adjacent elements of a head.
    noble_heads heads(PyObject* o, int64_t rows, int64_t n, int64_t D) {
        const at::Tensor* t = tensor(o);
        if (!t || t->scalar_type() != sd || t->device() != dev || t->dim() != 3 || t->size(0) != rows || t->size(1) != n ||
            t->size(2) != D || (D > 1 && t->stride(2) != 1)) {
            ok = false;
            return {};
        }
        return {t->data_ptr(), rows > 1 ? t->stride(0) : 0, n > 1 ? t->stride(1) : 0};
    }
    int64_t integer(PyObject* o, int64_t lo, int64_t hi) {
        int wide = 0;
        const int64_t v = ok && PyLong_CheckExact(o) ? PyLong_AsLongAndOverflow(o, &wide) : (ok = false, 0);
        if (wide || v < lo || v > hi) ok = false;
        return v;
    }
    bool truth(PyObject* o) {
        if (o != Py_True && o != Py_False) ok = false;
        return o == Py_True;
    }
    float number(PyObject* o) {
        if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
        ok = false;
        return 0.f;
    }
    float scale(PyObject* o, int64_t D) { return o == Py_None ? (float)std::pow((double)D, -0.5) : number(o); }
    void* stream() const { return at::hip::getCurrentHIPStreamMasqueradingAsCUDA(dev.index()).stream(); }
    at::Tensor empty(c10::IntArrayRef shape, at::ScalarType dt) const {
        return at::empty(shape, at::TensorOptions().dtype(dt).device(dev));
    }
    at::Tensor work(size_t n) const { return empty({(int64_t)std::max<size_t>(n, 16)}, at::kByte); }
};

// A given output, or a new one; `t` keeps it.
struct Output {
    at::Tensor t;
    Output(Call& c, PyObject* given, c10::IntArrayRef shape, at::ScalarType dt) {
        if (!c.ok) return;
        if (given == Py_None) {
            t = c.empty(shape, dt);
            return;
        }
        const at::Tensor* g = c.tensor(given);
        if (g && g->scalar_type() == dt && g->device() == c.dev && g->sizes().equals(shape)) t = *g;
        else c.ok = false;
    }
    void* dense(Call& c) const {
        if (c.ok && !t.is_contiguous()) c.ok = false;
        return c.ok ? t.data_ptr() : nullptr;
    }
    noble_heads heads(Call& c) const {
        if (!c.ok || (t.size(2) > 1 && t.stride(2) != 1)) {
            c.ok = false;
            return {};
        }
        return {t.data_ptr(), t.size(0) > 1 ? t.stride(0) : 0, t.size(1) > 1 ? t.stride(1) : 0};
    }
};

PyObject* tuple(std::initializer_list<const at::Tensor*> ts) {
    PyObject* out = PyTuple_New((Py_ssize_t)ts.size());
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor* t : ts) {
        PyObject* o = t->defined() ? THPVariable_Wrap(*t) : Py_None;
        if (!t->defined()) Py_INCREF(o);
        PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}

}  // namespace

#define NOBLE_FAST(fn) {#fn, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
