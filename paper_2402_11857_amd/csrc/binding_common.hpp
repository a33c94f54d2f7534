// What the Python sides of the operators' headers share: tensors, checks, the call, and how errors leave a function.
//
// Types that do not fit raise TypeError, shapes and strides ValueError, what the library refuses its own error class; no C++
// exception leaves a function.
#pragma once
#include <torch/extension.h>

#include <algorithm>
#include <new>
#include <string>

#include "liec_train.h"

namespace liec_binding {

inline PyObject* g_error = nullptr;       // raised with (status, name) where the library refuses
inline PyObject* g_stream = nullptr;      // device index -> hipStream_t as an int

struct Raise {                     // a Python error to raise; what == "": it has been set already
    PyObject* type;
    std::string what;
};
[[noreturn]] inline void type_error(const std::string& s) { throw Raise{PyExc_TypeError, s}; }
[[noreturn]] inline void value_error(const std::string& s) { throw Raise{PyExc_ValueError, s}; }

inline std::string text(at::IntArrayRef s) {
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + (s.size() == 1 ? ",)" : ")");
}

inline const at::Tensor* optional_tensor(PyObject* o, const char* what) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) type_error(std::string(what) + " must be a tensor");
    return &THPVariable_Unpack(o);
}
inline const at::Tensor& tensor(PyObject* o, const char* what) {
    const at::Tensor* t = optional_tensor(o, what);
    if (!t) type_error(std::string(what) + " must be a tensor");
    return *t;
}
inline double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raise{nullptr, ""};
    return v;
}

inline int code_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return LIEC_F32;
        case at::kBFloat16: return LIEC_BF16;
        case at::kHalf: return LIEC_F16;
        default: return -1;
    }
}

inline at::Tensor new_tensor(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
    return at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
}

// A call has written to t: automatic differentiation refuses to use what it saved of it.
inline void written(const at::Tensor* t) {
    if (t && t->defined() && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

inline void* stream_of(const at::Tensor& t) {
    PyObject* const index = PyLong_FromLong(t.get_device());
    PyObject* const s = index ? PyObject_CallOneArg(g_stream, index) : nullptr;
    Py_XDECREF(index);
    if (!s) throw Raise{nullptr, ""};
    void* const r = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (!r && PyErr_Occurred()) throw Raise{nullptr, ""};
    return r;
}

// Calls an entry point with the tensors' device current and the interpreter free for other threads.
template <typename F>
void call(const char* name, const at::Tensor& on, F f) {
    const c10::DeviceGuard guard(on.device());
    liec_status status;
    Py_BEGIN_ALLOW_THREADS;
    status = f();
    Py_END_ALLOW_THREADS;
    if (status == LIEC_OK) return;
    PyObject* const e = PyObject_CallFunction(g_error, "is", (int)status, name);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Raise{nullptr, ""};
}

inline float* data_of(const at::Tensor* t) { return t ? static_cast<float*>(t->data_ptr()) : nullptr; }

// The distance of dimensions [from, to) of t seen as one; false where they are not evenly spaced.
inline bool merged(const at::Tensor& t, int64_t from, int64_t to, int64_t* stride) {
    int64_t next = -1;                 // what the next dimension's distance has to be; -1: any
    *stride = 0;
    for (int64_t d = to - 1; d >= from; --d) {
        if (t.size(d) == 1) continue;
        if (next < 0) *stride = t.stride(d);
        else if (t.stride(d) != next) return false;
        next = t.stride(d) * t.size(d);
    }
    return true;
}

inline void check_like(const at::Tensor& t, const at::Tensor& x, const char* what) {
    if (t.scalar_type() != x.scalar_type() || t.device() != x.device()) type_error(std::string(what) + " must have the activations' type and device");
    if (t.sizes() != x.sizes()) value_error(std::string(what) + " has shape " + text(t.sizes()) + ", expected " + text(x.sizes()));
}

// The type of the weights, biases and their gradients that are there.
inline int params_code(const at::Tensor& x, std::initializer_list<const at::Tensor*> params) {
    int code = -1;
    for (const at::Tensor* p : params) {
        if (!p) continue;
        const int c = code_of(*p);
        if (c < 0 || (code >= 0 && c != code) || p->device() != x.device())
            type_error("weights, biases and their gradients must be of one type, float32, bfloat16 or float16, on the activations' GPU");
        code = c;
    }
    return code < 0 ? (int)LIEC_F32 : code;
}

// Gradients with a row for each worker need room for each: one vector seen N times would hold the sum over all of them.
inline void check_rows_apart(const at::Tensor* p, const char* what) {
    if (p && p->dim() == 2 && p->size(0) > 1 && p->stride(0) == 0)
        value_error(std::string(what) + " is an expanded tensor, which cannot hold a sum for each worker: pass one vector for the sum over all of them");
}

inline liec_param param_of(const at::Tensor* p) { return p ? liec_param{p->data_ptr(), p->dim() == 2 ? p->stride(0) : 0} : liec_param{nullptr, 0}; }

inline int activations_code(const at::Tensor& x) {
    const int code = code_of(x);
    if (code < 0 || !x.is_cuda()) type_error("activations must be float32, bfloat16 or float16 on the GPU");
    return code;
}

struct Sizes {
    int64_t N, R, C;
    int64_t split;                     // dimensions before this one are the workers', those from it up to the columns the rows'
};

// t as workers' rows; false where no two distances describe it.
inline bool as_rows(const at::Tensor& t, const Sizes& s, liec_rows* r) {
    r->data = t.data_ptr();
    r->worker_stride = s.R * s.C;
    r->row_stride = s.C;
    if (t.is_contiguous()) return true;
    return merged(t, 0, s.split, &r->worker_stride) && merged(t, s.split, t.dim() - 1, &r->row_stride);
}

// Workers, rows of each and columns of activations x under these weights, biases and their gradients (some of them nullptr).  Where
// none of them has rows for the workers any split of the dimensions will do: the first that all operands are laid out for.
inline Sizes sizes_of(const at::Tensor& x, std::initializer_list<const at::Tensor*> params, std::initializer_list<const at::Tensor*> operands) {
    const int64_t dims = x.dim(), C = dims ? x.size(-1) : 0;
    if (C < 1) value_error("activations of shape " + text(x.sizes()) + " have no columns");
    int64_t N = 0;
    for (const at::Tensor* p : params) {
        if (!p) continue;
        if (p->dim() < 1 || p->dim() > 2 || p->size(-1) != C || (C > 1 && p->stride(-1) != 1))
            value_error("a weight or bias of shape " + text(p->sizes()) + " does not fit " + std::to_string(C) + " columns, or its columns are not contiguous");
        if (p->dim() == 2) {
            N = p->size(0);
            if (dims < 2 || N != x.size(0) || !N) value_error("weights of " + std::to_string(N) + " workers do not fit activations of shape " + text(x.sizes()));
        }
    }
    const int64_t rows = x.numel() / C;
    if (N) return {N, rows / N, C, 1};
    N = 1;
    for (int64_t split = 0; rows && split < std::max<int64_t>(1, dims - 1); N *= x.size(split++)) {
        const Sizes s{N, rows / N, C, split};
        bool all = N <= 65535 && s.R < ((int64_t)1 << 31);       // what the library takes
        liec_rows r;
        for (const at::Tensor* t : operands) all = all && (!t || as_rows(*t, s, &r));
        if (all) return s;
    }
    return {1, rows, C, 0};
}

inline liec_rows rows_of(const at::Tensor& t, const Sizes& s, const char* what) {
    if (s.C > 1 && t.stride(-1) != 1 && !t.is_contiguous()) value_error(std::string("the columns of ") + what + " must be contiguous");
    liec_rows r;
    if (!as_rows(t, s, &r))
        value_error(std::string(what) + " of strides " + text(t.strides()) + " is not " + std::to_string(s.N) + " workers' rows at equal distances");
    return r;
}

inline int32_t workers_of(const Sizes& s) {
    if (s.N > 65535) value_error(std::to_string(s.N) + " workers are more than the library takes");
    return (int32_t)s.N;
}

template <PyObject* (*F)(PyObject* const*), Py_ssize_t ARGS>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != ARGS) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", ARGS, n);
        return nullptr;
    }
    if (!g_error) {
        PyErr_SetString(PyExc_RuntimeError, "the library has not been loaded");
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Raise& e) {
        if (!e.what.empty()) PyErr_SetString(e.type, e.what.c_str());
    } catch (const std::bad_alloc&) {
        PyErr_NoMemory();
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

template <typename F>
PyCFunction as_method(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)); }

}  // namespace liec_binding
