// Python side of include/liec_train.h: argument checks, outputs, scratch and the call, in one step per operator.  A call through
// ctypes with the checks in Python cost the host 15 to 25 us, more than the GPU needs for small tensors; this takes 6 to 10.
//
// The entry points' addresses come from the library that binding.py has loaded.  Types that do not fit raise TypeError, shapes
// and strides ValueError, what the library refuses its own error class; no C++ exception leaves a function.
#include <torch/extension.h>

#include <algorithm>
#include <new>
#include <string>
#include <vector>

#include "liec_train.h"

namespace {

decltype(&liec_grads_workspace) p_grads_workspace;
decltype(&liec_grad_norm) p_grad_norm;
decltype(&liec_clip_grads) p_clip_grads;
decltype(&liec_gather_grads) p_gather_grads;
decltype(&liec_layer_norm) p_layer_norm;
decltype(&liec_layer_norm_workspace) p_layer_norm_workspace;
decltype(&liec_layer_norm_backward) p_layer_norm_backward;
PyObject* g_error = nullptr;       // raised with (status, name) where the library refuses
PyObject* g_stream = nullptr;      // device index -> hipStream_t as an int

struct Raise {                     // a Python error to raise; what == "": it has been set already
    PyObject* type;
    std::string what;
};
[[noreturn]] void type_error(const std::string& s) { throw Raise{PyExc_TypeError, s}; }
[[noreturn]] void value_error(const std::string& s) { throw Raise{PyExc_ValueError, s}; }

std::string text(at::IntArrayRef s) {
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + (s.size() == 1 ? ",)" : ")");
}

const at::Tensor* optional_tensor(PyObject* o, const char* what) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) type_error(std::string(what) + " must be a tensor");
    return &THPVariable_Unpack(o);
}
const at::Tensor& tensor(PyObject* o, const char* what) {
    const at::Tensor* t = optional_tensor(o, what);
    if (!t) type_error(std::string(what) + " must be a tensor");
    return *t;
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raise{nullptr, ""};
    return v;
}

int code_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return LIEC_F32;
        case at::kBFloat16: return LIEC_BF16;
        case at::kHalf: return LIEC_F16;
        default: return -1;
    }
}

at::Tensor new_tensor(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
    return at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
}

// A call has written to t: automatic differentiation refuses to use what it saved of it.
void written(const at::Tensor* t) {
    if (t && t->defined() && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

void* stream_of(const at::Tensor& t) {
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

// ---- gradients -------------------------------------------------------------------------------------------------------
struct Grads {
    PyObject* sequence = nullptr;      // a tuple of the tensors, held while they are used
    std::vector<liec_grad_tensor> table;
    int64_t total = 0;
    int32_t N = 0;
    const at::Tensor* first = nullptr;
    at::Tensor workspace;
    int64_t bytes = 0;
    ~Grads() { Py_XDECREF(sequence); }
    void written_all() const {
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(sequence); ++i) written(&THPVariable_Unpack(PyTuple_GET_ITEM(sequence, i)));
    }
};

void read_grads(Grads& g, PyObject* list, const at::Tensor* norms, bool whole) {
    if (THPVariable_Check(list)) type_error("gradients must be a sequence of tensors, not a tensor");
    PyObject* const fast = PySequence_Fast(list, "gradients must be a sequence of tensors");
    g.sequence = fast ? PySequence_Tuple(fast) : nullptr;
    Py_XDECREF(fast);
    if (!g.sequence) throw Raise{nullptr, ""};
    const Py_ssize_t T = PyTuple_GET_SIZE(g.sequence);
    if (T > LIEC_GRAD_MAX_TENSORS) value_error(std::to_string(T) + " tensors are more than the library takes");
    if (!T && !norms) value_error("no gradients, and no norms to tell the number of workers");
    g.first = T ? &tensor(PyTuple_GET_ITEM(g.sequence, 0), "a gradient") : norms;
    const c10::Device device = g.first->device();
    if (!g.first->is_cuda()) type_error("gradients must be on the GPU");
    if (norms) {
        if (norms->scalar_type() != at::kFloat || norms->device() != device || norms->dim() != 1 || !norms->is_contiguous())
            type_error("norms must be a contiguous float32 vector on the gradients' GPU");
    }
    const int64_t N = whole ? 1 : norms ? norms->size(0) : g.first->dim() ? g.first->size(0) : 0;
    if (norms && norms->size(0) != N) value_error("norms has " + std::to_string(norms->size(0)) + " values, expected " + std::to_string(N));
    if (N < 1 || N > 65535) value_error(std::to_string(N) + " workers are none, or more than the library takes");
    g.N = (int32_t)N;
    g.table.reserve((size_t)T);
    for (Py_ssize_t i = 0; i < T; ++i) {
        const at::Tensor& t = tensor(PyTuple_GET_ITEM(g.sequence, i), "a gradient");
        const int code = code_of(t);
        if (code < 0 || t.device() != device) type_error("gradients must be float32, bfloat16 or float16 tensors on one GPU");
        int64_t count = t.numel(), stride = count;
        if (whole) {
            if (!t.is_contiguous()) value_error("gradients of one worker must be contiguous");
        } else {
            if (!t.dim() || t.size(0) != N) value_error("a gradient has shape " + text(t.sizes()) + ", expected " + std::to_string(N) + " workers as its leading dimension");
            stride = count /= N;
            if (!t.is_contiguous()) {
                if (!t.select(0, 0).is_contiguous()) value_error("the gradients of a worker must be contiguous within each tensor");
                stride = t.stride(0);
            }
        }
        g.table.push_back(liec_grad_tensor{t.data_ptr(), count, stride, code, 0});
        g.total += count;
    }
    g.bytes = p_grads_workspace(g.N, (int32_t)T);
    if (g.bytes < 0) value_error(std::to_string(T) + " tensors of " + std::to_string(N) + " workers are more than the library takes");
    g.workspace = new_tensor({g.bytes}, at::kByte, *g.first);
}

float* data_of(const at::Tensor* t) { return t ? static_cast<float*>(t->data_ptr()) : nullptr; }

PyObject* grad_norm(PyObject* const* a) {      // grads, norms, whole
    const at::Tensor* norms = optional_tensor(a[1], "norms");
    Grads g;
    read_grads(g, a[0], norms, a[2] == Py_True);
    at::Tensor made;
    if (!norms) {
        made = new_tensor({g.N}, at::kFloat, *g.first);
        norms = &made;
    }
    void* const st = stream_of(*g.first);
    call("liec_grad_norm", *g.first,
         [&] { return p_grad_norm(g.table.data(), (int32_t)g.table.size(), g.N, data_of(norms), g.workspace.data_ptr(), g.bytes, st); });
    if (made.defined()) return THPVariable_Wrap(made);
    written(norms);
    Py_INCREF(a[1]);
    return a[1];
}

PyObject* clip_grads(PyObject* const* a) {     // grads, max_norm, norms, whole
    const at::Tensor* const norms = optional_tensor(a[2], "norms");
    const float bound = (float)number(a[1]);
    Grads g;
    read_grads(g, a[0], norms, a[3] == Py_True);
    void* const st = stream_of(*g.first);
    call("liec_clip_grads", *g.first,
         [&] { return p_clip_grads(g.table.data(), (int32_t)g.table.size(), g.N, bound, data_of(norms), g.workspace.data_ptr(), g.bytes, st); });
    g.written_all();
    written(norms);
    Py_RETURN_NONE;
}

PyObject* gather_grads(PyObject* const* a) {   // grads, rows, max_norm, norms, whole
    const at::Tensor& rows = tensor(a[1], "rows");
    const float bound = (float)number(a[2]);
    const at::Tensor* const norms = optional_tensor(a[3], "norms");
    Grads g;
    read_grads(g, a[0], norms, a[4] == Py_True);
    if (rows.scalar_type() != at::kFloat || rows.device() != g.first->device() || rows.dim() != 2 || (rows.size(1) > 1 && rows.stride(1) != 1))
        type_error("rows must be a float32 [N, d] tensor on the gradients' GPU whose rows are contiguous");
    if (rows.size(0) != g.N || rows.size(1) != g.total)
        value_error("rows has shape " + text(rows.sizes()) + ", expected (" + std::to_string(g.N) + ", " + std::to_string(g.total) + ")");
    void* const st = stream_of(*g.first);
    call("liec_gather_grads", *g.first, [&] {
        return p_gather_grads(g.table.data(), (int32_t)g.table.size(), g.N, static_cast<float*>(rows.data_ptr()), rows.stride(0), bound, data_of(norms),
                              g.workspace.data_ptr(), g.bytes, st);
    });
    written(&rows);
    written(norms);
    Py_RETURN_NONE;
}

// ---- layer normalisation ---------------------------------------------------------------------------------------------
struct Sizes {
    int64_t N, R, C;
    int64_t split;                     // dimensions before this one are the workers', those from it up to the columns the rows'
};

// The distance of dimensions [from, to) of t seen as one; false where they are not evenly spaced.
bool merged(const at::Tensor& t, int64_t from, int64_t to, int64_t* stride) {
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

// t as workers' rows; false where no two distances describe it.
bool as_rows(const at::Tensor& t, const Sizes& s, liec_rows* r) {
    r->data = t.data_ptr();
    r->worker_stride = s.R * s.C;
    r->row_stride = s.C;
    if (t.is_contiguous()) return true;
    return merged(t, 0, s.split, &r->worker_stride) && merged(t, s.split, t.dim() - 1, &r->row_stride);
}

// Workers, rows of each and columns of activations x under these weights, biases and their gradients (some of them nullptr).  Where
// none of them has rows for the workers any split of the dimensions will do: the first that all operands are laid out for.
Sizes sizes_of(const at::Tensor& x, std::initializer_list<const at::Tensor*> params, std::initializer_list<const at::Tensor*> operands) {
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

liec_rows rows_of(const at::Tensor& t, const Sizes& s, const char* what) {
    if (s.C > 1 && t.stride(-1) != 1 && !t.is_contiguous()) value_error(std::string("the columns of ") + what + " must be contiguous");
    liec_rows r;
    if (!as_rows(t, s, &r))
        value_error(std::string(what) + " of strides " + text(t.strides()) + " is not " + std::to_string(s.N) + " workers' rows at equal distances");
    return r;
}

void check_like(const at::Tensor& t, const at::Tensor& x, const char* what) {
    if (t.scalar_type() != x.scalar_type() || t.device() != x.device()) type_error(std::string(what) + " must have the activations' type and device");
    if (t.sizes() != x.sizes()) value_error(std::string(what) + " has shape " + text(t.sizes()) + ", expected " + text(x.sizes()));
}

// The type of the weights, biases and their gradients that are there.
int params_code(const at::Tensor& x, std::initializer_list<const at::Tensor*> params) {
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
void check_rows_apart(const at::Tensor* p, const char* what) {
    if (p && p->dim() == 2 && p->size(0) > 1 && p->stride(0) == 0)
        value_error(std::string(what) + " is an expanded tensor, which cannot hold a sum for each worker: pass one vector for the sum over all of them");
}

liec_param param_of(const at::Tensor* p) { return p ? liec_param{p->data_ptr(), p->dim() == 2 ? p->stride(0) : 0} : liec_param{nullptr, 0}; }

int activations_code(const at::Tensor& x) {
    const int code = code_of(x);
    if (code < 0 || !x.is_cuda()) type_error("activations must be float32, bfloat16 or float16 on the GPU");
    return code;
}

int32_t workers_of(const Sizes& s) {
    if (s.N > 65535) value_error(std::to_string(s.N) + " workers are more than the library takes");
    return (int32_t)s.N;
}

PyObject* layer_norm(PyObject* const* a) {     // x, weight, bias, eps, out
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor *weight = optional_tensor(a[1], "weight"), *bias = optional_tensor(a[2], "bias"), *out = optional_tensor(a[4], "out");
    const double eps = number(a[3]);
    const int code = activations_code(x), pcode = params_code(x, {weight, bias});
    if (out) check_like(*out, x, "out");
    const Sizes s = sizes_of(x, {weight, bias}, {&x, out});
    const at::Tensor y = out ? *out : new_tensor(x.sizes(), x.scalar_type(), x);
    const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
    const at::Tensor mean = new_tensor(lead, at::kFloat, x), rstd = new_tensor(lead, at::kFloat, x);
    const liec_rows xr = rows_of(x, s, "x"), yr = rows_of(y, s, "out");
    const liec_param w = param_of(weight), b = param_of(bias);
    const int32_t N = workers_of(s);
    void* const st = stream_of(x);
    call("liec_layer_norm", x, [&] {
        return p_layer_norm(&xr, &w, &b, &yr, data_of(&mean), data_of(&rstd), N, s.R, s.C, (float)eps, (liec_dtype)code, (liec_dtype)pcode, st);
    });
    written(out);
    if (out) Py_INCREF(a[4]);
    PyObject* const first = out ? a[4] : THPVariable_Wrap(y);
    PyObject* const second = first ? THPVariable_Wrap(mean) : nullptr;
    PyObject* const third = second ? THPVariable_Wrap(rstd) : nullptr;
    PyObject* const r = third ? PyTuple_Pack(3, first, second, third) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    Py_XDECREF(third);
    if (!r) throw Raise{nullptr, ""};
    return r;
}

PyObject* layer_norm_backward(PyObject* const* a) {   // dy, x, mean, rstd, weight, dx, dweight, dbias, need_dx
    const at::Tensor &dy = tensor(a[0], "dy"), &x = tensor(a[1], "x"), &mean = tensor(a[2], "mean"), &rstd = tensor(a[3], "rstd");
    const at::Tensor *weight = optional_tensor(a[4], "weight"), *dweight = optional_tensor(a[6], "dweight"), *dbias = optional_tensor(a[7], "dbias");
    const bool need = a[8] == Py_True;
    const at::Tensor* const given = need ? optional_tensor(a[5], "dx") : nullptr;
    const int code = activations_code(x), pcode = params_code(x, {weight, dweight, dbias});
    check_like(dy, x, "dy");
    if (given) check_like(*given, x, "dx");
    const Sizes s = sizes_of(x, {weight, dweight, dbias}, {&x, &dy, given});
    check_rows_apart(dweight, "dweight");
    check_rows_apart(dbias, "dbias");
    const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
    for (const at::Tensor* t : {&mean, &rstd})
        if (t->scalar_type() != at::kFloat || t->device() != x.device() || t->sizes() != lead || !t->is_contiguous())
            type_error("mean and rstd must be what liec_layer_norm returned");
    const int32_t N = workers_of(s);
    const at::Tensor dx = given ? *given : need ? new_tensor(x.sizes(), x.scalar_type(), x) : at::Tensor();
    at::Tensor ws;
    int64_t bytes = 0;
    if (dweight || dbias) {
        bytes = p_layer_norm_workspace(N, s.R, s.C);
        if (bytes < 0) value_error("activations of shape " + text(x.sizes()) + " are more than the library takes");
        if (bytes) ws = new_tensor({bytes}, at::kByte, x);
    }
    const liec_rows gr = rows_of(dy, s, "dy"), xr = rows_of(x, s, "x"), dr = dx.defined() ? rows_of(dx, s, "dx") : liec_rows{nullptr, 0, 0};
    const liec_param w = param_of(weight), dw = param_of(dweight), db = param_of(dbias);
    void* const st = stream_of(x);
    call("liec_layer_norm_backward", x, [&] {
        return p_layer_norm_backward(&gr, &xr, data_of(&mean), data_of(&rstd), &w, &dr, &dw, &db, N, s.R, s.C, (liec_dtype)code, (liec_dtype)pcode,
                                     bytes ? ws.data_ptr() : nullptr, bytes, st);
    });
    for (const at::Tensor* t : {given, dweight, dbias}) written(t);
    if (!need) Py_RETURN_NONE;
    if (!given) return THPVariable_Wrap(dx);
    Py_INCREF(a[5]);
    return a[5];
}

// ---- module ----------------------------------------------------------------------------------------------------------
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

// bind(error class, stream function, address of each entry point in the order below)
PyObject* bind(PyObject*, PyObject* args) {
    PyObject *error, *stream;
    unsigned long long p[7];
    if (!PyArg_ParseTuple(args, "OOKKKKKKK", &error, &stream, p, p + 1, p + 2, p + 3, p + 4, p + 5, p + 6)) return nullptr;
    p_grads_workspace = reinterpret_cast<decltype(p_grads_workspace)>(p[0]);
    p_grad_norm = reinterpret_cast<decltype(p_grad_norm)>(p[1]);
    p_clip_grads = reinterpret_cast<decltype(p_clip_grads)>(p[2]);
    p_gather_grads = reinterpret_cast<decltype(p_gather_grads)>(p[3]);
    p_layer_norm = reinterpret_cast<decltype(p_layer_norm)>(p[4]);
    p_layer_norm_workspace = reinterpret_cast<decltype(p_layer_norm_workspace)>(p[5]);
    p_layer_norm_backward = reinterpret_cast<decltype(p_layer_norm_backward)>(p[6]);
    Py_INCREF(error);
    Py_INCREF(stream);
    Py_XDECREF(g_error);
    Py_XDECREF(g_stream);
    g_error = error;
    g_stream = stream;
    Py_RETURN_NONE;
}

template <typename F>
PyCFunction as_method(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)); }

PyMethodDef g_methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"grad_norm", as_method(entry<grad_norm, 3>), METH_FASTCALL, nullptr},
    {"clip_grads", as_method(entry<clip_grads, 4>), METH_FASTCALL, nullptr},
    {"gather_grads", as_method(entry<gather_grads, 5>), METH_FASTCALL, nullptr},
    {"layer_norm", as_method(entry<layer_norm, 5>), METH_FASTCALL, nullptr},
    {"layer_norm_backward", as_method(entry<layer_norm_backward, 9>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_train", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__train() { return PyModule_Create(&g_module); }
