// Python side of include/liec_activations.h: argument checks, outputs, scratch and the call, in one step per operator.
#include <torch/csrc/Dtype.h>

#include <limits>

#include "binding_common.hpp"
#include "liec_activations.h"

using namespace liec_binding;

namespace {

decltype(&liec_checkpoint_save) p_checkpoint_save;
decltype(&liec_checkpoint_load) p_checkpoint_load;
decltype(&liec_group_norm_workspace) p_group_norm_workspace;
decltype(&liec_group_norm) p_group_norm;
decltype(&liec_group_norm_backward) p_group_norm_backward;
decltype(&liec_weight_grad_workspace) p_weight_grad_workspace;
decltype(&liec_weight_grad) p_weight_grad;

PyObject* pack(std::initializer_list<at::Tensor> made) {
    PyObject* const r = PyTuple_New((Py_ssize_t)made.size());
    if (!r) throw Raise{nullptr, ""};
    Py_ssize_t i = 0;
    for (const at::Tensor& t : made) {
        PyObject* const o = THPVariable_Wrap(t);
        if (!o) {
            Py_DECREF(r);
            throw Raise{nullptr, ""};
        }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}
PyObject* given_or(PyObject* given, const at::Tensor& made) {
    if (given == Py_None) return THPVariable_Wrap(made);
    Py_INCREF(given);
    return given;
}

at::Tensor scratch(int64_t bytes, const at::Tensor& x, const char* what) {
    if (bytes < 0) value_error(std::string(what) + " of shape " + text(x.sizes()) + " are more than the library takes");
    return bytes ? new_tensor({bytes}, at::kByte, x) : at::Tensor();
}

// ---- checkpoints -----------------------------------------------------------------------------------------------------
std::vector<int64_t> exponent_sizes(at::IntArrayRef x) {
    std::vector<int64_t> r(x.begin(), x.end());
    r.back() = (r.back() + LIEC_CHECKPOINT_COLUMNS - 1) / LIEC_CHECKPOINT_COLUMNS;
    return r;
}
struct Checkpoint {
    at::Tensor values, exponents;
    liec_checkpoint raw() const { return {static_cast<int8_t*>(values.data_ptr()), static_cast<uint8_t*>(exponents.data_ptr())}; }
};
Checkpoint new_checkpoint(const at::Tensor& x) {
    return {new_tensor(x.sizes(), at::kChar, x), new_tensor(exponent_sizes(x.sizes()), at::kByte, x)};
}
bool is_pair(PyObject* o) { return PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 2; }
Checkpoint read_checkpoint(PyObject* o) {
    if (!is_pair(o)) type_error("a checkpoint must be what liec_checkpoint_save returned");
    const Checkpoint s{tensor(PyTuple_GET_ITEM(o, 0), "a checkpoint's values"), tensor(PyTuple_GET_ITEM(o, 1), "a checkpoint's exponents")};
    if (s.values.scalar_type() != at::kChar || s.exponents.scalar_type() != at::kByte || !s.values.is_cuda() || s.values.device() != s.exponents.device())
        type_error("a checkpoint's values must be int8 and its exponents uint8, on one GPU");
    if (!s.values.dim() || s.values.size(-1) < 1 || s.exponents.sizes() != at::IntArrayRef(exponent_sizes(s.values.sizes())))
        value_error("a checkpoint's values of shape " + text(s.values.sizes()) + " do not fit exponents of shape " + text(s.exponents.sizes()));
    if (!s.values.is_contiguous() || !s.exponents.is_contiguous()) value_error("a checkpoint's values and exponents must be contiguous");
    return s;
}
void check_checkpoint(const Checkpoint& s, const at::Tensor& x) {
    if (s.values.device() != x.device()) type_error("a checkpoint must be on the activations' GPU");
    if (s.values.sizes() != x.sizes()) value_error("a checkpoint has shape " + text(s.values.sizes()) + ", expected " + text(x.sizes()));
}

PyObject* checkpoint_save(PyObject* const* a) {      // x, out
    const at::Tensor& x = tensor(a[0], "x");
    const int code = activations_code(x);
    const Sizes s = sizes_of(x, {}, {&x});
    const liec_rows xr = rows_of(x, s, "x");
    const int32_t N = workers_of(s);
    const Checkpoint out = a[1] == Py_None ? new_checkpoint(x) : read_checkpoint(a[1]);
    check_checkpoint(out, x);
    const liec_checkpoint raw = out.raw();
    void* const st = stream_of(x);
    call("liec_checkpoint_save", x, [&] { return p_checkpoint_save(&xr, &raw, N, s.R, s.C, (liec_dtype)code, st); });
    if (a[1] == Py_None) return pack({out.values, out.exponents});
    written(&out.values);
    written(&out.exponents);
    Py_INCREF(a[1]);
    return a[1];
}

PyObject* checkpoint_load(PyObject* const* a) {      // checkpoint, dtype, out
    const Checkpoint saved = read_checkpoint(a[0]);
    const at::Tensor* const out = optional_tensor(a[2], "out");
    if (!out && !THPDtype_Check(a[1])) type_error("dtype must be torch.float32, torch.bfloat16 or torch.float16");
    const at::Tensor y = out ? *out : new_tensor(saved.values.sizes(), reinterpret_cast<THPDtype*>(a[1])->scalar_type, saved.values);
    const int code = activations_code(y);
    check_checkpoint(saved, y);
    const Sizes s = sizes_of(y, {}, {&y});
    const liec_rows yr = rows_of(y, s, "out");
    const int32_t N = workers_of(s);
    const liec_checkpoint raw = saved.raw();
    void* const st = stream_of(y);
    call("liec_checkpoint_load", y, [&] { return p_checkpoint_load(&raw, &yr, N, s.R, s.C, (liec_dtype)code, st); });
    written(out);
    return given_or(a[2], y);
}

// ---- group normalisation ---------------------------------------------------------------------------------------------
struct ImageSizes {
    int32_t N;
    int64_t B, S, C, G;
};
ImageSizes images_of(const at::Tensor& x, int64_t G, std::initializer_list<const at::Tensor*> params) {
    if (x.dim() < 3) value_error("images must be [workers, images, ..., channels], got shape " + text(x.sizes()));
    const int64_t N = x.size(0), C = x.size(-1);
    if (N < 1 || N > 65535) value_error(std::to_string(N) + " workers are none, or more than the library takes");
    if (C < 1 || G < 1 || C % G) value_error(std::to_string(C) + " channels do not fall into " + std::to_string(G) + " groups");
    for (const at::Tensor* p : params)
        if (p && (p->dim() < 1 || p->dim() > 2 || p->size(-1) != C || (C > 1 && p->stride(-1) != 1) || (p->dim() == 2 && p->size(0) != N)))
            value_error("a weight or bias of shape " + text(p->sizes()) + " does not fit " + std::to_string(N) + " workers' " + std::to_string(C) +
                        " channels, or its channels are not contiguous");
    int64_t S = 1;
    for (int64_t d = 2; d < x.dim() - 1; ++d) S *= x.size(d);
    return {(int32_t)N, x.size(1), S, C, G};
}
liec_images images(const at::Tensor& t, const ImageSizes& s, const char* what) {
    liec_images r{t.data_ptr(), s.B * s.S * s.C, s.S * s.C, s.C};
    if (t.is_contiguous()) return r;
    if (s.C > 1 && t.stride(-1) != 1) value_error(std::string("the channels of ") + what + " must be contiguous");
    r.worker_stride = t.stride(0);
    r.image_stride = t.stride(1);
    if (!merged(t, 2, t.dim() - 1, &r.row_stride)) value_error(std::string("the positions of ") + what + " of strides " + text(t.strides()) + " are not at equal distances");
    return r;
}
int64_t whole_number(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raise{nullptr, ""};
    return v;
}

PyObject* group_norm(PyObject* const* a) {           // x, groups, weight, bias, eps, activation, out, save
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor *weight = optional_tensor(a[2], "weight"), *bias = optional_tensor(a[3], "bias"), *out = optional_tensor(a[6], "out");
    const double eps = number(a[4]);
    const int64_t G = whole_number(a[1]), act = whole_number(a[5]);
    const int code = activations_code(x), pcode = params_code(x, {weight, bias});
    if (out) check_like(*out, x, "out");
    const ImageSizes s = images_of(x, G, {weight, bias});
    const int64_t bytes = p_group_norm_workspace(s.N, s.B, s.S, s.C, s.G);
    const at::Tensor ws = scratch(bytes, x, "images"), y = out ? *out : new_tensor(x.sizes(), x.scalar_type(), x);
    const at::Tensor mean = new_tensor({s.N, s.B, s.G}, at::kFloat, x), rstd = new_tensor({s.N, s.B, s.G}, at::kFloat, x);
    if (!s.S)                          // means of nothing: the library leaves them alone
        for (const at::Tensor* t : {&mean, &rstd}) t->fill_(std::numeric_limits<float>::quiet_NaN());
    const bool save = a[7] == Py_True;
    const Checkpoint saved = save ? new_checkpoint(x) : Checkpoint{};
    const liec_checkpoint raw = save ? saved.raw() : liec_checkpoint{nullptr, nullptr};
    const liec_images xi = images(x, s, "x"), yi = images(y, s, "out");
    const liec_param w = param_of(weight), b = param_of(bias);
    void* const st = stream_of(x);
    call("liec_group_norm", x, [&] {
        return p_group_norm(&xi, &w, &b, &yi, data_of(&mean), data_of(&rstd), save ? &raw : nullptr, s.N, s.B, s.S, s.C, s.G, (float)eps, (liec_activation)act,
                            (liec_dtype)code, (liec_dtype)pcode, bytes ? ws.data_ptr() : nullptr, bytes, st);
    });
    written(out);
    return save ? pack({y, mean, rstd, saved.values, saved.exponents}) : pack({y, mean, rstd});
}

PyObject* group_norm_backward(PyObject* const* a) {  // dy, x or checkpoint, mean, rstd, weight, bias, activation, dx, dweight, dbias, need_dx
    const at::Tensor &dy = tensor(a[0], "dy"), &mean = tensor(a[2], "mean"), &rstd = tensor(a[3], "rstd");
    const at::Tensor *weight = optional_tensor(a[4], "weight"), *bias = optional_tensor(a[5], "bias");
    const at::Tensor *dweight = optional_tensor(a[8], "dweight"), *dbias = optional_tensor(a[9], "dbias");
    const int64_t act = whole_number(a[6]);
    const bool need = a[10] == Py_True;
    const at::Tensor* const given = need ? optional_tensor(a[7], "dx") : nullptr;
    const int code = activations_code(dy), pcode = params_code(dy, {weight, bias, dweight, dbias});
    const bool kept = is_pair(a[1]);
    const Checkpoint saved = kept ? read_checkpoint(a[1]) : Checkpoint{};
    const at::Tensor* const x = kept ? nullptr : &tensor(a[1], "x");
    if (kept) check_checkpoint(saved, dy);
    else check_like(*x, dy, "x");
    if (given) check_like(*given, dy, "dx");
    if (dy.dim() < 3) value_error("images must be [workers, images, ..., channels], got shape " + text(dy.sizes()));
    for (const at::Tensor* t : {&mean, &rstd})
        if (t->scalar_type() != at::kFloat || t->device() != dy.device() || t->dim() != 3 || t->size(0) != dy.size(0) || t->size(1) != dy.size(1) || !t->is_contiguous())
            type_error("mean and rstd must be what liec_group_norm returned");
    if (mean.size(2) != rstd.size(2)) type_error("mean and rstd must be what liec_group_norm returned");
    const ImageSizes s = images_of(dy, mean.size(2), {weight, bias, dweight, dbias});
    check_rows_apart(dweight, "dweight");
    check_rows_apart(dbias, "dbias");
    const int64_t bytes = p_group_norm_workspace(s.N, s.B, s.S, s.C, s.G);
    const at::Tensor ws = scratch(bytes, dy, "images"), dx = given ? *given : need ? new_tensor(dy.sizes(), dy.scalar_type(), dy) : at::Tensor();
    const liec_checkpoint raw = kept ? saved.raw() : liec_checkpoint{nullptr, nullptr};
    const liec_images gi = images(dy, s, "dy"), xi = x ? images(*x, s, "x") : liec_images{}, di = dx.defined() ? images(dx, s, "dx") : liec_images{};
    const liec_param w = param_of(weight), b = param_of(bias), dw = param_of(dweight), db = param_of(dbias);
    void* const st = stream_of(dy);
    call("liec_group_norm_backward", dy, [&] {
        return p_group_norm_backward(&gi, &xi, &raw, data_of(&mean), data_of(&rstd), &w, &b, &di, &dw, &db, s.N, s.B, s.S, s.C, s.G, (liec_activation)act,
                                     (liec_dtype)code, (liec_dtype)pcode, bytes ? ws.data_ptr() : nullptr, bytes, st);
    });
    for (const at::Tensor* t : {given, dweight, dbias}) written(t);
    if (!need) Py_RETURN_NONE;
    return given_or(given ? a[7] : Py_None, dx);
}

// ---- weight gradients ------------------------------------------------------------------------------------------------
PyObject* weight_grad(PyObject* const* a) {          // dy, checkpoint, dweight, dbias
    const at::Tensor& dy = tensor(a[0], "dy");
    const Checkpoint saved = read_checkpoint(a[1]);
    const at::Tensor *given = optional_tensor(a[2], "dweight"), *dbias = optional_tensor(a[3], "dbias");
    const int code = activations_code(dy), pcode = params_code(dy, {given, dbias});
    if (dy.dim() < 2 || dy.size(-1) < 1) value_error("dy must be [workers, ..., outputs], got shape " + text(dy.sizes()));
    if (saved.values.device() != dy.device()) type_error("a checkpoint must be on the activations' GPU");
    if (saved.values.sizes().slice(0, saved.values.dim() - 1) != dy.sizes().slice(0, dy.dim() - 1))
        value_error("a checkpoint of shape " + text(saved.values.sizes()) + " does not fit dy of shape " + text(dy.sizes()));
    const int64_t O = dy.size(-1), C = saved.values.size(-1), rows = dy.numel() / O;
    const bool each = !given || given->dim() == 3;             // a sum for each worker, or one over all of them
    const int64_t N = each ? dy.size(0) : 1;
    if (N < 1 || N > 65535) value_error(std::to_string(N) + " workers are none, or more than the library takes");
    if (!given && pcode != (int)LIEC_F32) type_error("dbias must be float32 where dweight is not given");
    const at::Tensor dw = given ? *given : new_tensor({N, O, C}, at::kFloat, dy);
    if ((dw.dim() != 3 && dw.dim() != 2) || dw.size(-1) != C || dw.size(-2) != O || (each && dw.size(0) != N) || (C > 1 && dw.stride(-1) != 1))
        value_error("dweight of shape " + text(dw.sizes()) + " does not fit " + std::to_string(N) + " workers' " + std::to_string(O) + " x " + std::to_string(C) +
                    " weights, or its columns are not contiguous");
    if (dbias && (dbias->dim() != (each ? 2 : 1) || dbias->size(-1) != O || (each && dbias->size(0) != N) || (O > 1 && dbias->stride(-1) != 1)))
        value_error("dbias of shape " + text(dbias->sizes()) + " does not go with dweight of shape " + text(dw.sizes()) + ", or its columns are not contiguous");
    check_rows_apart(dbias, "dbias");
    const Sizes s{N, rows / N, O, each ? 1 : 0};
    const liec_rows gr = rows_of(dy, s, "dy");
    const liec_matrices out{dw.data_ptr(), each ? dw.stride(0) : 0, dw.stride(-2)};
    const liec_param db = param_of(dbias);
    const liec_checkpoint raw = saved.raw();
    const int64_t bytes = p_weight_grad_workspace((int32_t)N, s.R, O, C);
    const at::Tensor ws = scratch(bytes, dy, "gradients");
    void* const st = stream_of(dy);
    call("liec_weight_grad", dy, [&] {
        return p_weight_grad(&gr, &raw, &out, &db, (int32_t)N, s.R, O, C, (liec_dtype)code, (liec_dtype)pcode, bytes ? ws.data_ptr() : nullptr, bytes, st);
    });
    written(given);
    written(dbias);
    return given_or(a[2], dw);
}

// ---- module ----------------------------------------------------------------------------------------------------------
// bind_activations(address of each entry point in the order below); after bind
PyObject* bind(PyObject*, PyObject* args) {
    unsigned long long p[7];
    if (!PyArg_ParseTuple(args, "KKKKKKK", p, p + 1, p + 2, p + 3, p + 4, p + 5, p + 6)) return nullptr;
    p_checkpoint_save = reinterpret_cast<decltype(p_checkpoint_save)>(p[0]);
    p_checkpoint_load = reinterpret_cast<decltype(p_checkpoint_load)>(p[1]);
    p_group_norm_workspace = reinterpret_cast<decltype(p_group_norm_workspace)>(p[2]);
    p_group_norm = reinterpret_cast<decltype(p_group_norm)>(p[3]);
    p_group_norm_backward = reinterpret_cast<decltype(p_group_norm_backward)>(p[4]);
    p_weight_grad_workspace = reinterpret_cast<decltype(p_weight_grad_workspace)>(p[5]);
    p_weight_grad = reinterpret_cast<decltype(p_weight_grad)>(p[6]);
    Py_RETURN_NONE;
}

}  // namespace

namespace liec_binding {

extern PyMethodDef activation_methods[];
PyMethodDef activation_methods[] = {
    {"bind_activations", bind, METH_VARARGS, nullptr},
    {"checkpoint_save", as_method(entry<checkpoint_save, 2>), METH_FASTCALL, nullptr},
    {"checkpoint_load", as_method(entry<checkpoint_load, 3>), METH_FASTCALL, nullptr},
    {"group_norm", as_method(entry<group_norm, 8>), METH_FASTCALL, nullptr},
    {"group_norm_backward", as_method(entry<group_norm_backward, 11>), METH_FASTCALL, nullptr},
    {"weight_grad", as_method(entry<weight_grad, 4>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

}  // namespace liec_binding
