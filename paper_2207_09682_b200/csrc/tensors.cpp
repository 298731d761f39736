// Argument marshalling of the operators on top of the trees: torch tensors in, calls of include/qgbdt.h out.
//
// The calls take a few microseconds on the GPU for small inputs, and clipping takes hundreds of tensors; fetching a
// tensor's address, sizes and type from Python costs a tenth of a microsecond each.  This extension module does that
// and the checks in C++ and holds no arithmetic; binding.py gives it the library's functions (bind) and wraps it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <limits>
#include <vector>

#include "qgbdt.h"

namespace {

// The library's functions and the exception class of binding.py.
struct Bound {
    decltype(&qgbdt_embed) embed;
    decltype(&qgbdt_embed_backward) embed_backward;
    decltype(&qgbdt_softmax_ce) softmax_ce;
    decltype(&qgbdt_softmax_ce_backward) softmax_ce_backward;
    decltype(&qgbdt_clip_grad_norm) clip_grad_norm;
    decltype(&qgbdt_last_error) last_error;
    PyObject *error;
} lib = {};

PyObject *fail(int code, const char *message) {
    PyObject *e = PyObject_CallFunction(lib.error, "is", code, message);
    if (e) {
        PyErr_SetObject(lib.error, e);
        Py_DECREF(e);
    }
    return nullptr;
}
PyObject *refuse(const char *message) { return fail(QGBDT_ERR_ARG, message); }
PyObject *refuse(const char *what, const char *message) {
    char text[256];
    snprintf(text, sizeof(text), "%s %s", what, message);
    return refuse(text);
}

int element(const at::Tensor &t) {
    switch (t.scalar_type()) {
        case at::kFloat: return QGBDT_F32;
        case at::kBFloat16: return QGBDT_BF16;
        case at::kHalf: return QGBDT_F16;
        default: return -1;
    }
}
int index_type(const at::Tensor &t) { return t.scalar_type() == at::kInt ? QGBDT_I32 : t.scalar_type() == at::kLong ? QGBDT_I64 : -1; }

// The first arguments of every call.
struct Call {
    qgbdt_ctx *ctx;
    int device;
    void *stream;
    bool take(PyObject *const *args, Py_ssize_t nargs, Py_ssize_t want) {
        if (!lib.error || nargs != want) {
            PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
            return false;
        }
        ctx = static_cast<qgbdt_ctx *>(PyLong_AsVoidPtr(args[0]));
        device = (int)PyLong_AsLong(args[1]);
        if (PyErr_Occurred()) return false;
        stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
        return true;
    }
    bool here(const at::Tensor &t) const { return t.is_cuda() && t.get_device() == device; }
    PyObject *result(int rc) const { return rc == QGBDT_OK ? nullptr : fail(rc, lib.last_error(ctx)); }
};

// Warns where autograd would be expected to record the call; false with an exception where warnings are errors.
bool unrecorded(const at::Tensor &t, const char *name) {
    if (!at::GradMode::is_enabled() || !t.requires_grad()) return true;
    char text[256];
    snprintf(text, sizeof(text), "%s requires a gradient, but autograd does not record this call and its result has no graph; the "
             "operators' *_backward calls give gradients (torch.no_grad() or detach() silences this)", name);
    return PyErr_WarnEx(PyExc_UserWarning, text, 1) == 0;
}

// The caller's tensor has been written: its version goes up, as with torch's own in-place operations, so that autograd
// notices where it was saved for a backward pass.
void written(const at::Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();   // (those keep no version)
}

// A tensor argument; NULL and an exception if it is none.
const at::Tensor *tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) {
        refuse(name, "must be a tensor");
        return nullptr;
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided || t.is_neg()) {   // the memory has to hold the values themselves
        refuse(name, "must be a dense tensor without a pending negation");
        return nullptr;
    }
    return &t;
}

// A matrix on the context's device whose rows are contiguous (any row stride).
struct Rows {
    const at::Tensor *t = nullptr;
    int64_t n = 0, d = 0, ld = 0;
    int type = -1;
    void *p() const { return t->data_ptr(); }
    bool take(const Call &c, PyObject *o, const char *name) {
        t = tensor(o, name);
        return t && check(c, name);
    }
    bool take_input(const Call &c, PyObject *o, const char *name) { return take(c, o, name) && unrecorded(*t, name); }
    bool check(const Call &c, const char *name) {
        if (!c.here(*t)) return refuse(name, "must be a CUDA tensor on the context's device"), false;
        if (t->dim() != 2) return refuse(name, "must be a matrix"), false;
        n = t->size(0), d = t->size(1);
        if (d > std::numeric_limits<int32_t>::max()) return refuse(name, "has too many columns"), false;   // the calls take 32 bits
        if (d > 1 && t->stride(1) != 1) return refuse(name, "must have contiguous rows"), false;
        ld = n > 1 ? t->stride(0) : d > 0 ? d : 1;
        type = element(*t);
        return true;
    }
};

// Tokens [N] or [N, bag].
struct Tokens {
    const at::Tensor *t;
    int64_t n, bag, ld;
    int type;
    bool take(const Call &c, PyObject *o) {
        t = tensor(o, "tokens");
        if (!t) return false;
        type = index_type(*t);
        if (type < 0) return refuse("tokens must be int32 or int64"), false;
        if (t->dim() == 1) {
            if (!c.here(*t)) return refuse("tokens must be a CUDA tensor on the context's device"), false;
            n = t->size(0), bag = 1, ld = n > 1 ? t->stride(0) : 1;
            return true;
        }
        Rows r;
        r.t = t;
        if (!r.check(c, "tokens")) return false;
        n = r.n, bag = r.d, ld = r.ld;
        return true;
    }
};

// Address of a contiguous vector of `count` elements, or NULL for None.
bool words(const Call &c, PyObject *o, const char *name, at::ScalarType type, int64_t count, void **out) {
    *out = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = tensor(o, name);
    if (!t) return false;
    if (!c.here(*t) || t->scalar_type() != type || t->numel() != count || !t->is_contiguous()) {
        char text[160];
        snprintf(text, sizeof(text), "must be a contiguous CUDA tensor of %lld elements of type %s", (long long)count, c10::toString(type));
        refuse(name, text);
        return false;
    }
    *out = t->data_ptr();
    return true;
}

// An output [n, d] of `like`'s type: the caller's, or a new one if None.
struct Output {
    at::Tensor made;
    Rows r;
    bool take(const Call &c, PyObject *o, const char *name, int64_t n, int64_t d, const at::Tensor &like) {
        if (o == Py_None) {
            if (n < 0) return refuse(name, "cannot have a negative size"), false;
            made = at::empty({n, d}, like.options().requires_grad(false));
            r.t = &made, r.n = n, r.d = d, r.ld = d > 0 ? d : 1;
            return true;
        }
        if (!r.take(c, o, name)) return false;
        if (r.n != n || r.d != d || r.t->scalar_type() != like.scalar_type()) return refuse(name, "has the wrong size or type"), false;
        return true;
    }
    PyObject *give(PyObject *o) const {   // a new reference
        if (o != Py_None) {
            written(*r.t);
            Py_INCREF(o);
            return o;
        }
        return THPVariable_Wrap(made);
    }
};

bool number(PyObject *o, double *out) {
    *out = PyFloat_AsDouble(o);
    return !PyErr_Occurred();
}

// embed(ctx, device, table, tokens, scale, out, status) -> out
PyObject *py_embed(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    Rows table;
    Tokens tok;
    Output out;
    double scale;
    void *status;
    if (!c.take(args, nargs, 7) || !table.take_input(c, args[2], "table") || !tok.take(c, args[3]) || !number(args[4], &scale)) return nullptr;
    if (table.type < 0) return refuse("table must be float32, bfloat16 or float16");
    if (!out.take(c, args[5], "out", tok.n, table.d, *table.t) || !words(c, args[6], "status", at::kInt, 1, &status)) return nullptr;
    const int rc = lib.embed(c.ctx, table.p(), table.type, table.n, (int32_t)table.d, table.ld, tok.t->data_ptr(), tok.type, tok.n, (int32_t)tok.bag, tok.ld,
                             (float)scale, out.r.p(), out.r.ld, (int32_t *)status, c.stream);
    return rc == QGBDT_OK ? out.give(args[5]) : c.result(rc);
    END_HANDLE_TH_ERRORS
}

// embed_backward(ctx, device, grad_out, tokens, n_entries, scale, grad_table, status) -> grad_table
PyObject *py_embed_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    Rows grad;
    Tokens tok;
    Output out;
    double scale;
    void *status;
    if (!c.take(args, nargs, 8) || !grad.take_input(c, args[2], "grad_out") || !tok.take(c, args[3]) || !number(args[5], &scale)) return nullptr;
    const int64_t entries = PyLong_AsLongLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    if (grad.type < 0) return refuse("grad_out must be float32, bfloat16 or float16");
    if (grad.n != tok.n) return refuse("grad_out and tokens differ in rows");
    if (!out.take(c, args[6], "grad_table", entries, grad.d, *grad.t) || !words(c, args[7], "status", at::kInt, 1, &status)) return nullptr;
    const int rc = lib.embed_backward(c.ctx, grad.p(), grad.type, grad.ld, tok.t->data_ptr(), tok.type, tok.n, (int32_t)tok.bag, tok.ld, (float)scale,
                                      out.r.p(), entries, (int32_t)grad.d, out.r.ld, (int32_t *)status, c.stream);
    return rc == QGBDT_OK ? out.give(args[6]) : c.result(rc);
    END_HANDLE_TH_ERRORS
}

// What both directions of the loss take: hidden, weight, labels, bias from args[2] on.
struct Classifier {
    Rows hidden, weight;
    const at::Tensor *labels;
    int label_type;
    void *bias, *label;
    bool take(const Call &c, PyObject *const *args) {
        if (!hidden.take_input(c, args[2], "hidden") || !weight.take_input(c, args[3], "weight") || !(labels = tensor(args[4], "labels"))) return false;
        if (hidden.type != weight.type || (hidden.type != QGBDT_BF16 && hidden.type != QGBDT_F16))
            return refuse("hidden and weight must both be bfloat16 or float16"), false;
        if (hidden.d != weight.d) return refuse("hidden and weight differ in columns"), false;
        label_type = index_type(*labels);
        if (label_type < 0 || labels->dim() != 1) return refuse("labels must be [N], int32 or int64"), false;
        return words(c, args[4], "labels", labels->scalar_type(), hidden.n, &label) && words(c, args[5], "bias", at::kFloat, weight.n, &bias) &&
               (args[5] == Py_None || unrecorded(THPVariable_Unpack(args[5]), "bias"));
    }
};

// softmax_ce(ctx, device, hidden, weight, labels, bias, status) -> (loss, losses, lse)
PyObject *py_softmax_ce(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    Classifier k;
    void *status;
    if (!c.take(args, nargs, 7) || !k.take(c, args) || !words(c, args[6], "status", at::kInt, 1, &status)) return nullptr;
    const int64_t n = k.hidden.n;
    const at::Tensor all = at::empty({2 * n + 1}, k.hidden.t->options().dtype(at::kFloat).requires_grad(false));
    float *p = all.data_ptr<float>();   // losses, lse, loss
    const int rc = lib.softmax_ce(c.ctx, k.hidden.p(), k.hidden.ld, k.weight.p(), k.weight.ld, k.hidden.type, (const float *)k.bias, k.label, k.label_type, n,
                                  k.weight.n, (int32_t)k.hidden.d, p + 2 * n, p, p + n, (int32_t *)status, c.stream);
    if (rc != QGBDT_OK) return c.result(rc);
    PyObject *const loss = THPVariable_Wrap(all.slice(0, 2 * n, 2 * n + 1)), *const losses = THPVariable_Wrap(all.slice(0, 0, n)),
                    *const lse = THPVariable_Wrap(all.slice(0, n, 2 * n));
    return Py_BuildValue("(NNN)", loss, losses, lse);
    END_HANDLE_TH_ERRORS
}

// softmax_ce_backward(ctx, device, hidden, weight, labels, bias, lse, grad_loss, grad_hidden, grad_weight, status)
//   -> (grad_hidden, grad_weight, grad_bias or None)
PyObject *py_softmax_ce_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    Classifier k;
    Output gh, gw;
    void *lse, *grad_loss, *status;
    if (!c.take(args, nargs, 11) || !k.take(c, args) || !words(c, args[6], "lse", at::kFloat, k.hidden.n, &lse) ||
        !words(c, args[7], "grad_loss", at::kFloat, 1, &grad_loss) || !gh.take(c, args[8], "grad_hidden", k.hidden.n, k.hidden.d, *k.hidden.t) ||
        !gw.take(c, args[9], "grad_weight", k.weight.n, k.weight.d, *k.weight.t) || !words(c, args[10], "status", at::kInt, 1, &status))
        return nullptr;
    at::Tensor gb;
    if (k.bias) gb = at::empty({k.weight.n}, k.hidden.t->options().dtype(at::kFloat).requires_grad(false));
    const int rc = lib.softmax_ce_backward(c.ctx, k.hidden.p(), k.hidden.ld, k.weight.p(), k.weight.ld, k.hidden.type, (const float *)k.bias, k.label,
                                           k.label_type, k.hidden.n, k.weight.n, (int32_t)k.hidden.d, (const float *)lse, (const float *)grad_loss, gh.r.p(),
                                           gh.r.ld, gw.r.p(), gw.r.ld, k.bias ? gb.data_ptr<float>() : nullptr, (int32_t *)status, c.stream);
    if (rc != QGBDT_OK) return c.result(rc);
    PyObject *bias;
    if (k.bias) bias = THPVariable_Wrap(gb);
    else Py_INCREF(Py_None), bias = Py_None;
    return Py_BuildValue("(NNN)", gh.give(args[8]), gw.give(args[9]), bias);
    END_HANDLE_TH_ERRORS
}

// clip_grad_norm(ctx, device, grads, max_norm, out) -> norm
PyObject *py_clip_grad_norm(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    double max_norm;
    if (!c.take(args, nargs, 5) || !number(args[3], &max_norm)) return nullptr;
    std::vector<void *> in, out;
    std::vector<int64_t> sizes;
    std::vector<int32_t> types;
    const bool to_out = args[4] != Py_None, in_place = !to_out && max_norm <= std::numeric_limits<double>::max();
    THPObjectPtr held[2];   // the tensors stay alive until the call has been made
    auto take = [&](PyObject *list, const char *name, bool first) {
        PyObject *const seq = PySequence_Fast(list, "expected a list of tensors");
        if (!seq) return false;
        held[!first] = THPObjectPtr(seq);
        const at::Tensor *recorded = nullptr;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
        bool ok = first || n == (Py_ssize_t)in.size() || (refuse("out must match the gradients in number"), false);
        for (Py_ssize_t i = 0; ok && i < n; ++i) {
            const at::Tensor *t = tensor(PySequence_Fast_GET_ITEM(seq, i), name);
            ok = t != nullptr;
            if (!ok) break;
            if (first && t->requires_grad()) recorded = t;
            const int type = element(*t);
            if (!c.here(*t) || !t->is_contiguous() || type < 0) {
                refuse(name, "must be contiguous float32, bfloat16 or float16 tensors on the context's device");
                ok = false;
            } else if (first) {
                in.push_back(t->data_ptr()), sizes.push_back(t->numel()), types.push_back(type);
            } else if (t->numel() != sizes[i] || type != types[i]) {
                refuse("out must match the gradients in sizes and types");
                ok = false;
            } else {
                out.push_back(t->data_ptr());
            }
        }
        return ok && (!recorded || unrecorded(*recorded, name));
    };
    if (!take(args[2], "gradients", true) || (to_out && !take(args[4], "out", false))) return nullptr;
    const at::Tensor norm = at::empty({1}, at::TensorOptions().dtype(at::kFloat).device(at::kCUDA, (c10::DeviceIndex)c.device));
    const int rc = lib.clip_grad_norm(c.ctx, in.data(), to_out ? out.data() : nullptr, sizes.data(), types.data(), (int32_t)in.size(), max_norm,
                                      norm.data_ptr<float>(), c.stream);
    if (rc != QGBDT_OK) return c.result(rc);
    if (in_place || to_out) {
        PyObject *const seq = held[to_out].get();
        for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(seq); ++i) {
            PyObject *const o = PySequence_Fast_GET_ITEM(seq, i);
            if (THPVariable_Check(o)) written(THPVariable_Unpack(o));   // (a warning's handler may have changed the list)
        }
    }
    return THPVariable_Wrap(norm);
    END_HANDLE_TH_ERRORS
}

// bind(error class, addresses of embed, embed_backward, softmax_ce, softmax_ce_backward, clip_grad_norm, last_error)
PyObject *py_bind(PyObject *, PyObject *args) {
    PyObject *error;
    unsigned long long p[6];
    if (!PyArg_ParseTuple(args, "OKKKKKK", &error, &p[0], &p[1], &p[2], &p[3], &p[4], &p[5])) return nullptr;
    Py_INCREF(error);
    Py_XDECREF(lib.error);
    lib = Bound{reinterpret_cast<decltype(lib.embed)>(p[0]),          reinterpret_cast<decltype(lib.embed_backward)>(p[1]),
                reinterpret_cast<decltype(lib.softmax_ce)>(p[2]),     reinterpret_cast<decltype(lib.softmax_ce_backward)>(p[3]),
                reinterpret_cast<decltype(lib.clip_grad_norm)>(p[4]), reinterpret_cast<decltype(lib.last_error)>(p[5]), error};
    Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(embed), FAST(embed_backward), FAST(softmax_ce), FAST(softmax_ce_backward), FAST(clip_grad_norm),
                         {"bind", py_bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", "Argument marshalling of the operators on top of the trees.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
