// Argument marshalling of the operators on top of the trees: torch tensors in, calls of include/qgbdt.h out.
//
// The calls take a few microseconds on the GPU for small inputs, and clipping takes hundreds of tensors; fetching a
// tensor's address, sizes and type from Python costs a tenth of a microsecond each.  This extension module does that
// and the checks in C++ and holds no arithmetic; binding.py gives it the library's functions (bind) and wraps it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/cuda/EmptyTensor.h>
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
    decltype(&qgbdt_layer_norm) layer_norm;
    decltype(&qgbdt_layer_norm_backward) layer_norm_backward;
    decltype(&qgbdt_adamw) adamw;
    decltype(&qgbdt_adamw_values) adamw_values;
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

// Whether autograd would have to know what is done with the tensor: it requires a gradient, or has a tangent (of forward mode).
bool followed(const at::Tensor &t) { return t.unsafeGetTensorImpl()->autograd_meta() && (t.requires_grad() || t._fw_grad(0).defined()); }   // (mostly not even asked)

// Warns where autograd would be expected to record the call or to carry a tangent on; false with an exception where warnings are errors.
bool unrecorded(const at::Tensor &t, const char *name) {
    if (!followed(t)) return true;
    const bool tangent = t._fw_grad(0).defined();     // (t may be gone after a warning)
    char text[256];
    if (at::GradMode::is_enabled() && t.requires_grad()) {
        snprintf(text, sizeof(text), "%s requires a gradient, but autograd does not record this call and its result has no graph; the "
                 "operators' *_backward calls give gradients (torch.no_grad() or detach() silences this)", name);
        if (PyErr_WarnEx(PyExc_UserWarning, text, 1)) return false;
    }
    if (!tangent) return true;
    snprintf(text, sizeof(text), "%s has a tangent, but this call does not carry it on and its result has none (torch.autograd.forward_ad.unpack_dual() "
             "gives the tensor without one)", name);
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

// New tensors without the dispatcher, which takes as long as a small call's kernel: contiguous, and parts [at, at + n) of a vector.
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const Call &c) {
    return at::detail::empty_cuda(sizes, type, at::Device(at::kCUDA, (c10::DeviceIndex)c.device), std::nullopt);
}
at::Tensor part(const at::Tensor &all, int64_t at, int64_t n) {
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(all.storage()), all.key_set(), all.dtype());
    t.unsafeGetTensorImpl()->set_storage_offset(all.storage_offset() + at);
    t.unsafeGetTensorImpl()->set_sizes_contiguous({n});
    return t;
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
    // as large as `x`
    bool take_or_make(const Call &c, PyObject *o, const char *name, const Rows &x) {
        if (o != Py_None) return take(c, o, name, x.n, x.d, *x.t);
        made = fresh({x.n, x.d}, x.t->scalar_type(), c);
        r.t = &made, r.n = x.n, r.d = x.d, r.ld = x.d > 0 ? x.d : 1;
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
    at::Tensor recorded;
    auto take = [&](PyObject *list, const char *name, bool first) {
        PyObject *const seq = PySequence_Fast(list, "expected a list of tensors");
        if (!seq) return false;
        held[!first] = THPObjectPtr(seq);
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
        bool ok = first || n == (Py_ssize_t)in.size() || (refuse("out must match the gradients in number"), false);
        for (Py_ssize_t i = 0; ok && i < n; ++i) {
            const at::Tensor *t = tensor(PySequence_Fast_GET_ITEM(seq, i), name);
            ok = t != nullptr;
            if (!ok) break;
            if (first && followed(*t)) recorded = *t;
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
        return ok;
    };
    auto collect = [&] {
        auto once = [&](int k, PyObject *o) { return held[k].get() ? held[k].get() : o; };     // what a generator gave
        return take(once(0, args[2]), "gradients", true) && (!to_out || take(once(1, args[4]), "out", false));
    };
    if (!collect()) return nullptr;
    if (recorded.defined()) {     // a warning's handler may have changed the lists, and with them what holds the tensors
        in.clear(), out.clear(), sizes.clear(), types.clear();
        if (!unrecorded(recorded, "gradients") || !collect()) return nullptr;
    }
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

// Weight and bias of a layer norm: vectors of float32 or of the rows' type, or None.
struct Affine {
    int type = QGBDT_F32;
    at::ScalarType scalar = at::kFloat;
    void *weight = nullptr, *bias = nullptr;
    bool take(const Call &c, const Rows &x, PyObject *w, PyObject *b) {
        for (PyObject *o : {w, b}) {
            if (o == Py_None) continue;
            const at::Tensor *t = tensor(o, o == w ? "weight" : "bias");
            if (!t) return false;
            if ((o == w || w == Py_None)) scalar = t->scalar_type();
            else if (t->scalar_type() != scalar) return refuse("weight and bias must have the same type"), false;
            if (!unrecorded(*t, o == w ? "weight" : "bias")) return false;
        }
        if (scalar != at::kFloat && scalar != x.t->scalar_type()) return refuse("weight and bias must be float32 or of the rows' type"), false;
        type = scalar == at::kFloat ? QGBDT_F32 : x.type;
        return words(c, w, "weight", scalar, x.d, &weight) && words(c, b, "bias", scalar, x.d, &bias);
    }
};

// layer_norm(ctx, device, x, weight, bias, eps, out) -> (out, mean, rstd)
PyObject *py_layer_norm(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    Rows x;
    Affine w;
    Output out;
    double eps;
    if (!c.take(args, nargs, 7) || !x.take_input(c, args[2], "x")) return nullptr;
    if (x.type < 0) return refuse("x must be float32, bfloat16 or float16");
    if (!w.take(c, x, args[3], args[4]) || !number(args[5], &eps) || !out.take_or_make(c, args[6], "out", x)) return nullptr;
    const at::Tensor both = fresh({2 * x.n}, at::kFloat, c);
    float *p = both.data_ptr<float>();   // mean, rstd
    const int rc = lib.layer_norm(c.ctx, x.p(), x.ld, x.type, w.weight, w.bias, w.type, x.n, (int32_t)x.d, eps, out.r.p(), out.r.ld, p, p + x.n, c.stream);
    if (rc != QGBDT_OK) return c.result(rc);
    PyObject *const mean = THPVariable_Wrap(part(both, 0, x.n)), *const rstd = THPVariable_Wrap(part(both, x.n, x.n));
    return Py_BuildValue("(NNN)", out.give(args[6]), mean, rstd);
    END_HANDLE_TH_ERRORS
}

// layer_norm_backward(ctx, device, grad_out, x, mean, rstd, weight, grad_x, bias) -> (grad_x, grad_weight or None, grad_bias or None)
PyObject *py_layer_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    Rows grad, x;
    Affine w;
    Output gx;
    void *mean, *rstd;
    if (!c.take(args, nargs, 9) || !grad.take_input(c, args[2], "grad_out") || !x.take_input(c, args[3], "x")) return nullptr;
    if (x.type < 0) return refuse("x must be float32, bfloat16 or float16");
    if (grad.type != x.type || grad.n != x.n || grad.d != x.d) return refuse("grad_out and x differ in size or type");
    if (args[4] == Py_None || args[5] == Py_None) return refuse("mean and rstd are those of the forward call");
    if (!words(c, args[4], "mean", at::kFloat, x.n, &mean) || !words(c, args[5], "rstd", at::kFloat, x.n, &rstd) ||
        !w.take(c, x, args[6], args[8]) || !gx.take_or_make(c, args[7], "grad_x", x))
        return nullptr;
    at::Tensor gw, gb;     // a weight alone gives both
    if (args[6] != Py_None) gw = fresh({x.d}, w.scalar, c);
    if (args[6] != Py_None || args[8] != Py_None) gb = fresh({x.d}, w.scalar, c);
    const int rc = lib.layer_norm_backward(c.ctx, grad.p(), grad.ld, x.p(), x.ld, x.type, (const float *)mean, (const float *)rstd, w.weight, w.type, x.n,
                                           (int32_t)x.d, gx.r.p(), gx.r.ld, gw.defined() ? gw.data_ptr() : nullptr, gb.defined() ? gb.data_ptr() : nullptr,
                                           c.stream);
    if (rc != QGBDT_OK) return c.result(rc);
    PyObject *const x_grad = gx.give(args[7]);
    auto give = [](const at::Tensor &t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); };
    PyObject *const weight_grad = give(gw), *const bias_grad = give(gb);
    return Py_BuildValue("(NNN)", x_grad, weight_grad, bias_grad);
    END_HANDLE_TH_ERRORS
}

// A list of contiguous tensors on the context's device.
struct List {
    THPObjectPtr held;   // the tensors stay alive until the call has been made
    Py_ssize_t n = 0;
    const char *name = "";
    bool take(PyObject *o, const char *what, Py_ssize_t want) {
        name = what;
        held = THPObjectPtr(PySequence_Fast(o, "expected a list of tensors"));
        if (!held.get()) return false;
        n = PySequence_Fast_GET_SIZE(held.get());
        return want < 0 || n == want || (refuse(name, "must match the parameters in number"), false);
    }
    bool none(Py_ssize_t i) const { return i < PySequence_Fast_GET_SIZE(held.get()) && PySequence_Fast_GET_ITEM(held.get(), i) == Py_None; }
    const at::Tensor *get(const Call &c, Py_ssize_t i) const {
        if (i >= PySequence_Fast_GET_SIZE(held.get())) return refuse(name, "changed during the call"), nullptr;
        const at::Tensor *t = tensor(PySequence_Fast_GET_ITEM(held.get(), i), name);
        if (t && (!c.here(*t) || !t->is_contiguous())) return refuse(name, "must be contiguous tensors on the context's device"), nullptr;
        return t;
    }
    void written_all() const {
        for (Py_ssize_t i = 0; held.get() && i < PySequence_Fast_GET_SIZE(held.get()); ++i) {
            PyObject *const o = PySequence_Fast_GET_ITEM(held.get(), i);
            if (THPVariable_Check(o)) written(THPVariable_Unpack(o));
        }
    }
};

// A number, or one in device memory: a CUDA tensor of one element of type `type`.
bool number_or_tensor(const Call &c, PyObject *o, const char *name, at::ScalarType type, void **at) {
    *at = nullptr;
    return !THPVariable_Check(o) || words(c, o, name, type, 1, at);
}

// adamw(ctx, device, params, grads, exp_avgs, exp_avg_sqs, exponents, copies, step, lr, beta1, beta2, eps, weight_decay, norm, max_norm, loss_scale, seed)
PyObject *py_adamw(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    List params, grads, ms, vs, exponents, copies;
    qgbdt_adamw_options o{};
    void *d_step, *d_lr, *d_norm;
    if (!c.take(args, nargs, 18) || !params.take(args[2], "params", -1) || !grads.take(args[3], "grads", params.n) || !ms.take(args[4], "exp_avgs", params.n) ||
        !vs.take(args[5], "exp_avg_sqs", params.n))
        return nullptr;
    const bool packed = args[6] != Py_None, copied = args[7] != Py_None;
    if ((packed && !exponents.take(args[6], "exponents", params.n)) || (copied && !copies.take(args[7], "copies", params.n))) return nullptr;
    if (!number_or_tensor(c, args[8], "step", at::kLong, &d_step) || !number_or_tensor(c, args[9], "lr", at::kFloat, &d_lr) ||
        !words(c, args[14], "norm", at::kFloat, 1, &d_norm))
        return nullptr;
    if (!d_step) o.step = PyLong_AsLongLong(args[8]);
    if (PyErr_Occurred()) return nullptr;
    if (!d_lr && !number(args[9], &o.lr)) return nullptr;
    if (!number(args[10], &o.beta1) || !number(args[11], &o.beta2) || !number(args[12], &o.eps) || !number(args[13], &o.weight_decay) ||
        !number(args[15], &o.max_norm) || !number(args[16], &o.loss_scale))
        return nullptr;
    o.seed = PyLong_AsUnsignedLongLongMask(args[17]);
    if (PyErr_Occurred()) return nullptr;
    o.d_step = (const int64_t *)d_step, o.d_lr = (const float *)d_lr, o.d_norm = (const float *)d_norm, o.state_bits = packed ? 8 : 32;
    std::vector<qgbdt_adamw_tensor> list((size_t)params.n);
    at::Tensor recorded;
    auto collect = [&] {
        for (Py_ssize_t i = 0; i < params.n; ++i) {
            const at::Tensor *p = params.get(c, i), *g = p ? grads.get(c, i) : nullptr, *m = g ? ms.get(c, i) : nullptr, *v = m ? vs.get(c, i) : nullptr;
            if (!v) return false;
            qgbdt_adamw_tensor &t = list[(size_t)i] = {};
            t.count = p->numel();
            t.param_type = element(*p), t.grad_type = element(*g);
            if (t.param_type < 0 || t.grad_type < 0) return refuse("params and grads must be float32, bfloat16 or float16"), false;
            if (g->numel() != t.count || m->numel() != t.count || v->numel() != t.count) return refuse("grads and states must match the parameters in sizes"), false;
            const at::ScalarType state = packed ? at::kByte : at::kFloat;
            if (m->scalar_type() != state || v->scalar_type() != state)
                return refuse(packed ? "states with exponents must be uint8" : "states must be float32 (or uint8, with exponents)"), false;
            if (followed(*g)) recorded = *g;
            t.param = p->data_ptr(), t.grad = g->data_ptr(), t.exp_avg = m->data_ptr(), t.exp_avg_sq = v->data_ptr();
            if (packed) {
                const at::Tensor *e = exponents.get(c, i);
                if (!e) return false;
                if (e->scalar_type() != at::kByte || e->dim() != 2 || e->size(0) != (t.count + 255) / 256 || e->size(1) != 2)
                    return refuse("exponents must be uint8 [ceil(elements / 256), 2]"), false;
                t.exponents = (uint8_t *)e->data_ptr();
            }
            if (copied && !copies.none(i)) {
                const at::Tensor *k = copies.get(c, i);
                if (!k) return false;
                t.copy_type = element(*k);
                if (t.copy_type < 0 || k->numel() != t.count) return refuse("copies must match the parameters in sizes and be float32, bfloat16 or float16"), false;
                t.copy = k->data_ptr();
            }
        }
        return true;
    };
    if (!collect()) return nullptr;
    // a warning's handler may have changed the lists, and with them what holds the tensors
    if (recorded.defined() && !(unrecorded(recorded, "grads") && collect())) return nullptr;
    const int rc = lib.adamw(c.ctx, list.data(), (int32_t)params.n, &o, c.stream);
    if (rc != QGBDT_OK) return c.result(rc);
    for (const List *l : {&params, &ms, &vs, &exponents, &copies}) l->written_all();
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// adamw_values(ctx, device, exp_avgs, exp_avg_sqs, exponents, bfloat16) -> (list of m, list of v)
PyObject *py_adamw_values(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    List ms, vs, exponents;
    if (!c.take(args, nargs, 6) || !ms.take(args[2], "exp_avgs", -1) || !vs.take(args[3], "exp_avg_sqs", ms.n) || !exponents.take(args[4], "exponents", ms.n))
        return nullptr;
    const int half = PyObject_IsTrue(args[5]);
    if (half < 0) return nullptr;
    std::vector<const uint8_t *> m, v, e;
    std::vector<at::Tensor> made[2];
    std::vector<void *> out[2];
    std::vector<int64_t> counts;
    for (Py_ssize_t i = 0; i < ms.n; ++i) {
        const at::Tensor *a = ms.get(c, i), *b = a ? vs.get(c, i) : nullptr, *x = b ? exponents.get(c, i) : nullptr;
        if (!x) return nullptr;
        const int64_t n = a->numel();
        if (a->scalar_type() != at::kByte || b->scalar_type() != at::kByte || b->numel() != n) return refuse("states must be uint8 and match in sizes");
        if (x->scalar_type() != at::kByte || x->dim() != 2 || x->size(0) != (n + 255) / 256 || x->size(1) != 2)
            return refuse("exponents must be uint8 [ceil(elements / 256), 2]");
        m.push_back((const uint8_t *)a->data_ptr()), v.push_back((const uint8_t *)b->data_ptr()), e.push_back((const uint8_t *)x->data_ptr());
        counts.push_back(n);
        for (int k = 0; k < 2; ++k) {
            made[k].push_back(fresh(a->sizes(), half ? at::kBFloat16 : at::kFloat, c));
            out[k].push_back(made[k].back().data_ptr());
        }
    }
    const int rc = lib.adamw_values(c.ctx, m.data(), v.data(), e.data(), out[0].data(), out[1].data(), counts.data(), (int32_t)ms.n,
                                    half ? QGBDT_BF16 : QGBDT_F32, c.stream);
    if (rc != QGBDT_OK) return c.result(rc);
    PyObject *lists[2];
    for (int k = 0; k < 2; ++k) {
        lists[k] = PyList_New(ms.n);
        if (!lists[k]) {
            if (k) Py_DECREF(lists[0]);
            return nullptr;
        }
        for (Py_ssize_t i = 0; i < ms.n; ++i) PyList_SET_ITEM(lists[k], i, THPVariable_Wrap(made[k][(size_t)i]));
    }
    return Py_BuildValue("(NN)", lists[0], lists[1]);
    END_HANDLE_TH_ERRORS
}

// bind(error class, addresses of embed, embed_backward, softmax_ce, softmax_ce_backward, clip_grad_norm, layer_norm, layer_norm_backward, adamw,
// adamw_values, last_error)
PyObject *py_bind(PyObject *, PyObject *args) {
    PyObject *error;
    unsigned long long p[10];
    if (!PyArg_ParseTuple(args, "OKKKKKKKKKK", &error, &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &p[7], &p[8], &p[9])) return nullptr;
    Py_INCREF(error);
    Py_XDECREF(lib.error);
    lib = Bound{reinterpret_cast<decltype(lib.embed)>(p[0]),          reinterpret_cast<decltype(lib.embed_backward)>(p[1]),
                reinterpret_cast<decltype(lib.softmax_ce)>(p[2]),     reinterpret_cast<decltype(lib.softmax_ce_backward)>(p[3]),
                reinterpret_cast<decltype(lib.clip_grad_norm)>(p[4]), reinterpret_cast<decltype(lib.layer_norm)>(p[5]),
                reinterpret_cast<decltype(lib.layer_norm_backward)>(p[6]), reinterpret_cast<decltype(lib.adamw)>(p[7]),
                reinterpret_cast<decltype(lib.adamw_values)>(p[8]),   reinterpret_cast<decltype(lib.last_error)>(p[9]), error};
    Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(embed), FAST(embed_backward), FAST(softmax_ce), FAST(softmax_ce_backward), FAST(clip_grad_norm),
                         FAST(layer_norm), FAST(layer_norm_backward), FAST(adamw), FAST(adamw_values),
                         {"bind", py_bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", "Argument marshalling of the operators on top of the trees.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
