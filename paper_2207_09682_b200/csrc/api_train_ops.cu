// C ABI of the layer norm and of the AdamW step: argument checks.
#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "ops_internal.cuh"

namespace {

using wide = __int128;   // rows times their stride: up to 2^72 bytes

// Rows of `width` bytes, `step` apart.
struct Rows {
    const void *p;
    wide n, step, width;
    wide at() const { return (wide) reinterpret_cast<uintptr_t>(p); }
    wide end() const { return at() + (n - 1) * step + width; }
};

// The smallest x >= 0 with low <= a x mod m <= high, -1 if there is none; a < m, 0 <= low <= high < m.
// No multiple of a in [low, high]: a x - m y is in there for the smallest y whose m y mod a is in [-high, -low] mod a.
wide first_between(wide a, wide m, wide low, wide high) {
    if (low == 0) return 0;
    if (a == 0) return -1;
    const wide x = (low + a - 1) / a;
    if (x * a <= high) return x;
    const wide y = first_between(m % a, a, (a - high % a) % a, (a - low % a) % a);
    return y < 0 ? -1 : (low + m * y + a - 1) / a;
}

// Whether a row of a and a row of b have a byte in common.  Rows of one matrix may lie between another one's.
bool meet(const Rows &a, const Rows &b) {
    if (!a.p || !b.p || a.n < 1 || b.n < 1 || a.end() <= b.at() || b.end() <= a.at()) return false;
    if (a.n > 1 && b.n == 1) return meet(b, a);
    // row i of a begins t = from + i a.step behind b's first row; among b's rows from its first to its last
    const wide from = a.at() - b.at(), last = (b.n - 1) * b.step + b.width - 1, begin = -a.width + 1;
    const wide i0 = a.n == 1 || from >= begin ? 0 : (begin - from + a.step - 1) / a.step, i1 = a.n == 1 ? 0 : std::min(a.n - 1, (last - from) / a.step);
    if (i0 > i1 || b.n == 1) return i0 <= i1;
    // it meets one of them where (t - begin) mod b.step is `room` at most
    const wide room = a.width + b.width - 2, m = b.step, t = (from + i0 * a.step - begin) % m;
    if (t <= room || room >= m) return true;
    const wide i = first_between(a.step % m, m, m - t, m - t + room);
    return i >= 0 && i0 + i <= i1;
}

int check_layer_norm(qgbdt_ctx *c, LayerNormArgs &a, bool backward) {
    const int step = 16 / (a.type == QGBDT_F32 ? 4 : 2);
    qg_single_row(a.rows, a.dim, step, &a.ld_x);
    qg_single_row(a.rows, a.dim, step, &a.ld_out);
    if (backward) qg_single_row(a.rows, a.dim, step, &a.ld_grad);
    const int rc = qg_ops_enter(c);
    if (rc != QGBDT_OK) return rc;
    if (!qg_type_ok(a.type)) return qg_fail(c, QGBDT_ERR_ARG, "element type must be QGBDT_F32, QGBDT_BF16 or QGBDT_F16");
    if (a.weight_type != QGBDT_F32 && a.weight_type != a.type) return qg_fail(c, QGBDT_ERR_ARG, "weight_type must be QGBDT_F32 or the rows' type");
    if (a.rows < 0 || a.rows >= (1ll << 31)) return qg_fail(c, QGBDT_ERR_ARG, "rows must be in [0, 2^31)");
    if (a.dim < 1 || a.dim > (1 << 20)) return qg_fail(c, QGBDT_ERR_ARG, "dim must be in [1, 2^20]");
    if (a.ld_x < a.dim || a.ld_out < a.dim || (backward && a.ld_grad < a.dim)) return qg_fail(c, QGBDT_ERR_ARG, "a row stride is smaller than the row");
    const int64_t most = 1ll << 39;
    if (a.ld_x >= most || a.ld_out >= most || (backward && a.ld_grad >= most)) return qg_fail(c, QGBDT_ERR_ARG, "row strides must be below 2^39");
    if (a.rows > 0 && (!a.x || !a.out || (backward && (!a.grad || !a.mean || !a.rstd)))) return qg_fail(c, QGBDT_ERR_ARG, "null pointer");
    if (!(a.eps >= 0.0f) || !std::isfinite(a.eps)) return qg_fail(c, QGBDT_ERR_ARG, "eps must be finite and >= 0");
    const int w = qg_type_size(a.type), ww = qg_type_size(a.weight_type);
    if (!qg_aligned(a.x, w) || !qg_aligned(a.out, w) || !qg_aligned(a.grad, w) || !qg_aligned(a.weight, ww) || !qg_aligned(a.bias, ww) || !qg_aligned(a.d_weight, ww) ||
        !qg_aligned(a.d_bias, ww) || !qg_aligned(a.mean, 4) || !qg_aligned(a.rstd, 4))
        return qg_fail(c, QGBDT_ERR_ARG, "a pointer is not aligned to its element");
    // the output is one of the inputs, or apart from them all
    const Rows out{a.out, a.rows, (wide)a.ld_out * w, (wide)a.dim * w}, x{a.x, a.rows, (wide)a.ld_x * w, (wide)a.dim * w}, grad{a.grad, a.rows, (wide)a.ld_grad * w, (wide)a.dim * w};
    auto apart = [&](const Rows &in) { return (out.p == in.p && (out.n <= 1 || out.step == in.step)) || !meet(out, in); };
    if (!apart(x) || !apart(grad)) return qg_fail(c, QGBDT_ERR_ARG, "the output's rows overlap an input's and are not the same");
    for (const Rows &in : {Rows{a.weight, 1, 0, (wide)a.dim * ww}, Rows{a.bias, 1, 0, (wide)a.dim * ww}, Rows{a.mean, 1, 0, (wide)a.rows * 4}, Rows{a.rstd, 1, 0, (wide)a.rows * 4}})
        if (meet(out, in)) return qg_fail(c, QGBDT_ERR_ARG, "the output's rows overlap the weight, the bias, mean or rstd");
    return QGBDT_OK;
}

// Whether two of the ranges overlap; `at` and `bytes` give entry i's.
template <typename A, typename B>
int overlapping(qgbdt_ctx *c, int32_t n, A at, B bytes, bool *found) {
    *found = false;
    uintptr_t end = 0;
    bool ascending = true;   // as tensors of one buffer are: nothing to sort
    for (int32_t i = 0; i < n && ascending; ++i) {
        if (bytes(i) == 0) continue;
        ascending = at(i) >= end;
        end = at(i) + bytes(i);
    }
    if (ascending) return QGBDT_OK;
    try {
        std::vector<std::pair<uintptr_t, uintptr_t>> r;
        for (int32_t i = 0; i < n; ++i)
            if (bytes(i)) r.emplace_back(at(i), at(i) + bytes(i));
        std::sort(r.begin(), r.end());
        for (size_t i = 1; i < r.size(); ++i) *found = *found || r[i].first < r[i - 1].second;
    } catch (const std::bad_alloc &) {
        return qg_fail(c, QGBDT_ERR_ALLOC, "no host memory to look the tensors over");
    }
    return QGBDT_OK;
}

int check_adamw(qgbdt_ctx *c, const qgbdt_adamw_tensor *t, int32_t n, const qgbdt_adamw_options *o) {
    int rc = qg_ops_enter(c);
    if (rc != QGBDT_OK) return rc;
    if (n < 0 || n > (1 << 20)) return qg_fail(c, QGBDT_ERR_ARG, "n_tensors must be in [0, 2^20]");
    if (!o || (n > 0 && !t)) return qg_fail(c, QGBDT_ERR_ARG, "null pointer");
    if (o->state_bits != 32 && o->state_bits != 8) return qg_fail(c, QGBDT_ERR_ARG, "state_bits must be 32 or 8");
    if (!(o->beta1 >= 0.0 && o->beta1 < 1.0) || !(o->beta2 >= 0.0 && o->beta2 < 1.0)) return qg_fail(c, QGBDT_ERR_ARG, "beta1 and beta2 must be in [0, 1)");
    if (!(o->eps >= 0.0) || !std::isfinite(o->eps)) return qg_fail(c, QGBDT_ERR_ARG, "eps must be finite and >= 0");
    if (!(o->weight_decay >= 0.0) || !std::isfinite(o->weight_decay)) return qg_fail(c, QGBDT_ERR_ARG, "weight_decay must be finite and >= 0");
    if (!o->d_lr && (!(o->lr >= 0.0) || !std::isfinite(o->lr))) return qg_fail(c, QGBDT_ERR_ARG, "lr must be finite and >= 0");
    if (!o->d_step && o->step < 1) return qg_fail(c, QGBDT_ERR_ARG, "step must be >= 1");
    if (o->d_norm && !(o->max_norm >= 0.0)) return qg_fail(c, QGBDT_ERR_ARG, "max_norm must be >= 0 (infinity: no clipping)");
    if (!(o->loss_scale >= 0x1p-127) || !std::isfinite(o->loss_scale)) return qg_fail(c, QGBDT_ERR_ARG, "loss_scale must be finite and >= 2^-127");
    if (!qg_aligned(o->d_lr, 4) || !qg_aligned(o->d_step, 8) || !qg_aligned(o->d_norm, 4)) return qg_fail(c, QGBDT_ERR_ARG, "a pointer is not aligned to its element");
    const bool packed = o->state_bits == 8;
    int64_t blocks = 0;
    for (int32_t i = 0; i < n; ++i) {
        const qgbdt_adamw_tensor &a = t[i];
        if (a.count < 0 || a.count > (1ll << 40)) return qg_fail(c, QGBDT_ERR_ARG, "tensor %d: the size must be in [0, 2^40]", i);
        if (!qg_type_ok(a.param_type) || !qg_type_ok(a.grad_type) || (a.copy && !qg_type_ok(a.copy_type)))
            return qg_fail(c, QGBDT_ERR_ARG, "tensor %d: element type must be QGBDT_F32, QGBDT_BF16 or QGBDT_F16", i);
        if (a.count == 0) continue;
        if (!a.param || !a.grad || !a.exp_avg || !a.exp_avg_sq || (packed && !a.exponents)) return qg_fail(c, QGBDT_ERR_ARG, "tensor %d is NULL", i);
        const int state = packed ? 1 : 4;
        if (!qg_aligned(a.param, qg_type_size(a.param_type)) || !qg_aligned(a.grad, qg_type_size(a.grad_type)) || !qg_aligned(a.exp_avg, state) ||
            !qg_aligned(a.exp_avg_sq, state) || (a.copy && !qg_aligned(a.copy, qg_type_size(a.copy_type))))
            return qg_fail(c, QGBDT_ERR_ARG, "tensor %d is not aligned to its element", i);
        // what the step writes of this tensor, and the gradient that it reads
        const void *const at[] = {a.param, a.exp_avg, a.exp_avg_sq, a.copy, packed ? a.exponents : nullptr, a.grad};
        const int64_t bytes[] = {a.count * qg_type_size(a.param_type), a.count * state, a.count * state, a.count * qg_type_size(a.copy_type), (a.count + 255) / 256 * 2,
                                 a.count * qg_type_size(a.grad_type)};
        for (int j = 0; j < 6; ++j)
            for (int k = 0; k < j; ++k)
                if (at[j] && at[k] && reinterpret_cast<uintptr_t>(at[j]) < reinterpret_cast<uintptr_t>(at[k]) + (uintptr_t)bytes[k] &&
                    reinterpret_cast<uintptr_t>(at[k]) < reinterpret_cast<uintptr_t>(at[j]) + (uintptr_t)bytes[j])
                    return qg_fail(c, QGBDT_ERR_ARG, "tensor %d: parameters, gradient, states and copy overlap", i);
        blocks += (a.count + 255) / 256;
        if (blocks >= (1ll << 32)) return qg_fail(c, QGBDT_ERR_ARG, "the tensors have 2^40 elements or more together");
    }
    bool twice = false;
    rc = overlapping(c, n, [&](int32_t i) { return reinterpret_cast<uintptr_t>(t[i].param); },
                     [&](int32_t i) { return (uintptr_t)t[i].count * qg_type_size(t[i].param_type); }, &twice);
    if (rc == QGBDT_OK && twice) rc = qg_fail(c, QGBDT_ERR_ARG, "two tensors of parameters overlap");
    return rc;
}

}  // namespace

extern "C" {

int qgbdt_layer_norm(qgbdt_ctx *c, const void *d_x, int64_t ld_x, int32_t type, const void *d_weight, const void *d_bias, int32_t weight_type,
                     int64_t n_rows, int32_t dim, double eps, void *d_out, int64_t ld_out, float *d_mean, float *d_rstd, void *stream) {
    LayerNormArgs a{};
    a.x = d_x, a.ld_x = ld_x, a.type = type, a.weight = d_weight, a.bias = d_bias, a.weight_type = weight_type, a.rows = n_rows, a.dim = dim;
    a.eps = (float)eps, a.out = d_out, a.ld_out = ld_out, a.mean = d_mean, a.rstd = d_rstd;
    const int rc = check_layer_norm(c, a, false);
    if (rc != QGBDT_OK || n_rows == 0) return rc;
    return qg_ops_leave(c, qg_layer_norm(c, a, (cudaStream_t)stream), stream);
}

int qgbdt_layer_norm_backward(qgbdt_ctx *c, const void *d_grad, int64_t ld_grad, const void *d_x, int64_t ld_x, int32_t type, const float *d_mean,
                              const float *d_rstd, const void *d_weight, int32_t weight_type, int64_t n_rows, int32_t dim, void *d_grad_x,
                              int64_t ld_grad_x, void *d_grad_weight, void *d_grad_bias, void *stream) {
    LayerNormArgs a{};
    a.grad = d_grad, a.ld_grad = ld_grad, a.x = d_x, a.ld_x = ld_x, a.type = type, a.weight = d_weight, a.weight_type = weight_type, a.rows = n_rows;
    a.dim = dim, a.mean = const_cast<float *>(d_mean), a.rstd = const_cast<float *>(d_rstd), a.out = d_grad_x, a.ld_out = ld_grad_x;
    a.d_weight = d_grad_weight, a.d_bias = d_grad_bias;
    const int rc = check_layer_norm(c, a, true);
    if (rc != QGBDT_OK) return rc;
    return qg_ops_leave(c, qg_layer_norm_backward(c, a, (cudaStream_t)stream), stream);
}

int qgbdt_adamw(qgbdt_ctx *c, const qgbdt_adamw_tensor *h_tensors, int32_t n_tensors, const qgbdt_adamw_options *h_options, void *stream) {
    const int rc = check_adamw(c, h_tensors, n_tensors, h_options);
    if (rc != QGBDT_OK) return rc;
    return qg_ops_leave(c, qg_adamw(c, h_tensors, n_tensors, *h_options, (cudaStream_t)stream), stream);
}

int qgbdt_adamw_values(qgbdt_ctx *c, const uint8_t *const *h_exp_avg, const uint8_t *const *h_exp_avg_sq, const uint8_t *const *h_exponents,
                       void *const *h_m, void *const *h_v, const int64_t *h_counts, int32_t n_tensors, int32_t type, void *stream) {
    const int rc = qg_ops_enter(c);
    if (rc != QGBDT_OK) return rc;
    if (n_tensors < 0 || n_tensors > (1 << 20)) return qg_fail(c, QGBDT_ERR_ARG, "n_tensors must be in [0, 2^20]");
    if (n_tensors > 0 && (!h_exp_avg || !h_exp_avg_sq || !h_exponents || !h_m || !h_v || !h_counts)) return qg_fail(c, QGBDT_ERR_ARG, "null pointer");
    if (type != QGBDT_F32 && type != QGBDT_BF16) return qg_fail(c, QGBDT_ERR_ARG, "the values' type must be QGBDT_F32 or QGBDT_BF16");
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (h_counts[i] < 0 || h_counts[i] > (1ll << 40)) return qg_fail(c, QGBDT_ERR_ARG, "tensor %d: the size must be in [0, 2^40]", i);
        if (h_counts[i] == 0) continue;
        if (!h_exp_avg[i] || !h_exp_avg_sq[i] || !h_exponents[i] || !h_m[i] || !h_v[i]) return qg_fail(c, QGBDT_ERR_ARG, "tensor %d is NULL", i);
        if (!qg_aligned(h_m[i], qg_type_size(type)) || !qg_aligned(h_v[i], qg_type_size(type))) return qg_fail(c, QGBDT_ERR_ARG, "tensor %d is not aligned to its element", i);
    }
    return qg_ops_leave(c, qg_adamw_values(c, h_exp_avg, h_exp_avg_sq, h_exponents, h_m, h_v, h_counts, n_tensors, type, (cudaStream_t)stream), stream);
}

}  // extern "C"
