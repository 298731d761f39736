// The argument checks of the layer norm and the AdamW step (csrc/api_train_ops.cu) over a stand-in for the CUDA runtime, without
// a GPU: what the C calls take, what they refuse before anything is launched.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "ops_internal.cuh"

#include "fake_cuda.h"

static int launched = 0;
static LayerNormArgs seen;
int qg_fail(qgbdt_ctx *, int code, const char *, ...) { return code; }
int qg_embed(qgbdt_ctx *, const EmbedArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_embed_backward(qgbdt_ctx *, const EmbedArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_softmax_ce(qgbdt_ctx *, const SoftmaxArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_softmax_ce_backward(qgbdt_ctx *, const SoftmaxArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_clip_grad_norm(qgbdt_ctx *, const void *const *, void *const *, const int64_t *, const int32_t *, int32_t, double, float *, cudaStream_t) { return QGBDT_OK; }
int qg_layer_norm(qgbdt_ctx *, const LayerNormArgs &a, cudaStream_t) { return seen = a, ++launched, QGBDT_OK; }
int qg_layer_norm_backward(qgbdt_ctx *, const LayerNormArgs &a, cudaStream_t) { return seen = a, ++launched, QGBDT_OK; }
int qg_adamw(qgbdt_ctx *, const qgbdt_adamw_tensor *, int32_t, const qgbdt_adamw_options &, cudaStream_t) { return ++launched, QGBDT_OK; }
int qg_adamw_values(qgbdt_ctx *, const uint8_t *const *, const uint8_t *const *, const uint8_t *const *, void *const *, void *const *, const int64_t *, int32_t, int32_t,
                    cudaStream_t) {
    return ++launched, QGBDT_OK;
}

static int failures = 0;
static void expect(bool ok, int line, const char *what) {
    if (!ok) printf("line %d: %s does not hold\n", line, what), ++failures;
}
#define TAKEN(call)                                                                                  \
    do {                                                                                             \
        launched = 0;                                                                                \
        expect((call) == QGBDT_OK && launched == 1, __LINE__, "taken: " #call);                      \
    } while (0)
#define NOTHING(call)                                                                                \
    do {                                                                                             \
        launched = 0;                                                                                \
        expect((call) == QGBDT_OK && launched == 0, __LINE__, "taken, nothing to do: " #call);       \
    } while (0)
#define REFUSED(call)                                                                                \
    do {                                                                                             \
        launched = 0;                                                                                \
        expect((call) == QGBDT_ERR_ARG && launched == 0, __LINE__, "refused: " #call);               \
    } while (0)

static qgbdt_ctx c;
static char *const P = reinterpret_cast<char *>(0x10000);   // addresses that nothing reads
static float *const F = reinterpret_cast<float *>(0x20000);

struct Norm {   // a call that is in order, to be changed in one place
    const void *x = P, *w = P, *b = P;
    int64_t ldx = 20, rows = 3, ldo = 24;
    int32_t type = QGBDT_BF16, wtype = QGBDT_F32, dim = 20;
    double eps = 1e-5;
    void *out = P + 4096;
    float *mean = F, *rstd = F;
    const void *grad = P;
    int64_t ldg = 20;
    void *dw = P, *db = P;
    int forward() const { return qgbdt_layer_norm(&c, x, ldx, type, w, b, wtype, rows, dim, eps, out, ldo, mean, rstd, nullptr); }
    int backward() const { return qgbdt_layer_norm_backward(&c, grad, ldg, x, ldx, type, mean, rstd, w, wtype, rows, dim, out, ldo, dw, db, nullptr); }
    template <typename T, typename V>
    Norm with(T Norm::*m, V v) const {
        Norm n = *this;
        n.*m = v;
        return n;
    }
};

struct Step {
    std::vector<qgbdt_adamw_tensor> t;
    qgbdt_adamw_options o{};
    Step() {
        o.lr = 0.1, o.beta1 = 0.9, o.beta2 = 0.999, o.eps = 1e-8, o.max_norm = 1.0, o.loss_scale = 1.0, o.step = 1, o.state_bits = 32;
        for (int i = 0; i < 3; ++i) {
            qgbdt_adamw_tensor a{};
            a.param = P + 4096 * i, a.grad = P + 0x20000, a.exp_avg = P + 0x30000, a.exp_avg_sq = P + 0x40000, a.count = 1000, a.param_type = QGBDT_F32, a.grad_type = QGBDT_BF16;
            a.copy_type = 77;   // of no meaning without a copy
            t.push_back(a);
        }
    }
    int run() const { return qgbdt_adamw(&c, t.data(), (int32_t)t.size(), &o, nullptr); }
    template <typename T, typename V>
    Step with(T qgbdt_adamw_options::*m, V v) const {
        Step s = *this;
        s.o.*m = v;
        return s;
    }
    template <typename T, typename V>
    Step with(T qgbdt_adamw_tensor::*m, V v) const {   // of the second tensor
        Step s = *this;
        s.t[1].*m = v;
        return s;
    }
};

int main() {
    const Norm n;
    TAKEN(n.forward());
    TAKEN(n.backward());
    TAKEN(n.with(&Norm::w, nullptr).with(&Norm::b, nullptr).with(&Norm::mean, nullptr).with(&Norm::rstd, nullptr).forward());
    TAKEN(n.with(&Norm::w, nullptr).with(&Norm::dw, nullptr).with(&Norm::db, nullptr).backward());
    TAKEN(n.with(&Norm::wtype, QGBDT_BF16).forward());
    TAKEN(n.with(&Norm::eps, 0.0).forward());
    TAKEN(n.with(&Norm::dim, 1).forward());
    NOTHING(n.with(&Norm::rows, 0).with(&Norm::x, nullptr).with(&Norm::out, nullptr).forward());
    TAKEN(n.with(&Norm::rows, 0).with(&Norm::x, nullptr).with(&Norm::grad, nullptr).with(&Norm::out, nullptr).with(&Norm::mean, nullptr).with(&Norm::rstd, nullptr).backward());
    TAKEN(n.with(&Norm::rows, 1).with(&Norm::ldx, 1ll << 60).forward());   // means nothing
    expect(seen.ld_x < 64 && seen.ld_x >= 20, __LINE__, "the stride of a single row is replaced");
    for (int64_t rows : {-1ll, 1ll << 31}) {
        REFUSED(n.with(&Norm::rows, rows).forward());
        REFUSED(n.with(&Norm::rows, rows).backward());
    }
    for (int32_t dim : {0, -1, 21, (1 << 20) + 1}) {   // 21: wider than a stride
        REFUSED(n.with(&Norm::dim, dim).forward());
        REFUSED(n.with(&Norm::dim, dim).backward());
    }
    for (int32_t type : {-1, 3, 77}) REFUSED(n.with(&Norm::type, type).forward());
    for (int32_t type : {-1, (int)QGBDT_F16, 77}) {
        REFUSED(n.with(&Norm::wtype, type).forward());
        REFUSED(n.with(&Norm::wtype, type).backward());
    }
    for (double eps : {-1e-5, (double)NAN, (double)INFINITY, 1e60}) REFUSED(n.with(&Norm::eps, eps).forward());
    for (int64_t ld : {19ll, 0ll, -20ll, 1ll << 39}) {
        REFUSED(n.with(&Norm::ldx, ld).forward());
        REFUSED(n.with(&Norm::ldo, ld).forward());
        REFUSED(n.with(&Norm::ldx, ld).backward());
        REFUSED(n.with(&Norm::ldo, ld).backward());
        REFUSED(n.with(&Norm::ldg, ld).backward());
    }
    REFUSED(n.with(&Norm::x, nullptr).forward());
    REFUSED(n.with(&Norm::out, nullptr).forward());
    REFUSED(n.with(&Norm::x, nullptr).backward());
    REFUSED(n.with(&Norm::grad, nullptr).backward());
    REFUSED(n.with(&Norm::mean, nullptr).backward());
    REFUSED(n.with(&Norm::rstd, nullptr).backward());
    REFUSED(n.with(&Norm::out, nullptr).backward());
    REFUSED(n.with(&Norm::x, P + 1).forward());
    REFUSED(n.with(&Norm::w, P + 2).forward());
    REFUSED(n.with(&Norm::out, P + 1).forward());
    REFUSED(n.with(&Norm::grad, P + 1).backward());
    REFUSED(n.with(&Norm::dw, P + 2).backward());
    REFUSED(n.with(&Norm::mean, reinterpret_cast<float *>(P + 2)).forward());
    REFUSED(qgbdt_layer_norm(nullptr, P, 20, 0, P, P, 0, 3, 20, 1e-5, P, 20, F, F, nullptr));

    const Step s;
    TAKEN(s.run());
    TAKEN(qgbdt_adamw(&c, nullptr, 0, &s.o, nullptr));
    TAKEN(s.with(&qgbdt_adamw_options::state_bits, 8).with(&qgbdt_adamw_tensor::count, 0).with(&qgbdt_adamw_options::state_bits, 32).run());
    {
        Step e = s;
        e.t[1] = qgbdt_adamw_tensor{};   // no elements: nothing is looked at
        TAKEN(e.run());
        e = s;
        e.o.state_bits = 8;
        REFUSED(e.run());   // without exponents
        for (qgbdt_adamw_tensor &a : e.t) a.exponents = reinterpret_cast<uint8_t *>(P + 0x50001), a.exp_avg = P + 0x30001, a.exp_avg_sq = P + 0x40003;
        TAKEN(e.run());
        e = s;
        std::swap(e.t[0].param, e.t[2].param);   // in any order
        TAKEN(e.run());
        e.t[1].param = e.t[0].param;
        REFUSED(e.run());
        e.t[1].param = reinterpret_cast<char *>(e.t[0].param) + 3996;   // the last element
        REFUSED(e.run());
        e = s;
        std::swap(e.t[0].param, e.t[2].param);
        no_memory = true;
        expect(e.run() == QGBDT_ERR_ALLOC, __LINE__, "no host memory is an error code");
        no_memory = false;
        e = s;
        for (int i = 0; i < 3; ++i) {   // too many together
            qgbdt_adamw_tensor &a = e.t[(size_t)i];
            char *const at = P + ((int64_t)(i + 1) << 46);
            a.count = 1ll << 39, a.param = at, a.grad = at + (1ll << 43), a.exp_avg = at + (2ll << 43), a.exp_avg_sq = at + (3ll << 43);
        }
        REFUSED(e.run());
        e.t.pop_back();
        REFUSED(e.run());   // 2^40 elements
    }
    REFUSED(qgbdt_adamw(&c, s.t.data(), 3, nullptr, nullptr));
    REFUSED(qgbdt_adamw(&c, nullptr, 3, &s.o, nullptr));
    REFUSED(qgbdt_adamw(&c, s.t.data(), -1, &s.o, nullptr));
    REFUSED(qgbdt_adamw(nullptr, s.t.data(), 3, &s.o, nullptr));
    for (double v : {-0.1, 1.0, (double)NAN, (double)INFINITY}) {
        REFUSED(s.with(&qgbdt_adamw_options::beta1, v).run());
        REFUSED(s.with(&qgbdt_adamw_options::beta2, v).run());
    }
    for (double v : {-0.1, (double)NAN, (double)INFINITY}) {
        REFUSED(s.with(&qgbdt_adamw_options::lr, v).run());
        REFUSED(s.with(&qgbdt_adamw_options::eps, v).run());
        REFUSED(s.with(&qgbdt_adamw_options::weight_decay, v).run());
        REFUSED(s.with(&qgbdt_adamw_options::loss_scale, v).run());
        TAKEN(s.with(&qgbdt_adamw_options::lr, v).with(&qgbdt_adamw_options::d_lr, F).run());
    }
    REFUSED(s.with(&qgbdt_adamw_options::loss_scale, 0.0).run());
    REFUSED(s.with(&qgbdt_adamw_options::max_norm, -1.0).with(&qgbdt_adamw_options::d_norm, F).run());
    REFUSED(s.with(&qgbdt_adamw_options::max_norm, (double)NAN).with(&qgbdt_adamw_options::d_norm, F).run());
    TAKEN(s.with(&qgbdt_adamw_options::max_norm, (double)INFINITY).with(&qgbdt_adamw_options::d_norm, F).run());
    for (int64_t v : {0ll, -1ll}) {
        REFUSED(s.with(&qgbdt_adamw_options::step, v).run());
        TAKEN(s.with(&qgbdt_adamw_options::step, v).with(&qgbdt_adamw_options::d_step, reinterpret_cast<int64_t *>(P)).run());
    }
    REFUSED(s.with(&qgbdt_adamw_options::d_step, reinterpret_cast<int64_t *>(P + 4)).run());
    REFUSED(s.with(&qgbdt_adamw_options::d_lr, reinterpret_cast<float *>(P + 2)).run());
    REFUSED(s.with(&qgbdt_adamw_options::d_norm, reinterpret_cast<float *>(P + 2)).run());
    for (int32_t v : {0, 16, 4}) REFUSED(s.with(&qgbdt_adamw_options::state_bits, v).run());
    for (int32_t v : {-1, 3}) {
        REFUSED(s.with(&qgbdt_adamw_tensor::param_type, v).run());
        REFUSED(s.with(&qgbdt_adamw_tensor::grad_type, v).run());
        REFUSED(s.with(&qgbdt_adamw_tensor::copy, P + 0x60000).with(&qgbdt_adamw_tensor::copy_type, v).run());
    }
    // what belongs to one tensor overlaps: the first and the last byte
    for (char *at : {P + 0x30000, P + 0x30000 + 3996, P + 0x30000 - 3996, P + 4096, P + 0x20000}) REFUSED(s.with(&qgbdt_adamw_tensor::exp_avg_sq, at).run());
    TAKEN(s.with(&qgbdt_adamw_tensor::exp_avg_sq, P + 0x30000 + 4000).run());
    TAKEN(s.with(&qgbdt_adamw_tensor::exp_avg_sq, P + 0x30000 - 4000).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::copy, P + 4096).with(&qgbdt_adamw_tensor::copy_type, QGBDT_F32).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::copy, P + 4096 - 1998).with(&qgbdt_adamw_tensor::copy_type, QGBDT_BF16).run());
    TAKEN(s.with(&qgbdt_adamw_tensor::copy, P + 0x60000).with(&qgbdt_adamw_tensor::copy_type, QGBDT_BF16).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::count, -1).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::param, nullptr).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::grad, nullptr).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::exp_avg, nullptr).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::exp_avg_sq, nullptr).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::param, P + 4098).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::grad, P + 1).run());
    REFUSED(s.with(&qgbdt_adamw_tensor::exp_avg, P + 2).run());

    const uint8_t *in[2] = {reinterpret_cast<uint8_t *>(P), nullptr};
    void *out[2] = {P, nullptr}, *odd[2] = {P + 2, nullptr};
    const int64_t counts[2] = {300, 0}, negative[2] = {300, -1}, both[2] = {300, 300};
    TAKEN(qgbdt_adamw_values(&c, in, in, in, out, out, counts, 2, QGBDT_F32, nullptr));
    TAKEN(qgbdt_adamw_values(&c, in, in, in, odd, out, counts, 2, QGBDT_BF16, nullptr));
    TAKEN(qgbdt_adamw_values(&c, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, QGBDT_F32, nullptr));
    REFUSED(qgbdt_adamw_values(&c, in, in, in, odd, out, counts, 2, QGBDT_F32, nullptr));
    REFUSED(qgbdt_adamw_values(&c, in, in, in, out, out, counts, 2, QGBDT_F16, nullptr));
    REFUSED(qgbdt_adamw_values(&c, in, in, in, out, out, negative, 2, QGBDT_F32, nullptr));
    REFUSED(qgbdt_adamw_values(&c, in, in, in, out, out, both, 2, QGBDT_F32, nullptr));
    REFUSED(qgbdt_adamw_values(&c, in, nullptr, in, out, out, counts, 2, QGBDT_F32, nullptr));
    REFUSED(qgbdt_adamw_values(&c, in, in, in, out, out, counts, -1, QGBDT_F32, nullptr));

    // a loss scale whose inverse single precision does not hold would make NaN of gradients that are zero
    for (double v : {1e-300, 1e-39, 0x1p-128}) REFUSED(s.with(&qgbdt_adamw_options::loss_scale, v).run());
    for (double v : {0x1p-127, 1e-38, 1e300}) TAKEN(s.with(&qgbdt_adamw_options::loss_scale, v).run());
    return failures ? 1 : 0;
}
