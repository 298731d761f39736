// Which outputs the layer norm's C calls (csrc/api_train_ops.cu) take beside which inputs, over a stand-in for the CUDA runtime: every
// answer against a count of the bytes.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "ops_internal.cuh"

#include "fake_cuda.h"

int qg_fail(qgbdt_ctx *, int code, const char *, ...) { return code; }
int qg_embed(qgbdt_ctx *, const EmbedArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_embed_backward(qgbdt_ctx *, const EmbedArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_softmax_ce(qgbdt_ctx *, const SoftmaxArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_softmax_ce_backward(qgbdt_ctx *, const SoftmaxArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_clip_grad_norm(qgbdt_ctx *, const void *const *, void *const *, const int64_t *, const int32_t *, int32_t, double, float *, cudaStream_t) { return QGBDT_OK; }
int qg_layer_norm(qgbdt_ctx *, const LayerNormArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_layer_norm_backward(qgbdt_ctx *, const LayerNormArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_adamw(qgbdt_ctx *, const qgbdt_adamw_tensor *, int32_t, const qgbdt_adamw_options &, cudaStream_t) { return QGBDT_OK; }
int qg_adamw_values(qgbdt_ctx *, const uint8_t *const *, const uint8_t *const *, const uint8_t *const *, void *const *, void *const *, const int64_t *, int32_t, int32_t,
                    cudaStream_t) {
    return QGBDT_OK;
}

static qgbdt_ctx c;
static char *const P = reinterpret_cast<char *>(1ll << 40);   // addresses that nothing reads
static float *const S = reinterpret_cast<float *>(1ll << 41);

static std::vector<bool> touched(int at, int rows, int ld, int dim) {
    std::vector<bool> t(4000, false);
    for (int i = 0; i < rows; ++i)
        for (int j = 0; j < dim; ++j) t[(size_t)(at + i * ld + j)] = true;
    return t;
}
static bool meet(const std::vector<bool> &a, const std::vector<bool> &b) {
    for (size_t i = 0; i < a.size(); ++i)
        if (a[i] && b[i]) return true;
    return false;
}
static int pick(int lo, int hi) { return lo + rand() % (hi - lo + 1); }

int main() {
    int failures = 0, refused = 0, between = 0, tries = 40000;
    srand(1);
    for (int k = 0; k < tries; ++k) {
        const int dim = pick(1, 12), rows = pick(1, 30), ldx = dim + pick(0, 40), ldo = k % 3 ? dim + pick(0, 40) : ldx, atx = pick(0, 300), ato = k % 5 ? pick(0, 300) : atx;
        const int ldg = dim + pick(0, 40), atg = 1700 + pick(0, 40);
        const auto x = touched(atx, rows, ldx, dim), out = touched(ato, rows, ldo, dim), g = touched(atg, rows, ldg, dim);
        char *const px = P + 4 * atx, *const po = P + 4 * ato, *const pg = P + 4 * atg;
        bool bad = meet(x, out) && !(atx == ato && (rows == 1 || ldx == ldo));
        int rc = qgbdt_layer_norm(&c, px, ldx, QGBDT_F32, nullptr, nullptr, QGBDT_F32, rows, dim, 1e-5, po, ldo, S, S + 64, nullptr);
        if (rc != (bad ? QGBDT_ERR_ARG : QGBDT_OK) && ++failures <= 20)
            printf("%d rows of %d: x at %d, %d apart, out at %d, %d apart: %d, bytes meet: %d\n", rows, dim, atx, ldx, ato, ldo, rc, (int)bad);
        refused += bad, between += !bad && ato < atx + (rows - 1) * ldx + dim && atx < ato + (rows - 1) * ldo + dim;
        bad = bad || meet(g, out);
        rc = qgbdt_layer_norm_backward(&c, pg, ldg, px, ldx, QGBDT_F32, S, S + 64, nullptr, QGBDT_F32, rows, dim, po, ldo, nullptr, nullptr, nullptr);
        const int swapped = qgbdt_layer_norm_backward(&c, px, ldx, pg, ldg, QGBDT_F32, S, S + 64, nullptr, QGBDT_F32, rows, dim, po, ldo, nullptr, nullptr, nullptr);
        if ((rc != (bad ? QGBDT_ERR_ARG : QGBDT_OK) || swapped != rc) && ++failures <= 20) printf("gradients, %d rows of %d: %d, %d, bytes meet: %d\n", rows, dim, rc, swapped, (int)bad);
        // the columns' weight and the rows' mean inside, between or beside the output's rows
        const int at = pick(0, 400), atm = pick(0, 400);
        const bool w = meet(touched(at, 1, dim, dim), out), m = meet(touched(atm, 1, rows, rows), out);
        char *const far = P + 40000;
        rc = qgbdt_layer_norm(&c, far, dim, QGBDT_F32, P + 4 * at, nullptr, QGBDT_F32, rows, dim, 1e-5, po, ldo, reinterpret_cast<float *>(P + 4 * atm), S, nullptr);
        if (rc != (w || m ? QGBDT_ERR_ARG : QGBDT_OK) && ++failures <= 20) printf("%d rows of %d: weight %d, mean %d: %d\n", rows, dim, (int)w, (int)m, rc);
    }
    if (refused < tries / 10 || between < tries / 10) printf("%d refused and %d between one another are too few\n", refused, between), ++failures;
    // the largest numbers: rows that lie 2^40 bytes apart, 2^31 - 1 of them, beside ones that fall between
    const int64_t most = (1ll << 31) - 1, ld = (1ll << 39) - 1;
    const auto far = [&](int64_t by, int64_t ldo) { return qgbdt_layer_norm(&c, P, ld, QGBDT_BF16, nullptr, nullptr, QGBDT_F32, most, 100, 1e-5, P + by, ldo, nullptr, nullptr, nullptr); };
    if (far(200, ld) != QGBDT_OK || far(198, ld) != QGBDT_ERR_ARG || far(0, ld) != QGBDT_OK || far(0, ld - 1) != QGBDT_ERR_ARG || far(-200, ld) != QGBDT_OK ||
        far(-198, ld) != QGBDT_ERR_ARG || far(200, ld - 1) != QGBDT_ERR_ARG)
        printf("rows far apart\n"), ++failures;
    return failures ? 1 : 0;
}
