// What the layer norm (csrc/layer_norm.cu) asks of the CUDA runtime, over a stand-in for it without a GPU: the launches for rows of
// all widths that are held in registers.
#include <cstdio>
#include <cstring>

#include "ops_internal.cuh"

#include "fake_cuda.h"

#ifndef __CUDA_ARCH__      // (for device code the headers define some of the runtime's calls)
// Shared memory of a block without leave for more, what k_ln_rows and k_ln_rows_backward hold besides what a launch gives them (2 x 32
// pairs of floats), and what a block can have at most.
constexpr int DEFAULT = 48 * 1024, OWN = 512, MOST = 227 * 1024;

static std::map<const void *, int> leave;      // bytes a launch may give a kernel, where that was set
static int launches = 0, failures = 0, lowered = 0;
static char what[160];

static void fail(const char *why, long a, long b) {
    if (++failures <= 20) printf("%s: %s (%ld, %ld)\n", what, why, a, b);
}
static int may(const void *f) { return leave.count(f) ? leave[f] : DEFAULT - OWN; }

extern "C" {
cudaError_t cudaFuncSetAttribute(const void *f, cudaFuncAttribute, int value) {
    if (value > MOST - OWN) fail("more shared memory than a block can have", value, 0);
    if (leave.count(f) && leave[f] > value) ++lowered;
    return leave[f] = value, cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int *n, const void *f, int, size_t smem, unsigned) {
    return *n = (long)smem > may(f) ? 0 : 2, cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *f, void **) {
    ++launches;
    if (c->gridDim.x < 1 || c->gridDim.y < 1) fail("an empty grid", c->gridDim.x, c->gridDim.y);
    if ((long)c->dynamicSmemBytes > may(f)) fail("more shared memory than the kernel has leave for", (long)c->dynamicSmemBytes, may(f));
    return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void *, dim3, dim3, void **, size_t, cudaStream_t) { return cudaErrorUnknown; }   // (not used)
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, cudaStream_t) { return 1; }
cudaError_t __cudaPopCallConfiguration(dim3 *, dim3 *, size_t *, void *) { return cudaErrorUnknown; }
void __cudaRegisterFunction(void **, const char *, char *, const char *, int, uint3 *, uint3 *, dim3 *, dim3 *, int *) {}
}
int qg_fail(qgbdt_ctx *, int code, const char *, ...) { return code; }
int qg_embed(qgbdt_ctx *, const EmbedArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_embed_backward(qgbdt_ctx *, const EmbedArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_softmax_ce(qgbdt_ctx *, const SoftmaxArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_softmax_ce_backward(qgbdt_ctx *, const SoftmaxArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_clip_grad_norm(qgbdt_ctx *, const void *const *, void *const *, const int64_t *, const int32_t *, int32_t, double, float *, cudaStream_t) { return QGBDT_OK; }

static qgbdt_ctx c;

static void call(bool backward, int type, int dim, int64_t rows, bool vectors) {
    char *const p = reinterpret_cast<char *>(0x100000);      // addresses that nothing reads
    snprintf(what, sizeof(what), "%s, type %d, %lld rows of %d columns%s", backward ? "gradients" : "forward", type, (long long)rows, dim, vectors ? "" : " that start anywhere");
    LayerNormArgs a{};
    a.x = p, a.weight = p, a.type = type, a.weight_type = QGBDT_F32, a.rows = rows, a.dim = dim, a.eps = 1e-5f;
    a.ld_x = a.ld_out = a.ld_grad = dim + (vectors ? 0 : 1);
    a.out = p, a.mean = a.rstd = reinterpret_cast<float *>(p);
    if (backward) a.grad = p, a.d_weight = a.d_bias = p;
    launches = 0;
    const int rc = backward ? qg_layer_norm_backward(&c, a, nullptr) : qg_layer_norm(&c, a, nullptr);
    if (rc != QGBDT_OK || launches == 0) fail("no launch", rc, launches);
    calls.clear();
}

// Rows of whole vectors from the smallest to the longest, those that fill their threads, the ends of the range whose copies ahead come
// to 48 KB; rows that start anywhere.
static std::vector<int> columns(int type, bool vectors) {
    std::vector<int> d;
    for (int i = vectors ? 8 : 1; i <= 16400; i += vectors ? 56 : 13) d.push_back(i);
    if (!vectors) return d;
    for (int i : {512, 1024, 2048, 2560, 2568, 3064, 3584, 4096, 5120, 5128, 6136, 6144, 8192, 12288, 14336, 16384}) d.push_back(i);
    if (type == QGBDT_F32)
        for (int i : {4, 100, 2564, 3068, 14340, 16380}) d.push_back(i);
    return d;
}

template <typename F>
static void all(F before) {
    for (const bool backward : {false, true})
        for (const int type : {QGBDT_F32, QGBDT_BF16, QGBDT_F16})
            for (const bool vectors : {true, false})
                for (const int dim : columns(type, vectors))
                    for (const int64_t rows : {1, 100, 100000}) {
                        before();
                        call(backward, type, dim, rows, vectors);
                    }
}

int main(int, char **argv) {
    c.sm_count = 148;
    if (!strcmp(argv[1], "first")) all([] { leave.clear(); });      // every call is the first one of its process
    else all([] {});                                                // one after the other
    if (lowered) printf("a kernel's leave for shared memory was lowered %d times\n", lowered);
    return failures || lowered ? 1 : 0;
}
#endif
