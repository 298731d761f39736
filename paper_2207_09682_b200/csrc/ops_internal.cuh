// Shared by the operators that sit on top of the trees (embedding of leaf numbers, layer norm, softmax
// cross entropy, clipping by the gradient norm, AdamW): element types, vector loads, the context's workspace.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "qgbdt_internal.cuh"

// ---- element types -------------------------------------------------------------------------------

template <typename T>
struct OpsType;
template <>
struct OpsType<float> {
    static __device__ __forceinline__ float load(float x) { return x; }
    static __device__ __forceinline__ float store(float x) { return x; }
};
template <>
struct OpsType<__nv_bfloat16> {
    static constexpr bool BF16 = true;
    static __device__ __forceinline__ float load(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 store(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct OpsType<__half> {
    static constexpr bool BF16 = false;
    static __device__ __forceinline__ float load(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half store(float x) { return __float2half_rn(x); }
};

// N elements moved by one load or store of N * sizeof(T) bytes.
template <typename T, int N>
struct alignas(sizeof(T) * N) OpsVec {
    T v[N];
};

static inline int qg_type_size(int type) { return type == QGBDT_F32 ? 4 : 2; }
static inline bool qg_type_ok(int type) { return type == QGBDT_F32 || type == QGBDT_BF16 || type == QGBDT_F16; }

// Widest vector (bytes, a power of two up to 16) that divides the address, the row stride and the row length.
static inline int qg_vec_bytes(const void *p, int64_t ld_bytes, int64_t len_bytes) {
    const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | (uintptr_t)ld_bytes | (uintptr_t)len_bytes | 16u;
    return (int)(bits & (~bits + 1));
}

// ---- argument checks ------------------------------------------------------------------------------

static inline bool qg_aligned(const void *p, int size) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)size == 0; }

// The row stride of a single row means nothing: one that suits the kernels, a multiple of `step` elements.
static inline void qg_single_row(int64_t rows, int64_t width, int step, int64_t *ld) {
    if (rows <= 1 && *ld >= width) *ld = (width + step - 1) / step * step;
}

// At the start and the end of a C entry: what an earlier kernel reported and the current device; the work buffer's use.
int qg_ops_enter(qgbdt_ctx *c);
int qg_ops_leave(qgbdt_ctx *c, int rc, void *stream);

// ---- launches ------------------------------------------------------------------------------------

// The operators' kernels are launched so that a kernel may start while the one before it on the stream ends:
// every one of them begins with qg_after_prior(), before which it touches no memory of the device.
__device__ __forceinline__ void qg_after_prior() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <typename... P, typename... A>
int qg_launch(qgbdt_ctx *c, void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, const A &...args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    QG_CUDA(c, cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
    c->n_launches++;
    return QGBDT_OK;
}
#define QG_RUN(expr)                        \
    do {                                    \
        const int rc_ = (expr);             \
        if (rc_ != QGBDT_OK) return rc_;    \
    } while (0)

// ---- workspace -----------------------------------------------------------------------------------

// A call's work memory: the context's one buffer, cut up from the front.  qg_ws_open makes the buffer
// at least `bytes` large and orders `st` after the last call that used it on another stream;
// qg_ws_close marks the end of this call's use (the C entries do that for calls that return an error in between).
struct QgWorkspace {
    char *at = nullptr, *end = nullptr;
    template <typename T>
    T *take(size_t count) {
        char *p = at;
        at += (count * sizeof(T) + 255) / 256 * 256;
        return reinterpret_cast<T *>(p);
    }
};
static inline size_t qg_ws_size(size_t count, size_t width) { return (count * width + 255) / 256 * 256; }

int qg_ws_open(qgbdt_ctx *c, size_t bytes, cudaStream_t st, QgWorkspace *ws);
int qg_ws_close(qgbdt_ctx *c, cudaStream_t st);

// ---- launchers (asynchronous on `st`, arguments already checked) -----------------------------------

struct EmbedArgs {
    const void *table;      // forward: [n_entries][ld]; backward: the gradient of the output, [rows][ld]
    int64_t ld;
    int64_t n_entries;
    int32_t dim;
    int32_t type;           // QGBDT_F32 / BF16 / F16
    const void *tokens;     // [rows][ld_tokens]
    int32_t token_type;     // QGBDT_I32 / I64
    int64_t rows, ld_tokens;
    int32_t bag;
    float scale;
    void *out;              // forward: [rows][ld_out]; backward: [n_entries][ld_out]
    int64_t ld_out;
    int32_t *status;
};
int qg_embed(qgbdt_ctx *c, const EmbedArgs &a, cudaStream_t st);
int qg_embed_backward(qgbdt_ctx *c, const EmbedArgs &a, cudaStream_t st);

struct SoftmaxArgs {
    const void *hidden, *weight;
    int32_t type;
    int64_t rows, ld_hidden, classes, ld_weight;
    int32_t dim;
    const float *bias;
    const void *labels;
    int32_t label_type;
    float *loss, *losses, *lse;             // forward outputs
    const float *grad_loss, *lse_in;        // backward inputs
    void *d_hidden, *d_weight;
    int64_t ld_d_hidden, ld_d_weight;
    float *d_bias;
    int32_t *status;
};
int qg_softmax_ce(qgbdt_ctx *c, const SoftmaxArgs &a, cudaStream_t st);
int qg_softmax_ce_backward(qgbdt_ctx *c, const SoftmaxArgs &a, cudaStream_t st);

int qg_clip_grad_norm(qgbdt_ctx *c, const void *const *in, void *const *out, const int64_t *counts, const int32_t *types,
                      int32_t n, double max_norm, float *d_norm, cudaStream_t st);

struct LayerNormArgs {
    const void *x, *grad;                   // grad: backward only
    int64_t ld_x, ld_grad;
    int32_t type, weight_type;
    const void *weight, *bias;              // NULL: 1, 0
    int64_t rows;
    int32_t dim;
    float eps;
    void *out;                              // backward: the gradient of x
    int64_t ld_out;
    float *mean, *rstd;                     // forward: NULL where not wanted; backward: read
    void *d_weight, *d_bias;
};
int qg_layer_norm(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st);
int qg_layer_norm_backward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st);

int qg_adamw(qgbdt_ctx *c, const qgbdt_adamw_tensor *t, int32_t n, const qgbdt_adamw_options &o, cudaStream_t st);
int qg_adamw_values(qgbdt_ctx *c, const uint8_t *const *m, const uint8_t *const *v, const uint8_t *const *exponents, void *const *out_m,
                    void *const *out_v, const int64_t *counts, int32_t n, int32_t type, cudaStream_t st);
