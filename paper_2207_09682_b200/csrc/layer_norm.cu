// Layer norm of rows, and its gradients.
//
//   mean = sum x / d,  rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),  out = (x - mean) rstd w + b
//   xh = (x - mean) rstd,  dx = rstd (w g - sum (w g) / d - xh sum (w g xh) / d),  dw = sum over rows of g xh,  db = sum over rows of g
//
// Sums and statistics are held in single precision; an output is rounded once, when it is written.
#include "ops_internal.cuh"

namespace {

// ---- rows of any length ----------------------------------------------------------------------------
// A block per row, which goes over the row once for each of its sums and once more to write (the later
// times from L1 or L2).

constexpr int LN_THREADS = 512;

// Sums of a and b over the block, the same in every thread, in a fixed order.  `at` alternates between two
// places of the shared memory, so that one barrier per sum is enough.
__device__ __forceinline__ float2 ln_block_sum(float2 s, float2 (&w)[2][32], int &at) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
        s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
    }
    if ((threadIdx.x & 31) == 0) w[at][threadIdx.x >> 5] = s;
    __syncthreads();
    s = make_float2(0.f, 0.f);
    for (int i = 0; i < (int)blockDim.x / 32; ++i) s.x += w[at][i].x, s.y += w[at][i].y;
    at ^= 1;
    return s;
}

template <typename T>
__device__ __forceinline__ float ln_weight(const void *w, bool f32, int col, float none) {
    if (!w) return none;
    return f32 ? reinterpret_cast<const float *>(w)[col] : OpsType<T>::load(reinterpret_cast<const T *>(w)[col]);
}

template <typename T, int V>
__global__ void __launch_bounds__(LN_THREADS) k_ln_long(const LayerNormArgs a) {
    qg_after_prior();
    __shared__ float2 w[2][32];
    int at = 0;
    const bool f32 = a.weight_type == QGBDT_F32;
    const float per = 1.f / (float)a.dim;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = reinterpret_cast<const T *>(a.x) + row * a.ld_x;
        T *out = reinterpret_cast<T *>(a.out) + row * a.ld_out;
        float2 s = make_float2(0.f, 0.f);
        for (int c = threadIdx.x * V; c < a.dim; c += LN_THREADS * V) {
            const OpsVec<T, V> v = *reinterpret_cast<const OpsVec<T, V> *>(x + c);
#pragma unroll
            for (int j = 0; j < V; ++j) s.x += OpsType<T>::load(v.v[j]);
        }
        const float mean = ln_block_sum(s, w, at).x * per;
        s = make_float2(0.f, 0.f);
        for (int c = threadIdx.x * V; c < a.dim; c += LN_THREADS * V) {
            const OpsVec<T, V> v = *reinterpret_cast<const OpsVec<T, V> *>(x + c);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float y = OpsType<T>::load(v.v[j]) - mean;
                s.x = fmaf(y, y, s.x);
            }
        }
        const float rstd = __frsqrt_rn(fmaf(ln_block_sum(s, w, at).x, per, a.eps));
        for (int c = threadIdx.x * V; c < a.dim; c += LN_THREADS * V) {
            OpsVec<T, V> v = *reinterpret_cast<const OpsVec<T, V> *>(x + c);
#pragma unroll
            for (int j = 0; j < V; ++j)
                v.v[j] = OpsType<T>::store(fmaf((OpsType<T>::load(v.v[j]) - mean) * rstd, ln_weight<T>(a.weight, f32, c + j, 1.f), ln_weight<T>(a.bias, f32, c + j, 0.f)));
            *reinterpret_cast<OpsVec<T, V> *>(out + c) = v;
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(LN_THREADS) k_ln_long_dx(const LayerNormArgs a) {
    qg_after_prior();
    __shared__ float2 w[2][32];
    int at = 0;
    const bool f32 = a.weight_type == QGBDT_F32;
    const float per = 1.f / (float)a.dim;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = reinterpret_cast<const T *>(a.x) + row * a.ld_x, *g = reinterpret_cast<const T *>(a.grad) + row * a.ld_grad;
        T *out = reinterpret_cast<T *>(a.out) + row * a.ld_out;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float2 s = make_float2(0.f, 0.f);
        for (int c = threadIdx.x * V; c < a.dim; c += LN_THREADS * V) {
            const OpsVec<T, V> v = *reinterpret_cast<const OpsVec<T, V> *>(x + c), u = *reinterpret_cast<const OpsVec<T, V> *>(g + c);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float y = OpsType<T>::load(u.v[j]) * ln_weight<T>(a.weight, f32, c + j, 1.f);
                s.x += y;
                s.y = fmaf(y, (OpsType<T>::load(v.v[j]) - mean) * rstd, s.y);
            }
        }
        s = ln_block_sum(s, w, at);
        const float c1 = s.x * per, c2 = s.y * per;
        for (int c = threadIdx.x * V; c < a.dim; c += LN_THREADS * V) {
            const OpsVec<T, V> v = *reinterpret_cast<const OpsVec<T, V> *>(x + c);
            OpsVec<T, V> u = *reinterpret_cast<const OpsVec<T, V> *>(g + c);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float y = OpsType<T>::load(u.v[j]) * ln_weight<T>(a.weight, f32, c + j, 1.f), xh = (OpsType<T>::load(v.v[j]) - mean) * rstd;
                u.v[j] = OpsType<T>::store((y - c1 - xh * c2) * rstd);
            }
            *reinterpret_cast<OpsVec<T, V> *>(out + c) = u;
        }
    }
}

// Sums over a slice of the rows, 32 columns per block: partial [slices][2][dim] (of the weight's gradient, of the bias's).
constexpr int LN_COLUMN_ROWS = 16;   // rows side by side

template <typename T>
__global__ void __launch_bounds__(32 * LN_COLUMN_ROWS) k_ln_columns(const LayerNormArgs a, float *partial) {
    qg_after_prior();
    __shared__ float2 w[LN_COLUMN_ROWS][32];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    const int64_t r0 = a.rows * blockIdx.y / gridDim.y, r1 = a.rows * (blockIdx.y + 1) / gridDim.y;
    float2 s = make_float2(0.f, 0.f);
    if (c < a.dim) {
#pragma unroll 4
        for (int64_t r = r0 + part; r < r1; r += LN_COLUMN_ROWS) {
            const float g = OpsType<T>::load(reinterpret_cast<const T *>(a.grad)[r * a.ld_grad + c]);
            const float x = OpsType<T>::load(reinterpret_cast<const T *>(a.x)[r * a.ld_x + c]);
            s.x = fmaf(g, (x - a.mean[r]) * a.rstd[r], s.x);
            s.y += g;
        }
    }
    w[part][lane] = s;
    __syncthreads();
    if (part == 0 && c < a.dim) {
        s = w[0][lane];
        for (int i = 1; i < LN_COLUMN_ROWS; ++i) s.x += w[i][lane].x, s.y += w[i][lane].y;
        float *p = partial + (int64_t)blockIdx.y * 2 * a.dim + c;
        p[0] = s.x;
        p[a.dim] = s.y;
    }
}

// The partial sums joined in their order: 32 columns per block, LN_JOIN parts of the slices side by side.
constexpr int LN_JOIN = 32;

template <typename T>
__global__ void __launch_bounds__(32 * LN_JOIN) k_ln_join(const LayerNormArgs a, const float *partial, int slices) {
    qg_after_prior();
    __shared__ float w[LN_JOIN][33];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    void *out = blockIdx.y ? a.d_bias : a.d_weight;
    if (!out) return;
    float s = 0.f;
    if (c < a.dim) {
        const float *p = partial + blockIdx.y * (int64_t)a.dim + c;
#pragma unroll 8
        for (int i = part; i < slices; i += LN_JOIN) s += p[(int64_t)i * 2 * a.dim];
    }
    w[part][lane] = s;
    __syncthreads();
    if (part == 0 && c < a.dim) {
        for (int i = 1; i < LN_JOIN; ++i) s += w[i][lane];
        if (a.weight_type == QGBDT_F32) reinterpret_cast<float *>(out)[c] = s;
        else reinterpret_cast<T *>(out)[c] = OpsType<T>::store(s);
    }
}

// ---- launches --------------------------------------------------------------------------------------

// Whether rows allow vectors of 16 bytes throughout.
bool wide(const void *p, int64_t ld, const LayerNormArgs &a) {
    const int w = qg_type_size(a.type);
    return !p || qg_vec_bytes(p, ld * w, (int64_t)a.dim * w) == 16;
}

template <typename T>
int forward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const int64_t most = (int64_t)c->sm_count * 4;
    const dim3 grid((unsigned)(a.rows < most ? a.rows : most));
    if (wide(a.x, a.ld_x, a) && wide(a.out, a.ld_out, a)) return qg_launch(c, k_ln_long<T, V>, grid, LN_THREADS, 0, st, a);
    return qg_launch(c, k_ln_long<T, 1>, grid, LN_THREADS, 0, st, a);
}

template <typename T>
int backward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    if (a.d_weight || a.d_bias) {
        // before the rows' gradients, which may take the place of an input
        const int tiles = (a.dim + 31) / 32;
        int64_t slices = (a.rows + LN_COLUMN_ROWS * 8 - 1) / (LN_COLUMN_ROWS * 8);
        const int64_t most = ((int64_t)c->sm_count * 8 + tiles - 1) / tiles;
        if (slices > most) slices = most;
        if (slices < 1) slices = 1;
        QgWorkspace ws;
        QG_RUN(qg_ws_open(c, qg_ws_size((size_t)slices * 2 * a.dim, sizeof(float)), st, &ws));
        float *partial = ws.take<float>((size_t)slices * 2 * a.dim);
        QG_RUN(qg_launch(c, k_ln_columns<T>, dim3(tiles, (unsigned)slices), 32 * LN_COLUMN_ROWS, 0, st, a, partial));
        QG_RUN(qg_launch(c, k_ln_join<T>, dim3(tiles, 2), 32 * LN_JOIN, 0, st, a, partial, (int)slices));
        QG_RUN(qg_ws_close(c, st));
    }
    if (a.rows == 0) return QGBDT_OK;
    const int64_t most = (int64_t)c->sm_count * 4;
    const dim3 grid((unsigned)(a.rows < most ? a.rows : most));
    if (wide(a.x, a.ld_x, a) && wide(a.grad, a.ld_grad, a) && wide(a.out, a.ld_out, a)) return qg_launch(c, k_ln_long_dx<T, V>, grid, LN_THREADS, 0, st, a);
    return qg_launch(c, k_ln_long_dx<T, 1>, grid, LN_THREADS, 0, st, a);
}

}  // namespace

int qg_layer_norm(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    if (a.type == QGBDT_F32) return forward<float>(c, a, st);
    if (a.type == QGBDT_BF16) return forward<__nv_bfloat16>(c, a, st);
    return forward<__half>(c, a, st);
}

int qg_layer_norm_backward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    if (a.type == QGBDT_F32) return backward<float>(c, a, st);
    if (a.type == QGBDT_BF16) return backward<__nv_bfloat16>(c, a, st);
    return backward<__half>(c, a, st);
}
