// Global gradient norm over many tensors, and clipping.
//
//   norm = sqrt(sum over tensors and elements of g^2),   out = g * min(1, max_norm / norm)
//
// Two launches (one for up to 32 chunks): the first takes the sum of squares (one double per block; the block that ends last adds
// the blocks' sums in their order and works out the factor), the second multiplies.  Bound by memory
// traffic: every tensor is read once, and read and written once more when the norm is above max_norm.
// 300 tensors, 1.07 GB, above max_norm: norm 0.17 ms (6.3 TB/s), scaling 0.32 ms (6.6 TB/s; what the first launch read is
// gone from L2 by then).  Six small tensors: one launch, 3 us.
//
// A tensor is cut into chunks of 4096 elements counted from its first 16-byte boundary (the elements
// before it ride with the first chunk).  A block finds its first chunk's tensor by a binary search over
// the tensors' first chunk numbers, which lie with the pointers in the kernel's parameters, and walks on
// from there.  The first launch has blocks that stay, each with a run of neighbouring chunks (few sums to
// add); the second has one block per CLIP_STEP chunks, so that the memory sees one moving front of reads
// and writes instead of hundreds.
//
// Squares are added in double precision: single precision would overflow from |g| = 1.8e19 on and lose
// everything below 1e-23, and the double-precision units have the throughput to spare here.  The tensors are multiplied in
// single precision, unless the factor is below its normal range (a norm above 8.5e37 times max_norm): it would lose bits
// there, and the products are taken in double precision.
#include "ops_internal.cuh"

namespace {

constexpr int CLIP_THREADS = 256;
constexpr int CLIP_CHUNK = 4096;
constexpr int CLIP_BLOCKS = 6;   // of the first launch, per SM
constexpr int CLIP_STEP = 2;     // chunks per block of the second launch
constexpr int CLIP_SMALL = 64, CLIP_LARGE = 1000;   // tensors per launch (parameters of 1.3 or 20 KB, with the outputs 1.8 or 28)

template <int CAP>
struct ClipTable {
    const void *in[CAP];
    long long count[CAP];      // elements | type << 56
    int first[CAP];            // first chunk
    int n, chunks;
};
template <int CAP>
struct ClipOut {
    void *out[CAP];
};

template <int CAP>
__device__ __forceinline__ int find_tensor(const ClipTable<CAP> &t, int chunk) {
    int lo = 0, hi = t.n;   // t.first[lo] <= chunk < t.first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Elements of a chunk: a scalar head (first chunk only), then [begin, end) from a 16-byte boundary.
struct ChunkRange {
    long long begin, end;
    int head;
};

__device__ __forceinline__ ChunkRange chunk_range(const void *p, int width, long long count, int k) {
    ChunkRange r;
    const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15);
    long long peel = off ? (16 - off) / width : 0;
    if (peel > count) peel = count;
    r.head = k == 0 ? (int)peel : 0;
    r.begin = peel + (long long)k * CLIP_CHUNK;
    r.end = r.begin + CLIP_CHUNK;
    if (r.end > count) r.end = count;
    if (r.begin > count) r.begin = count;
    return r;
}

template <typename T>
__device__ __forceinline__ double sum_squares(const T *p, const ChunkRange &r) {
    constexpr int V = 16 / sizeof(T);
    double s = 0.0;
    if ((int)threadIdx.x < r.head) {
        const double x = (double)OpsType<T>::load(p[threadIdx.x]);
        s = fma(x, x, s);
    }
    const int n = (int)(r.end - r.begin), nv = n / V;
    const OpsVec<T, V> *q = reinterpret_cast<const OpsVec<T, V> *>(p + r.begin);
    if (nv == CLIP_CHUNK / V) {
        OpsVec<T, V> x[CLIP_CHUNK / V / CLIP_THREADS];
#pragma unroll
        for (int i = 0; i < CLIP_CHUNK / V / CLIP_THREADS; ++i) x[i] = q[threadIdx.x + i * CLIP_THREADS];
#pragma unroll
        for (int i = 0; i < CLIP_CHUNK / V / CLIP_THREADS; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const double y = (double)OpsType<T>::load(x[i].v[j]);
                s = fma(y, y, s);
            }
    } else {
        for (int i = threadIdx.x; i < nv; i += CLIP_THREADS) {
            const OpsVec<T, V> x = q[i];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const double y = (double)OpsType<T>::load(x.v[j]);
                s = fma(y, y, s);
            }
        }
        for (int i = nv * V + threadIdx.x; i < n; i += CLIP_THREADS) {
            const double y = (double)OpsType<T>::load(p[r.begin + i]);
            s = fma(y, y, s);
        }
    }
    return s;
}

// Sum over the block, the same in every thread; a fixed tree.
__device__ __forceinline__ double block_sum(double s) {
    __shared__ double w[CLIP_THREADS / 32];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) w[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int i = 0; i < CLIP_THREADS / 32; ++i) s += w[i];
    __syncthreads();
    return s;
}

// What the second launch reads.
struct ClipFactor {
    double exact;
    float coef;     // the same in single precision
    int scale;      // 0: the tensors keep their values; 1: times coef; 2: times exact
};

// From the sum of squares; the norm goes to *d_norm (unless NULL).
__device__ __forceinline__ ClipFactor factor_of(double s, double max_norm, float *d_norm) {
    const double norm = sqrt(s);
    if (d_norm) *d_norm = (float)norm;
    // false also for a norm that is not finite: the tensors keep their values then
    const bool clip = norm > max_norm && norm <= 1.7976931348623157e308;
    const double exact = clip ? max_norm / norm : 1.0;
    return ClipFactor{exact, (float)exact, !clip ? 0 : exact < 1.17549435082228751e-38 ? 2 : 1};
}

// n_before: sums of earlier launches of the same call; the last launch (`final`) adds them all.
template <int CAP>
__global__ void __launch_bounds__(CLIP_THREADS, CLIP_BLOCKS) k_norm_partial(const __grid_constant__ ClipTable<CAP> t, double *partial, int n_before,
                                                                            bool final, double max_norm, unsigned *arrived, ClipFactor *factor,
                                                                            float *d_norm) {
    qg_after_prior();
    __shared__ bool last;
    double s = 0.0;
    const int c0 = (int)((long long)t.chunks * blockIdx.x / gridDim.x), c1 = (int)((long long)t.chunks * (blockIdx.x + 1) / gridDim.x);
    int i = c0 < c1 ? find_tensor(t, c0) : 0;
    for (int c = c0; c < c1; ++c) {
        while (i + 1 < t.n && t.first[i + 1] <= c) ++i;
        const long long count = t.count[i] & ((1ll << 56) - 1);
        const int type = (int)(t.count[i] >> 56), k = c - t.first[i];
        const void *p = t.in[i];
        const ChunkRange r = chunk_range(p, type == QGBDT_F32 ? 4 : 2, count, k);
        if (type == QGBDT_F32) s += sum_squares(reinterpret_cast<const float *>(p), r);
        else if (type == QGBDT_BF16) s += sum_squares(reinterpret_cast<const __nv_bfloat16 *>(p), r);
        else s += sum_squares(reinterpret_cast<const __half *>(p), r);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) {
        partial[n_before + blockIdx.x] = s;
        __threadfence();
        last = final && atomicAdd(arrived, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    s = 0.0;
    for (int k = threadIdx.x; k < n_before + (int)gridDim.x; k += CLIP_THREADS) s += *(volatile double *)&partial[k];
    s = block_sum(s);
    if (threadIdx.x == 0) {
        *factor = factor_of(s, max_norm, d_norm);
        *arrived = 0;
    }
}

template <typename T, typename F>
__device__ __forceinline__ void scale_chunk(const T *p, T *o, const ChunkRange &r, F coef) {   // F: precision of the products
    constexpr int V = 16 / sizeof(T);
    auto scaled = [coef](T x) { return OpsType<T>::store((float)((F)OpsType<T>::load(x) * coef)); };
    if ((int)threadIdx.x < r.head) o[threadIdx.x] = scaled(p[threadIdx.x]);
    const int n = (int)(r.end - r.begin);
    const bool vec = (reinterpret_cast<uintptr_t>(o + r.begin) & 15) == 0;   // the output may be aligned differently
    const int nv = vec ? n / V : 0;
    const OpsVec<T, V> *q = reinterpret_cast<const OpsVec<T, V> *>(p + r.begin);
    OpsVec<T, V> *w = reinterpret_cast<OpsVec<T, V> *>(o + r.begin);
    if (nv == CLIP_CHUNK / V) {
        OpsVec<T, V> x[CLIP_CHUNK / V / CLIP_THREADS];
#pragma unroll
        for (int i = 0; i < CLIP_CHUNK / V / CLIP_THREADS; ++i) x[i] = q[threadIdx.x + i * CLIP_THREADS];
#pragma unroll
        for (int i = 0; i < CLIP_CHUNK / V / CLIP_THREADS; ++i) {
#pragma unroll
            for (int j = 0; j < V; ++j) x[i].v[j] = scaled(x[i].v[j]);
            w[threadIdx.x + i * CLIP_THREADS] = x[i];
        }
    } else {
        for (int i = threadIdx.x; i < nv; i += CLIP_THREADS) {
            OpsVec<T, V> x = q[i];
#pragma unroll
            for (int j = 0; j < V; ++j) x.v[j] = scaled(x.v[j]);
            w[i] = x;
        }
        for (int i = nv * V + threadIdx.x; i < n; i += CLIP_THREADS)
            o[r.begin + i] = scaled(p[r.begin + i]);
    }
}
template <typename F>
__device__ __forceinline__ void scale_any(const void *p, void *o, int type, const ChunkRange &r, F coef) {
    if (type == QGBDT_F32) scale_chunk(reinterpret_cast<const float *>(p), reinterpret_cast<float *>(o), r, coef);
    else if (type == QGBDT_BF16) scale_chunk(reinterpret_cast<const __nv_bfloat16 *>(p), reinterpret_cast<__nv_bfloat16 *>(o), r, coef);
    else scale_chunk(reinterpret_cast<const __half *>(p), reinterpret_cast<__half *>(o), r, coef);
}

template <int CAP>
__global__ void __launch_bounds__(CLIP_THREADS) k_clip_scale(const __grid_constant__ ClipTable<CAP> t, const __grid_constant__ ClipOut<CAP> o,
                                                             const ClipFactor *factor, bool in_place) {
    qg_after_prior();
    const ClipFactor f = *factor;
    if (!f.scale && in_place) return;
    const int c0 = blockIdx.x * CLIP_STEP, c1 = min(t.chunks, c0 + CLIP_STEP);
    int i = find_tensor(t, c0);
    for (int c = c0; c < c1; ++c) {
        while (i + 1 < t.n && t.first[i + 1] <= c) ++i;
        const long long count = t.count[i] & ((1ll << 56) - 1);
        const int type = (int)(t.count[i] >> 56), k = c - t.first[i];
        const void *p = t.in[i];
        void *w = o.out[i];
        const ChunkRange r = chunk_range(p, type == QGBDT_F32 ? 4 : 2, count, k);
        if (f.scale == 2) scale_any(p, w, type, r, f.exact);
        else scale_any(p, w, type, r, f.coef);
    }
}

// Few chunks: one launch.  A cluster of eight blocks, each with every eighth chunk; the blocks' sums are exchanged
// through the cluster's shared memory.
constexpr int CLIP_CLUSTER = 8, CLIP_FEW_CHUNKS = 32;

__global__ void __cluster_dims__(CLIP_CLUSTER) __launch_bounds__(CLIP_THREADS)
    k_clip_few(const __grid_constant__ ClipTable<CLIP_SMALL> t, const __grid_constant__ ClipOut<CLIP_SMALL> o, double max_norm, bool in_place,
               float *d_norm) {
    qg_after_prior();
    __shared__ double mine;
    double s = 0.0;
    for (int c = blockIdx.x; c < t.chunks; c += CLIP_CLUSTER) {
        const int i = find_tensor(t, c);
        const long long count = t.count[i] & ((1ll << 56) - 1);
        const int type = (int)(t.count[i] >> 56);
        const ChunkRange r = chunk_range(t.in[i], type == QGBDT_F32 ? 4 : 2, count, c - t.first[i]);
        if (type == QGBDT_F32) s += sum_squares(reinterpret_cast<const float *>(t.in[i]), r);
        else if (type == QGBDT_BF16) s += sum_squares(reinterpret_cast<const __nv_bfloat16 *>(t.in[i]), r);
        else s += sum_squares(reinterpret_cast<const __half *>(t.in[i]), r);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) mine = s;
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    s = 0.0;
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(&mine);
#pragma unroll
    for (uint32_t k = 0; k < CLIP_CLUSTER; ++k) {
        double x;
        asm volatile("{\n.reg .b32 a;\nmapa.shared::cluster.u32 a, %1, %2;\nld.shared::cluster.f64 %0, [a];\n}" : "=d"(x) : "r"(at), "r"(k) : "memory");
        s += x;
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");   // before any block ends
    const ClipFactor f = factor_of(s, max_norm, blockIdx.x == 0 && threadIdx.x == 0 ? d_norm : nullptr);
    if (!f.scale && in_place) return;
    for (int c = blockIdx.x; c < t.chunks; c += CLIP_CLUSTER) {
        const int i = find_tensor(t, c);
        const long long count = t.count[i] & ((1ll << 56) - 1);
        const int type = (int)(t.count[i] >> 56);
        const ChunkRange r = chunk_range(t.in[i], type == QGBDT_F32 ? 4 : 2, count, c - t.first[i]);
        if (f.scale == 2) scale_any(t.in[i], o.out[i], type, r, f.exact);
        else scale_any(t.in[i], o.out[i], type, r, f.coef);
    }
}

template <int CAP>
int fill(ClipTable<CAP> &t, ClipOut<CAP> &o, const void *const *in, void *const *out, const int64_t *counts, const int32_t *types, int32_t &at,
         int32_t n) {
    t.n = 0;
    long long chunks = 0;
    for (; at < n && t.n < CAP; ++at) {
        if (counts[at] == 0) continue;
        // one chunk even for a tensor that ends before its first 16-byte boundary
        const int width = qg_type_size(types[at]), off = (int)(reinterpret_cast<uintptr_t>(in[at]) & 15);
        const long long body = counts[at] - (off ? (16 - off) / width : 0);
        const long long k = body > 0 ? (body + CLIP_CHUNK - 1) / CLIP_CHUNK : 1;
        if (t.n > 0 && chunks + k > 0x40000000ll) break;
        if (k > 0x40000000ll) return -1;
        t.in[t.n] = in[at];
        o.out[t.n] = out[at];
        t.count[t.n] = counts[at] | (long long)types[at] << 56;
        t.first[t.n] = (int)chunks;
        chunks += k;
        ++t.n;
    }
    t.chunks = (int)chunks;
    return 0;
}

int norm_grid(const qgbdt_ctx *c, int chunks) {
    const int full = c->sm_count * CLIP_BLOCKS;
    return chunks < full ? (chunks > 0 ? chunks : 1) : full;
}

template <int CAP>
int clip_groups(qgbdt_ctx *c, const void *const *in, void *const *out, const int64_t *counts, const int32_t *types, int32_t n, double max_norm,
                float *d_norm, double *partial, cudaStream_t st) {
    ClipTable<CAP> t;
    ClipOut<CAP> o;
    bool in_place = true;
    for (int32_t i = 0; i < n; ++i) in_place = in_place && (in[i] == out[i] || counts[i] == 0);
    if constexpr (CAP == CLIP_SMALL) {
        int32_t at = 0;
        if (fill(t, o, in, out, counts, types, at, n) != 0) return qg_fail(c, QGBDT_ERR_ARG, "a tensor is too large");
        if (at >= n && t.chunks <= CLIP_FEW_CHUNKS) return qg_launch(c, k_clip_few, dim3(CLIP_CLUSTER), CLIP_THREADS, 0, st, t, o, max_norm, in_place, d_norm);
    }
    ClipFactor *factor = reinterpret_cast<ClipFactor *>(partial);   // in front of the sums
    partial += 16;
    int n_partial = 0;
    int32_t at = 0;
    do {
        if (fill(t, o, in, out, counts, types, at, n) != 0) return qg_fail(c, QGBDT_ERR_ARG, "a tensor is too large");
        const int grid = norm_grid(c, t.chunks);
        QG_RUN(qg_launch(c, k_norm_partial<CAP>, dim3(grid), CLIP_THREADS, 0, st, t, partial, n_partial, at >= n, max_norm, c->d_ops_counters + 1, factor,
                         d_norm));
        n_partial += grid;
    } while (at < n);
    if (in_place && max_norm > 1.7976931348623157e308) return QGBDT_OK;   // the norm alone
    at = 0;
    do {
        if (t.n == n) at = n;   // a single group: still in t
        else fill(t, o, in, out, counts, types, at, n);
        if (t.chunks > 0)
            QG_RUN(qg_launch(c, k_clip_scale<CAP>, dim3((t.chunks + CLIP_STEP - 1) / CLIP_STEP), CLIP_THREADS, 0, st, t, o, factor, in_place));
    } while (at < n);
    return QGBDT_OK;
}

}  // namespace

int qg_clip_grad_norm(qgbdt_ctx *c, const void *const *in, void *const *out, const int64_t *counts, const int32_t *types, int32_t n,
                      double max_norm, float *d_norm, cudaStream_t st) {
    QgWorkspace ws;
    const size_t groups = (size_t)n / CLIP_SMALL + 2;
    int rc = qg_ws_open(c, qg_ws_size(groups * c->sm_count * CLIP_BLOCKS + 16, sizeof(double)), st, &ws);
    if (rc != QGBDT_OK) return rc;
    double *partial = ws.take<double>(groups * c->sm_count * CLIP_BLOCKS + 16);
    rc = n <= CLIP_SMALL ? clip_groups<CLIP_SMALL>(c, in, out, counts, types, n, max_norm, d_norm, partial, st)
                         : clip_groups<CLIP_LARGE>(c, in, out, counts, types, n, max_norm, d_norm, partial, st);
    if (rc != QGBDT_OK) return rc;
    return qg_ws_close(c, st);
}
