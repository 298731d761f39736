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

// ---- rows that fit in registers ---------------------------------------------------------------------
// `lanes` threads have a row: a power of two up to 32, or whole warps; thread g has the vectors g, g + lanes, ... of V
// elements, N of them.  What belongs to the columns stays in registers over all rows of the group, and the next row is
// loaded under this one's work.

// Elements of a row per thread and threads of a row, at most; narrow vectors take more registers each.
template <int V>
constexpr int LN_EACH = V <= 2 ? 8 : 16;
template <int V>
constexpr int LN_MOST = V <= 2 ? 1024 : 512;
constexpr int LN_ROW = 8192;     // the product of the two

__device__ __forceinline__ float ln_lanes_sum(float s, int lanes) {   // a power of two of neighbouring lanes
#pragma unroll
    for (int o = 16; o; o >>= 1)
        if (o < lanes) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// What each warp of a row (lanes / 32 of them) has to give, handed round: lane i gets warp i's.  `at` alternates between two places
// of the shared memory, so that one barrier is enough; `barrier` is the row's own.
__device__ __forceinline__ float2 ln_exchange(float2 mine, int lanes, float2 (&part)[2][32], int &at, int barrier) {
    const int first = threadIdx.x / lanes * (lanes / 32), lane = threadIdx.x & 31;
    if (lane == 0) part[at][threadIdx.x / 32] = mine;
    asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(lanes) : "memory");
    const float2 other = lane < lanes / 32 ? part[at][first + lane] : make_float2(0.f, 0.f);
    at ^= 1;
    return other;
}

// Lanes that `warps` warps' sums are in, as a power of two.
__device__ __forceinline__ int ln_power(int warps) { return warps <= 1 ? 1 : 2 << (31 - __clz(warps - 1)); }

// A thread's vectors of the coming rows: copied asynchronously to places of the shared memory that are the thread's own, DEPTH rows
// ahead (so that nobody waits for another thread's copies; 64 KB and more on their way per SM, which is what the memory's latency under
// load takes).  Vectors of 2 bytes, which such copies do not come in, are kept in registers, one row ahead.
template <typename T, int V, int N, int DEPTH>
struct LnRows {
    static constexpr bool RING = sizeof(T) * V >= 4;
    using Vec = OpsVec<T, V>;
    static constexpr size_t bytes(int threads) { return RING ? sizeof(Vec) * N * DEPTH * threads : 0; }
    Vec v[N];      // the row's
    Vec next[RING ? 1 : N];
    __device__ __forceinline__ void fetch(Vec *ring, int slot, const void *p, int64_t at, int dim, int g, int lanes) {
        const T *q = reinterpret_cast<const T *>(p) + at;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = (g + i * lanes) * V;
            if (c >= dim) continue;
            if constexpr (RING) {
                const uint32_t to = (uint32_t)__cvta_generic_to_shared(ring + (slot * N + i) * blockDim.x + threadIdx.x);
                if constexpr (sizeof(Vec) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(q + c) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(q + c), "n"(sizeof(Vec)) : "memory");
            } else {
                next[i] = *reinterpret_cast<const Vec *>(q + c);
            }
        }
    }
    __device__ __forceinline__ void take(const Vec *ring, int slot) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (RING) v[i] = ring[(slot * N + i) * blockDim.x + threadIdx.x];
            else v[i] = next[i];
        }
    }
    __device__ __forceinline__ float get(int i) const { return OpsType<T>::load(v[i / V].v[i % V]); }
    __device__ __forceinline__ void set(int i, float x) { v[i / V].v[i % V] = OpsType<T>::store(x); }
    __device__ __forceinline__ void store(void *p, int64_t at, int dim, int g, int lanes) const {
        T *q = reinterpret_cast<T *>(p) + at;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = (g + i * lanes) * V;
            if (c < dim) *reinterpret_cast<Vec *>(q + c) = v[i];
        }
    }
};
__device__ __forceinline__ void ln_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void ln_arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }   // all but the last LEFT

constexpr int LN_AHEAD = 4, LN_AHEAD_BACKWARD = 3;   // rows

// Mean and sum of squared differences from it: over a warp in two passes; the warps' are joined by
//   sum over warps of M2 + count (mean of the warp - mean)^2,
// which takes one exchange and loses nothing where the mean is large beside the differences.
template <typename T, int V, int N, bool MULTI>
__global__ void __launch_bounds__(MULTI ? LN_MOST<V> : 128) k_ln_rows(const LayerNormArgs a, int lanes) {
    qg_after_prior();
    extern __shared__ __align__(16) unsigned char shared_bytes[];
    using Rows = LnRows<T, V, N, LN_AHEAD>;
    constexpr int AHEAD = Rows::RING ? LN_AHEAD : 1;
    typename Rows::Vec *const ring = reinterpret_cast<typename Rows::Vec *>(shared_bytes);
    __shared__ float2 part[2][32];
    constexpr int E = N * V;
    const int groups = MULTI ? 1 : blockDim.x / lanes, group = MULTI ? 0 : threadIdx.x / lanes, g = MULTI ? threadIdx.x : threadIdx.x & (lanes - 1);
    const int64_t stride = (int64_t)gridDim.x * groups;
    const float per = 1.f / (float)a.dim;
    const bool f32 = a.weight_type == QGBDT_F32;
    // elements of a row that a warp has: this one, and the one with this lane's number
    auto elements = [&](int warp) {
        int n = 0;
        for (int i = 0; i < N; ++i) n += max(0, min(32, a.dim / V - warp * 32 - i * lanes)) * V;
        return (float)n;
    };
    const float count = MULTI && (int)(threadIdx.x & 31) < lanes / 32 ? elements(threadIdx.x & 31) : 0.f, warp_count = MULTI ? elements(threadIdx.x / 32) : (float)a.dim;
    const float warp_per = warp_count > 0.f ? 1.f / warp_count : 0.f;
    const int warps = ln_power(lanes / 32);
    int at = 0;
    int64_t row = (int64_t)blockIdx.x * groups + group;
    Rows x;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
        if (row + k * stride < a.rows) x.fetch(ring, k, a.x, (row + k * stride) * a.ld_x, a.dim, g, lanes);
        ln_commit();
    }
    int slot = 0;
    float w[E], b[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int c = (g + i / V * lanes) * V + i % V;
        w[i] = c < a.dim ? ln_weight<T>(a.weight, f32, c, 1.f) : 0.f;
        b[i] = c < a.dim ? ln_weight<T>(a.bias, f32, c, 0.f) : 0.f;
    }
    for (int64_t base = row - group; base < a.rows; base += stride, row += stride) {
        ln_arrived<AHEAD - 1>();
        x.take(ring, slot);
        float y[E], s = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            y[i] = (g + i / V * lanes) * V < a.dim ? x.get(i) : 0.f;
            s += y[i];
        }
        if (row + AHEAD * stride < a.rows) x.fetch(ring, slot, a.x, (row + AHEAD * stride) * a.ld_x, a.dim, g, lanes);
        ln_commit();
        slot = slot + 1 < AHEAD ? slot + 1 : 0;
        float mean = ln_lanes_sum(s, MULTI ? 32 : lanes) * warp_per;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float z = (g + i / V * lanes) * V < a.dim ? y[i] - mean : 0.f;
            s = fmaf(z, z, s);
        }
        s = ln_lanes_sum(s, MULTI ? 32 : lanes);
        if constexpr (MULTI) {
            const float2 other = ln_exchange(make_float2(mean, s), lanes, part, at, 1);
            mean = ln_lanes_sum(other.x * count, warps) * per;
            const float z = other.x - mean;
            s = ln_lanes_sum(fmaf(z * count, z, other.y), warps);
            if (warps < 32) mean = __shfl_sync(0xffffffffu, mean, 0), s = __shfl_sync(0xffffffffu, s, 0);
        }
        const float rstd = __frsqrt_rn(fmaf(s, per, a.eps));
        if (row >= a.rows) continue;
        Rows out;
#pragma unroll
        for (int i = 0; i < E; ++i) out.set(i, fmaf((y[i] - mean) * rstd, w[i], b[i]));
        out.store(a.out, row * a.ld_out, a.dim, g, lanes);
        if (g == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// The gradients; the sums over the rows are gathered by column in registers, joined in shared memory over the block's groups and
// written as the block's part of partial [blocks][2][dim], or, from a single block, as they are.
template <typename T, int V, int N, bool MULTI>
__global__ void __launch_bounds__(MULTI ? LN_MOST<V> : 256) k_ln_rows_backward(const LayerNormArgs a, float *partial, int lanes) {
    qg_after_prior();
    extern __shared__ __align__(16) unsigned char shared_bytes[];
    using Rows = LnRows<T, V, N, LN_AHEAD_BACKWARD>;
    constexpr int AHEAD = Rows::RING ? LN_AHEAD_BACKWARD : 1;
    // weight [dim]; the coming rows of x and of the gradient, afterwards the columns' sums [N * V][threads]
    float *const weight = reinterpret_cast<float *>(shared_bytes), *const joined = weight + (a.dim + 3) / 4 * 4;
    typename Rows::Vec *const ring_x = reinterpret_cast<typename Rows::Vec *>(joined), *const ring_u = ring_x + N * AHEAD * blockDim.x;
    __shared__ float2 part[2][32];
    constexpr int E = N * V;
    const int groups = blockDim.x / lanes, group = threadIdx.x / lanes, g = threadIdx.x - group * lanes;
    const int64_t stride = (int64_t)gridDim.x * groups;
    const float per = 1.f / (float)a.dim;
    const bool f32 = a.weight_type == QGBDT_F32;
    const int warps = ln_power(lanes / 32);
    int at = 0, slot = 0;
    int64_t row = (int64_t)blockIdx.x * groups + group;
    Rows x, u;
    auto fetch = [&](int to, int64_t r) {
        if (r < a.rows) {
            x.fetch(ring_x, to, a.x, r * a.ld_x, a.dim, g, lanes);
            u.fetch(ring_u, to, a.grad, r * a.ld_grad, a.dim, g, lanes);
        }
        ln_commit();
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) fetch(k, row + k * stride);
    // mean and rstd: a lane has those of one of the group's next `turns` rows, and of as many after those
    const int turns = lanes < 32 ? lanes : 32, mine = threadIdx.x & (turns - 1);
    float2 stats, later = make_float2(0.f, 0.f);
    auto statistics = [&](int64_t r) { return r < a.rows ? make_float2(a.mean[r], a.rstd[r]) : make_float2(0.f, 0.f); };
    stats = statistics(row + mine * stride);
    int turn = 0;
    for (int c = threadIdx.x; c < a.dim; c += blockDim.x) weight[c] = ln_weight<T>(a.weight, f32, c, 1.f);
    __syncthreads();
    float dw[E] = {}, db[E] = {};
    for (int64_t base = row - group; base < a.rows; base += stride, row += stride) {
        if (turn == 0) later = statistics(row + (mine + turns) * stride);
        const float mean = __shfl_sync(0xffffffffu, stats.x, turn, turns), r = __shfl_sync(0xffffffffu, stats.y, turn, turns);
        if (++turn == turns) turn = 0, stats = later;
        ln_arrived<AHEAD - 1>();
        x.take(ring_x, slot);
        u.take(ring_u, slot);
        float xh[E], y[E];
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int c = (g + k * lanes) * V;
            const bool in = c < a.dim && row < a.rows;
            OpsVec<float, V> w = {};
            if (in) w = *reinterpret_cast<const OpsVec<float, V> *>(weight + c);
#pragma unroll
            for (int i = k * V; i < (k + 1) * V; ++i) {
                xh[i] = in ? (x.get(i) - mean) * r : 0.f;
                const float v = in ? u.get(i) : 0.f;
                db[i] += v;
                dw[i] = fmaf(v, xh[i], dw[i]);
                y[i] = v * w.v[i % V];
                s.x += y[i];
                s.y = fmaf(y[i], xh[i], s.y);
            }
        }
        fetch(slot, row + AHEAD * stride);
        slot = slot + 1 < AHEAD ? slot + 1 : 0;
        s.x = ln_lanes_sum(s.x, MULTI ? 32 : lanes), s.y = ln_lanes_sum(s.y, MULTI ? 32 : lanes);
        if constexpr (MULTI) {
            s = ln_exchange(s, lanes, part, at, 1 + group);
            s.x = __shfl_sync(0xffffffffu, ln_lanes_sum(s.x, warps), 0), s.y = __shfl_sync(0xffffffffu, ln_lanes_sum(s.y, warps), 0);
        }
        if (row >= a.rows) continue;
        const float c1 = s.x * per, c2 = s.y * per;
        Rows out;
#pragma unroll
        for (int i = 0; i < E; ++i) out.set(i, (y[i] - c1 - xh[i] * c2) * r);
        out.store(a.out, row * a.ld_out, a.dim, g, lanes);
    }
    if (!a.d_weight && !a.d_bias) return;
    ln_arrived<0>();
    for (int which = 0; which < 2; ++which) {
        void *const final = which ? a.d_bias : a.d_weight;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < E; ++i) joined[i * blockDim.x + threadIdx.x] = which ? db[i] : dw[i];
        __syncthreads();
        // column c of a group: vector c / V, element c % V
        for (int c = threadIdx.x; c < a.dim; c += blockDim.x) {
            const int v = c / V, i = v / lanes * V + c % V;
            float s = 0.f;
            for (int k = 0; k < groups; ++k) s += joined[i * blockDim.x + k * lanes + v % lanes];
            if (gridDim.x > 1) partial[((int64_t)blockIdx.x * 2 + which) * a.dim + c] = s;
            else if (!final) continue;
            else if (f32) reinterpret_cast<float *>(final)[c] = s;
            else reinterpret_cast<T *>(final)[c] = OpsType<T>::store(s);
        }
    }
}

// ---- launches --------------------------------------------------------------------------------------

// Widest vector (bytes) that the rows allow throughout.
int common(const LayerNormArgs &a) {
    const int w = qg_type_size(a.type);
    int bytes = qg_vec_bytes(a.x, a.ld_x * w, (int64_t)a.dim * w);
    const int out = qg_vec_bytes(a.out, a.ld_out * w, (int64_t)a.dim * w);
    if (out < bytes) bytes = out;
    if (a.grad) {
        const int grad = qg_vec_bytes(a.grad, a.ld_grad * w, (int64_t)a.dim * w);
        if (grad < bytes) bytes = grad;
    }
    return bytes;
}

// Threads of a row: one vector each up to a warp's worth, then as many vectors each as there may be, then more warps.
template <int V>
int ln_lanes(int dim) {
    const int vectors = (dim + V - 1) / V;
    if (vectors > 32) return (vectors + 32 * (LN_EACH<V> / V) - 1) / (32 * (LN_EACH<V> / V)) * 32;
    int lanes = 1;
    while (lanes < vectors) lanes *= 2;
    return lanes;
}

// Blocks of `threads` that the GPU holds at once.
template <typename K>
int ln_resident(qgbdt_ctx *c, K kernel, int threads, size_t smem, int64_t *blocks) {
    int each = 0;
    QG_CUDA(c, cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, threads, smem));
    *blocks = (int64_t)each * c->sm_count;
    return QGBDT_OK;
}

template <typename T, int V, int N, bool MULTI>
int rows_forward(qgbdt_ctx *c, const LayerNormArgs &a, int lanes, cudaStream_t st) {
    const int threads = MULTI ? lanes : 128, groups = threads / lanes;
    const int64_t want = (a.rows + groups - 1) / groups;
    const size_t smem = LnRows<T, V, N, LN_AHEAD>::bytes(threads);
    if (smem > 48 * 1024) QG_CUDA(c, cudaFuncSetAttribute(k_ln_rows<T, V, N, MULTI>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    int64_t grid = want;
    if (want > c->sm_count) {
        QG_RUN(ln_resident(c, k_ln_rows<T, V, N, MULTI>, threads, smem, &grid));
        if (want < grid) grid = want;
    }
    return qg_launch(c, k_ln_rows<T, V, N, MULTI>, dim3((unsigned)grid), threads, smem, st, a, lanes);
}

template <typename T, int V>
int rows_forward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    const int lanes = ln_lanes<V>(a.dim);
    const int each = (a.dim + lanes * V - 1) / (lanes * V);
    constexpr int most = LN_EACH<V> / V;
    if (lanes > 32) return rows_forward<T, V, most, true>(c, a, lanes, st);
    if (each == 1) return rows_forward<T, V, 1, false>(c, a, lanes, st);
    if constexpr (most > 4) {
        if (each <= 4) return rows_forward<T, V, 4, false>(c, a, lanes, st);
    }
    return rows_forward<T, V, most, false>(c, a, lanes, st);
}

template <typename T>
int forward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const int bytes = common(a);
    const bool vectors = bytes == 16;
    if (a.dim <= LN_ROW) {
        if (vectors) return rows_forward<T, V>(c, a, st);
        if constexpr (sizeof(T) == 2) {
            if (bytes >= 4) return rows_forward<T, 2>(c, a, st);
        }
        return rows_forward<T, 1>(c, a, st);
    }
    const int64_t most = (int64_t)c->sm_count * 4;
    const dim3 grid((unsigned)(a.rows < most ? a.rows : most));
    if (vectors) return qg_launch(c, k_ln_long<T, V>, grid, LN_THREADS, 0, st, a);
    return qg_launch(c, k_ln_long<T, 1>, grid, LN_THREADS, 0, st, a);
}

template <typename T, int V, int N, bool MULTI>
int rows_backward(qgbdt_ctx *c, const LayerNormArgs &a, int lanes, cudaStream_t st) {
    const int threads = lanes >= 256 ? lanes : 256 / lanes * lanes, groups = threads / lanes;
    const size_t sums_bytes = (size_t)threads * N * V * sizeof(float), ring = 2 * LnRows<T, V, N, LN_AHEAD_BACKWARD>::bytes(threads);
    const size_t smem = (size_t)(a.dim + 3) / 4 * 4 * sizeof(float) + (ring > sums_bytes ? ring : sums_bytes);
    if (smem > 48 * 1024) QG_CUDA(c, cudaFuncSetAttribute(k_ln_rows_backward<T, V, N, MULTI>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    int64_t grid = 0;
    QG_RUN(ln_resident(c, k_ln_rows_backward<T, V, N, MULTI>, threads, smem, &grid));
    // four rows per group at least: the partial sums are as large as one and a half
    const int64_t want = (a.rows + groups * 4 - 1) / (groups * 4);
    if (want < grid) grid = want;
    if (grid < 1) grid = 1;
    const bool sums = a.d_weight || a.d_bias;
    if (!sums || grid == 1) return qg_launch(c, k_ln_rows_backward<T, V, N, MULTI>, dim3((unsigned)grid), threads, smem, st, a, (float *)nullptr, lanes);
    QgWorkspace ws;
    QG_RUN(qg_ws_open(c, qg_ws_size((size_t)grid * 2 * a.dim, sizeof(float)), st, &ws));
    float *partial = ws.take<float>((size_t)grid * 2 * a.dim);
    QG_RUN(qg_launch(c, k_ln_rows_backward<T, V, N, MULTI>, dim3((unsigned)grid), threads, smem, st, a, partial, lanes));
    QG_RUN(qg_launch(c, k_ln_join<T>, dim3((a.dim + 31) / 32, 2), 32 * LN_JOIN, 0, st, a, partial, (int)grid));
    return qg_ws_close(c, st);
}

template <typename T, int V>
int rows_backward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    const int lanes = ln_lanes<V>(a.dim);
    const int each = (a.dim + lanes * V - 1) / (lanes * V);
    constexpr int most = LN_EACH<V> / V;
    if (lanes > 32) return rows_backward<T, V, most, true>(c, a, lanes, st);
    if (each == 1) return rows_backward<T, V, 1, false>(c, a, lanes, st);
    if constexpr (most > 4) {
        if (each <= 4) return rows_backward<T, V, 4, false>(c, a, lanes, st);
    }
    return rows_backward<T, V, most, false>(c, a, lanes, st);
}

template <typename T>
int backward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const int bytes = common(a);
    const bool vectors = bytes == 16;
    if (a.dim <= LN_ROW) {
        if (vectors) return rows_backward<T, V>(c, a, st);
        if constexpr (sizeof(T) == 2) {
            if (bytes >= 4) return rows_backward<T, 2>(c, a, st);
        }
        return rows_backward<T, 1>(c, a, st);
    }
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
    if (vectors) return qg_launch(c, k_ln_long_dx<T, V>, grid, LN_THREADS, 0, st, a);
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
