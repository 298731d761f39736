// Layer norm of rows, and its gradients.
//
//   mean = sum x / d,  rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),  out = (x - mean) rstd w + b
//   xh = (x - mean) rstd,  dx = rstd (w g - sum (w g) / d - xh sum (w g xh) / d),  dw = sum over rows of g xh,  db = sum over rows of g
//
// Sums and statistics are held in single precision; an output is rounded once, when it is written.
//
// Rows of up to 8192 columns (forward mostly 16384) are held in registers and read once: bound by memory traffic where a row's threads have many
// elements (16384 x 8192 bf16: 90 to 99 us, 5.4 to 6.0 TB/s; gradients of 65536 x 1024 bf16: 73 us, 5.5 TB/s), by instructions where they have
// few (65536 x 256 bf16: 13 us, 5.1 TB/s; 13 instructions per element, of which the elements' own are 5) and where rows start anywhere
// (60000 x 1001 bf16: 67 us, 3.6 TB/s; 25 instructions).  Small calls are bound by the launch, and, where the sums over the rows come from
// several blocks, by a second one (3.5 us).  Longer rows are cut into segments and read twice.
#include <type_traits>

#include "ops_internal.cuh"

namespace {

// ---- rows longer than a block's registers -----------------------------------------------------------
// A row is cut into segments of LN_SEGMENT elements, so that few long rows occupy the GPU too.  A first launch takes every
// segment's share of the row's sums (forward: mean and sum of squared differences from it, backward: sums of w g and w g xh), a second one
// joins the shares of the row in their order, in every block that needs them, and writes.  Inputs are read twice, the
// second time from L2 where they fit: 1.5 times the bytes forward, 1.67 backward.  One row of 2^20 columns in bf16 takes 8.6 us (by
// a single block: 354), 2048 x 32768 136 us, gradients of 4096 x 16384 164 us.  That is 2.2 and 1.6 times what those bytes take: the shares are
// bound by instructions (18 per element, 69 % of the issue slots), the writers by latency (a row is asked for when the one before it is
// done: 45 % of the issue slots, 4 to 5 warps waiting for memory per instruction).

constexpr int LN_THREADS = 256, LN_PIECE = 16;      // elements per thread
constexpr int LN_SEGMENT = LN_THREADS * LN_PIECE;

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

// A thread's elements of a segment: vectors tid, tid + LN_THREADS, ...; zeros outside the row.  V = 1: rows that start anywhere.
template <typename T, int V>
struct LnPiece {
    static constexpr int N = LN_PIECE / V;
    OpsVec<T, V> v[N];
    __device__ __forceinline__ static int column(int i) { return (i * LN_THREADS + (int)threadIdx.x) * V; }
    __device__ __forceinline__ void load(const void *p, int64_t at, int n) {      // n: elements of the segment
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = OpsVec<T, V>{};
            if (column(i) < n) v[i] = *reinterpret_cast<const OpsVec<T, V> *>(reinterpret_cast<const T *>(p) + at + column(i));
        }
    }
    __device__ __forceinline__ void store(void *p, int64_t at, int n) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (column(i) < n) *reinterpret_cast<OpsVec<T, V> *>(reinterpret_cast<T *>(p) + at + column(i)) = v[i];
    }
    __device__ __forceinline__ float get(int e) const { return OpsType<T>::load(v[e / V].v[e % V]); }
    __device__ __forceinline__ void set(int e, float x) { v[e / V].v[e % V] = OpsType<T>::store(x); }
    __device__ __forceinline__ static int place(int e) { return column(e / V) + e % V; }
};

// Elements of segment i of a row.
__device__ __forceinline__ int ln_segment(int dim, int i) { return min(LN_SEGMENT, dim - i * LN_SEGMENT); }

// The columns' weights of a thread's elements of a segment, of n elements from column `first` on; zeros outside the row.
template <typename T, int V>
__device__ __forceinline__ void ln_weights(float (&w)[LN_PIECE], const void *weight, bool f32, int first, int n, float none) {
#pragma unroll
    for (int e = 0; e < LN_PIECE; ++e) w[e] = LnPiece<T, V>::place(e) < n ? ln_weight<T>(weight, f32, first + LnPiece<T, V>::place(e), none) : 0.f;
}

// A block has a segment (blockIdx.x) of every gridDim.y-th row, so that the columns' weights stay in registers.
template <typename T, int V, bool BACKWARD>
__global__ void __launch_bounds__(LN_THREADS) k_ln_shares(const LayerNormArgs a, float2 *shares, int segments) {
    qg_after_prior();
    __shared__ float2 part[2][32];
    int at = 0;
    const int segment = blockIdx.x, n = ln_segment(a.dim, segment), first = segment * LN_SEGMENT;
    float w[LN_PIECE];
    if (BACKWARD) ln_weights<T, V>(w, a.weight, a.weight_type == QGBDT_F32, first, n, 1.f);
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        LnPiece<T, V> x;
        x.load(a.x, row * a.ld_x + first, n);
        float2 s = make_float2(0.f, 0.f);
        if constexpr (!BACKWARD) {
#pragma unroll
            for (int e = 0; e < LN_PIECE; ++e) s.x += x.get(e);
            const float mean = ln_block_sum(s, part, at).x / (float)n;
            s.x = 0.f;
#pragma unroll
            for (int e = 0; e < LN_PIECE; ++e) {
                const float y = x.get(e) - mean;
                if (x.place(e) < n) s.x = fmaf(y, y, s.x);
            }
            s = ln_block_sum(s, part, at);
            if (threadIdx.x == 0) shares[row * segments + segment] = make_float2(mean, s.x);
        } else {
            const float mean = a.mean[row], rstd = a.rstd[row];
            LnPiece<T, V> u;
            u.load(a.grad, row * a.ld_grad + first, n);
#pragma unroll
            for (int e = 0; e < LN_PIECE; ++e) {
                const float y = u.get(e) * w[e];      // zero outside the row
                s.x += y;
                s.y = fmaf(y, (x.get(e) - mean) * rstd, s.y);
            }
            s = ln_block_sum(s, part, at);
            if (threadIdx.x == 0) shares[row * segments + segment] = s;
        }
    }
}

__device__ __forceinline__ float ln_warp_sum(float s) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

template <typename T, int V>
__global__ void __launch_bounds__(LN_THREADS) k_ln_segments(const LayerNormArgs a, const float2 *shares, int segments) {
    qg_after_prior();
    const bool f32 = a.weight_type == QGBDT_F32;
    const int lane = threadIdx.x & 31, segment = blockIdx.x, n = ln_segment(a.dim, segment), first = segment * LN_SEGMENT;
    const float per = 1.f / (float)a.dim;
    float w[LN_PIECE], b[LN_PIECE];
    ln_weights<T, V>(w, a.weight, f32, first, n, 1.f);
    ln_weights<T, V>(b, a.bias, f32, first, n, 0.f);
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        LnPiece<T, V> x;
        x.load(a.x, row * a.ld_x + first, n);
        const float2 *const of = shares + row * segments;
        float s = 0.f;
        for (int i = lane; i < segments; i += 32) s = fmaf(of[i].x, (float)ln_segment(a.dim, i), s);
        const float mean = ln_warp_sum(s) * per;
        s = 0.f;
        for (int i = lane; i < segments; i += 32) {
            const float z = of[i].x - mean;
            s += fmaf(z * (float)ln_segment(a.dim, i), z, of[i].y);
        }
        const float rstd = rsqrtf(fmaf(ln_warp_sum(s), per, a.eps));
#pragma unroll
        for (int e = 0; e < LN_PIECE; ++e) x.set(e, fmaf((x.get(e) - mean) * rstd, w[e], b[e]));
        x.store(a.out, row * a.ld_out + first, n);
        if (segment == 0 && threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// A block has a segment of a slice of the rows, and the sums over those rows: partial [slices][2][dim] (of the weight's gradient, of
// the bias's).
template <typename T, int V>
__global__ void __launch_bounds__(LN_THREADS, 2) k_ln_segments_backward(const LayerNormArgs a, const float2 *shares, float *partial, int segments) {
    qg_after_prior();
    const int lane = threadIdx.x & 31, segment = blockIdx.x, n = ln_segment(a.dim, segment), first = segment * LN_SEGMENT;
    const int64_t r0 = a.rows * blockIdx.y / gridDim.y, r1 = a.rows * (blockIdx.y + 1) / gridDim.y;
    const float per = 1.f / (float)a.dim;
    float w[LN_PIECE], dw[LN_PIECE] = {}, db[LN_PIECE] = {};
    ln_weights<T, V>(w, a.weight, a.weight_type == QGBDT_F32, first, n, 1.f);
    for (int64_t row = r0; row < r1; ++row) {
        LnPiece<T, V> x, u;
        x.load(a.x, row * a.ld_x + first, n);
        u.load(a.grad, row * a.ld_grad + first, n);
        const float mean = a.mean[row], rstd = a.rstd[row];
        float2 s = make_float2(0.f, 0.f);
        for (int i = lane; i < segments; i += 32) s.x += shares[row * segments + i].x, s.y += shares[row * segments + i].y;
        const float c1 = ln_warp_sum(s.x) * per, c2 = ln_warp_sum(s.y) * per;
#pragma unroll
        for (int e = 0; e < LN_PIECE; ++e) {
            const float g = u.get(e), xh = (x.get(e) - mean) * rstd;
            dw[e] = fmaf(g, xh, dw[e]);      // (outside the row: never read)
            db[e] += g;
            u.set(e, (g * w[e] - c1 - xh * c2) * rstd);
        }
        u.store(a.out, row * a.ld_out + first, n);
    }
    if (!partial) return;
    float *const to = partial + (int64_t)blockIdx.y * 2 * a.dim + first;
#pragma unroll
    for (int e = 0; e < LN_PIECE; ++e) {
        const int c = LnPiece<T, V>::place(e);
        if (c < n) to[c] = dw[e], to[a.dim + c] = db[e];
    }
}

// The partial sums joined in their order: 32 columns per block, LN_JOIN parts of the slices side by side.
constexpr int LN_JOIN = 32;      // (a warp's lanes)

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
    const int64_t column = (int64_t)blockIdx.x * 32 + part;       // a warp per column
    s = w[lane][part];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0 && column < a.dim) {
        if (a.weight_type == QGBDT_F32) reinterpret_cast<float *>(out)[column] = s;
        else reinterpret_cast<T *>(out)[column] = OpsType<T>::store(s);
    }
}

// Few slices: a thread per column, of the weight's gradient and then of the bias's.
constexpr int LN_FEW = 16;

template <typename T>
__global__ void __launch_bounds__(LN_THREADS) k_ln_join_few(const LayerNormArgs a, const float *partial, int slices) {
    qg_after_prior();
    const int64_t i = (int64_t)blockIdx.x * LN_THREADS + threadIdx.x, c = i < a.dim ? i : i - a.dim;
    void *const out = i < a.dim ? a.d_weight : a.d_bias;
    if (i >= 2 * (int64_t)a.dim || !out) return;
    float s = 0.f;
#pragma unroll 8
    for (int k = 0; k < slices; ++k) s += partial[(int64_t)k * 2 * a.dim + i];
    if (a.weight_type == QGBDT_F32) reinterpret_cast<float *>(out)[c] = s;
    else reinterpret_cast<T *>(out)[c] = OpsType<T>::store(s);
}

template <typename T>
int ln_join(qgbdt_ctx *c, const LayerNormArgs &a, const float *partial, int slices, cudaStream_t st) {
    if (slices <= LN_FEW) return qg_launch(c, k_ln_join_few<T>, dim3((unsigned)((2 * (int64_t)a.dim + LN_THREADS - 1) / LN_THREADS)), LN_THREADS, 0, st, a, partial, slices);
    return qg_launch(c, k_ln_join<T>, dim3((a.dim + 31) / 32, 2), 32 * LN_JOIN, 0, st, a, partial, slices);
}

// ---- rows that fit in registers ---------------------------------------------------------------------
// `lanes` threads have a row: a power of two up to 32, or whole warps.  A warp has N * 32 neighbouring vectors of 16 bytes (V elements),
// each of its threads every 32nd of them (fewer threads: every lanes-th).  What belongs to the columns stays in registers over all
// rows.  EXACT: every vector is inside the row.  Single elements: so are those of all warps but the last, which take a loop without
// checks (60000 x 1000 bf16 that starts anywhere: 64 instead of 78 us when it came; 16-byte vectors have one loop, whose registers decide there:
// 7000 x 8192 gradients 84 us, 104 with two).
// Instructions bound these kernels as soon as the memory does not: sums and products are taken of two elements at once,
// and rows whose threads have few elements are worked on two at a time, which share the exchanges of their sums.

constexpr int LN_ROW = 8192;     // elements of a row, at most
constexpr int LN_LONG = 16384;   // forward, vectors, where the copies ahead fit (4096 x 16384 bf16: 50 us, in segments 136)
constexpr int LN_SHARED = 224 * 1024;   // bytes of shared memory that a block can have for them
// What a launch may give a block without leave for more, and with it: 48 and 227 KB, less what the kernels hold themselves.
using LnParts = float2[2][32];
constexpr size_t LN_LEAVE = 48 * 1024 - sizeof(LnParts);
constexpr int LN_MOST = 227 * 1024 - (int)sizeof(LnParts);
constexpr int LN_EACH = 16;      // per thread of a warp that has rows of its own, at most
// Elements per thread where a row has several warps.  Forward, vectors of 16-bit elements: 32, so that the sums and loops are for more of
// them (16384 x 8192 bf16: 92 instead of 100 us; f32: no difference, 16).  Backward: 16, and 8 in rows of f32 above 2048 columns, whose
// threads then come to 32 instead of 16 warps of an SM (7324 x 4096: 73 instead of 76 us; bf16: 47 instead of 45).
template <typename T, int V>
constexpr int LN_MANY = V > 1 && sizeof(T) == 2 ? 32 : 16;
constexpr int LN_WIDE = 2048;
// Threads that the registers of a row's threads leave room for, single elements forward: two rows of up to 5120 columns on an SM
// (10000 x 4097 f32: 62 us, with registers for 512 threads 84; for 768 threads 15000 x 4096 bf16 takes 59 instead of 69 us, but
// 60000 x 1000 78 instead of 67).
constexpr int LN_LOOSE = 640;
template <int E, bool MULTI>
constexpr int LN_PAIR = !MULTI && E <= 8 ? 2 : 1;    // rows at a time

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(*reinterpret_cast<uint64_t *>(&r)) : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(*reinterpret_cast<uint64_t *>(&r)) : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(*reinterpret_cast<uint64_t *>(&r))
        : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)), "l"(*reinterpret_cast<uint64_t *>(&c)));
    return r;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Sums of K values over a power of two of neighbouring lanes, the same in all of them, in a fixed order.  Two values cost little
// more than one: each half of the lanes takes one of them from the other half and goes on with that; then they are handed back.
template <int K>
__device__ __forceinline__ void ln_sum(float (&v)[K], int lanes) {
    if constexpr (K == 1) {
#pragma unroll
        for (int o = 16; o; o >>= 1)
            if (o < lanes) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    } else {
        if (lanes < 2) return;
        const int half = lanes / 2;
        const bool upper = threadIdx.x & half;
        float w[K / 2];
#pragma unroll
        for (int k = 0; k < K / 2; ++k) {
            const float give = upper ? v[k] : v[k + K / 2];
            w[k] = (upper ? v[k + K / 2] : v[k]) + __shfl_xor_sync(0xffffffffu, give, half);
        }
        ln_sum<K / 2>(w, half);
#pragma unroll
        for (int k = 0; k < K / 2; ++k) {
            const float other = __shfl_xor_sync(0xffffffffu, w[k], half);
            v[k] = upper ? other : w[k];
            v[k + K / 2] = upper ? w[k] : other;
        }
    }
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

// Which vectors of a row a thread has: from `home` on every APART-th (0: every lanes-th).
template <int V, int N, int APART>
struct LnPlace {
    int dim, lanes, home;
    __device__ __forceinline__ LnPlace(int dim_, int lanes_, int g) : dim(dim_), lanes(lanes_), home(APART ? (g & ~31) * N + (g & 31) : g) {}
    __device__ __forceinline__ static int apart_of(int lanes) { return APART ? APART : lanes; }
    __device__ __forceinline__ int apart() const { return apart_of(lanes); }
    __device__ __forceinline__ int column(int i) const { return (home + i * apart()) * V; }
    template <bool WHOLE>
    __device__ __forceinline__ bool in(int i) const {
        return WHOLE || column(i) < dim;
    }
    // whether all vectors of the warp are inside the row
    __device__ __forceinline__ bool whole() const { return (APART ? (home / (32 * N) + 1) * 32 : lanes) * N * V <= dim; }
};
// Known to the compiler where a row always has a warp or more: rows_cut() takes the first N that is enough for a warp, so the
// next one, if at most twice that, has all 32.
template <int V, int N, bool MULTI>
constexpr int LN_APART = MULTI || N == (V > 1 ? 2 : 8) || (V == 1 && N == 16) ? 32 : 0;

// A thread's vectors of a row.  V = 1: single elements, of rows that start anywhere.
template <typename T, int V, int N>
struct LnRow {
    using Vec = OpsVec<T, V>;
    static constexpr int E = N * V, PAIRS = E / 2;
    Vec v[N];
    template <bool WHOLE, typename PLACE>
    __device__ __forceinline__ void store(T *p, const PLACE &place) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (place.template in<WHOLE>(i)) *reinterpret_cast<Vec *>(p + place.column(i)) = v[i];
    }
    __device__ __forceinline__ float2 get(int p) const {   // elements 2 p and 2 p + 1
        if constexpr (V == 1 || sizeof(T) == 4) {
            return make_float2(OpsType<T>::load(v[2 * p / V].v[2 * p % V]), OpsType<T>::load(v[(2 * p + 1) / V].v[(2 * p + 1) % V]));
        } else {
            const unsigned w = *reinterpret_cast<const unsigned *>(&v[2 * p / V].v[2 * p % V]);
            if constexpr (OpsType<T>::BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
            else return __half22float2(*reinterpret_cast<const __half2 *>(&w));
        }
    }
    __device__ __forceinline__ void set(int p, float2 x) {
        if constexpr (V == 1 || sizeof(T) == 4) {
            v[2 * p / V].v[2 * p % V] = OpsType<T>::store(x.x), v[(2 * p + 1) / V].v[(2 * p + 1) % V] = OpsType<T>::store(x.y);
        } else {
            T *const q = &v[2 * p / V].v[2 * p % V];
            if constexpr (OpsType<T>::BF16) *reinterpret_cast<__nv_bfloat162 *>(q) = __float22bfloat162_rn(x);
            else *reinterpret_cast<__half2 *>(q) = __float22half2_rn(x);
        }
    }
};

// The coming rows of an input, copied asynchronously to the shared memory, DEPTH steps of ROWS rows ahead: the memory's latency under
// load takes 64 KB on their way per SM.  A thread's vectors go to places of its own, so that nobody waits for another thread's copies.
// Rows that start anywhere (V = 1): such copies come in aligned vectors, so a row is copied as the aligned vectors that hold it, by its threads
// for one another.  (Where a row starts inside a vector, the elements in front of it come along; what is in front of the
// first row is not read.  The last vector is copied as far as the row goes, and zeros follow up to the threads' last elements.)
template <typename T, int V, int N, int ROWS, int DEPTH>
struct LnAhead {
    static constexpr bool LOOSE = V == 1;
    using Row = LnRow<T, V, N>;
    using Vec = typename Row::Vec;
    // vectors of 16 bytes of a row in a slot
    __host__ __device__ static constexpr int vectors(int lanes) { return LOOSE ? (lanes * N * (int)sizeof(T) + 15) / 16 + 1 : lanes * N; }
    __host__ __device__ static constexpr size_t bytes(int threads, int lanes) { return (size_t)16 * vectors(lanes) * (threads / lanes) * ROWS * DEPTH; }
    const T *from, *first;    // the next row to be fetched; the first of all
    int64_t ld, step;         // elements
    const unsigned char *ring;   // the group's first row, or the thread's first vector
    uint32_t ring_at;         // its shared address
    int slot_bytes;
    unsigned before, before_step, before_row;   // LOOSE: bytes of a vector in front of the first row to be taken; what a step and a row add
    __device__ __forceinline__ LnAhead(const void *p, int64_t ld_, unsigned unit, unsigned stride, int lanes, int group, void *shared)
        : from(reinterpret_cast<const T *>(p) + (int64_t)unit * ROWS * ld_), first(reinterpret_cast<const T *>(p)), ld(ld_), step((int64_t)stride * ROWS * ld_) {
        slot_bytes = 16 * vectors(lanes) * (blockDim.x / lanes);
        ring = reinterpret_cast<const unsigned char *>(shared) + (LOOSE ? group * vectors(lanes) : (int)threadIdx.x) * 16;
        ring_at = (uint32_t)__cvta_generic_to_shared(ring);
        before = (unsigned)reinterpret_cast<uintptr_t>(from) & 15, before_step = (unsigned)step * sizeof(T) & 15, before_row = (unsigned)ld * sizeof(T) & 15;
    }
    template <bool WHOLE, typename PLACE>
    __device__ __forceinline__ void fetch(int slot, unsigned row, unsigned rows, const PLACE &place, int g) {
        const int dim = place.dim, lanes = place.lanes;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (row + r >= rows) continue;
            const T *const q = from + r * ld;
            const uint32_t to = ring_at + (slot * ROWS + r) * slot_bytes;
            if constexpr (LOOSE) {
                const int front = (int)(reinterpret_cast<uintptr_t>(q) & 15), all = front + dim * (int)sizeof(T);   // bytes
                const char *const w = reinterpret_cast<const char *>(q) - front;
                const bool begins = g == 0 && w < reinterpret_cast<const char *>(first);
                if (begins)
                    for (int e = 0; e < (16 - front) / (int)sizeof(T); ++e) {
                        const bool is = e < dim;
                        if constexpr (sizeof(T) == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + front + 4 * e), "f"(is ? q[e] : 0.f) : "memory");
                        else asm volatile("st.shared.b16 [%0], %1;" ::"r"(to + front + 2 * e), "h"(is ? reinterpret_cast<const unsigned short *>(q)[e] : (unsigned short)0) : "memory");
                    }
                auto upto_end = [&](int j) {
                    const int left = max(0, min(16, all - 16 * j));
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + 16 * j), "l"(w + 16 * min(j, (all - 1) / 16)), "r"(left) : "memory");
                };
                if constexpr (N * sizeof(T) >= 16) {     // each warp the vectors of its elements, the first thread the one more
                    constexpr int K = N * (int)sizeof(T) / 16;
                    const int own = PLACE::apart_of(lanes), j = own == lanes ? g : (g & ~31) * K + (g & 31);
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        if (k == 0 && begins) continue;
                        if (WHOLE) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 16 * (j + k * own)), "l"(w + 16 * (j + k * own)) : "memory");
                        else upto_end(j + k * own);
                    }
                    if (g == 0) upto_end(vectors(lanes) - 1);
                } else {
                    for (int j = begins ? lanes : g; j < vectors(lanes); j += lanes) upto_end(j);
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (place.template in<WHOLE>(i))
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * blockDim.x * 16), "l"(q + place.column(i)) : "memory");
            }
        }
        from += step;
    }
    // Zeros outside the row.
    template <bool WHOLE, typename PLACE>
    __device__ __forceinline__ void take(Row &x, int slot, int r, const PLACE &place) const {
        const unsigned char *const at = ring + (slot * ROWS + r) * slot_bytes;
        if constexpr (LOOSE) {
            const T *const q = reinterpret_cast<const T *>(at + ((before + r * before_row) & 15)) + place.home;
#pragma unroll
            for (int i = 0; i < N; ++i) x.v[i].v[0] = q[i * place.apart()];
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint4 q = make_uint4(0, 0, 0, 0);
                if (place.template in<WHOLE>(i)) q = reinterpret_cast<const uint4 *>(at)[i * blockDim.x];
                *reinterpret_cast<uint4 *>(&x.v[i]) = q;
            }
        }
    }
    __device__ __forceinline__ void taken() { before = (before + before_step) & 15; }   // a step
};

__device__ __forceinline__ void ln_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void ln_arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }   // all but the last LEFT
// The same for the copies of all threads of a row.
template <int LEFT, bool LOOSE, bool MULTI>
__device__ __forceinline__ void ln_row_arrived(int lanes, int barrier) {
    ln_arrived<LEFT>();
    if constexpr (LOOSE && MULTI) asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(lanes) : "memory");
    else if constexpr (LOOSE) __syncwarp();
}

template <int ROWS>
constexpr int LN_AHEAD = ROWS == 1 ? 4 : 2;             // steps
template <int ROWS>
constexpr int LN_AHEAD_BACKWARD = ROWS == 1 ? 3 : 2;

// Mean and sum of squared differences from it: over a warp in two passes; the warps' are joined by
//   sum over warps of M2 + count (mean of the warp - mean)^2,
// which takes one exchange and loses nothing where the mean is large beside the differences.
template <typename T, int V, int N, bool MULTI, bool EXACT>
__global__ void __launch_bounds__(MULTI ? (V > 1 ? LN_LONG / (N * V) : LN_LOOSE) : 128, 1) k_ln_rows(const LayerNormArgs a, int lanes) {
    qg_after_prior();
    extern __shared__ __align__(16) unsigned char shared_bytes[];
    __shared__ LnParts part;
    constexpr int E = N * V, R = LN_PAIR<E, MULTI>, AHEAD = LN_AHEAD<R>;
    using Ahead = LnAhead<T, V, N, R, AHEAD>;
    constexpr bool LOOSE = Ahead::LOOSE;
    using Row = typename Ahead::Row;
    constexpr int P = Row::PAIRS;
    const int groups = MULTI ? 1 : blockDim.x / lanes, group = MULTI ? 0 : threadIdx.x / lanes, g = MULTI ? threadIdx.x : threadIdx.x & (lanes - 1), dim = a.dim;
    const unsigned rows = (unsigned)a.rows, stride = gridDim.x * groups, units = (rows + R - 1) / R;
    const float per = 1.f / (float)dim;
    unsigned unit = blockIdx.x * groups + group;
    const LnPlace<V, N, LN_APART<V, N, MULTI>> place(dim, lanes, g);
    Ahead in(a.x, a.ld_x, unit, stride, lanes, group, shared_bytes);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
        in.template fetch<EXACT>(k, (unit + k * stride) * R, rows, place, g);
        ln_commit();
    }
    // elements of a row that a warp has: this one, and the one with this lane's number
    auto elements = [&](int warp) { return (float)max(0, min(32 * E, dim - warp * 32 * E)); };
    const float count = MULTI && (int)(threadIdx.x & 31) < lanes / 32 ? elements(threadIdx.x & 31) : 0.f, warp_count = MULTI ? elements(threadIdx.x / 32) : (float)dim;
    const float warp_per = warp_count > 0.f ? 1.f / warp_count : 0.f;
    const int warps = ln_power(lanes / 32);
    const bool f32 = a.weight_type == QGBDT_F32;
    float2 w[P], b[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        float *const q[2] = {&w[p].x, &b[p].x};
        for (int k = 0; k < 2; ++k) {
            const int e = 2 * p + k, c = place.column(e / V) + e % V;
            const bool is = c < dim;
            q[0][k] = is ? ln_weight<T>(a.weight, f32, c, 1.f) : 0.f;
            q[1][k] = is ? ln_weight<T>(a.bias, f32, c, 0.f) : 0.f;
        }
    }
    T *out = reinterpret_cast<T *>(a.out) + (int64_t)unit * R * a.ld_out;
    const int64_t out_step = (int64_t)stride * R * a.ld_out;
    int at = 0, slot = 0;
    auto work = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        for (unsigned base = unit - group; base < units; base += stride, unit += stride, out += out_step) {
            ln_row_arrived<AHEAD - 1, LOOSE, MULTI>(lanes, 1);
            float2 y[R][P];
            float s[R], mean[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                Row x;
                in.template take<WHOLE>(x, slot, r, place);
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int p = 0; p < P; ++p) y[r][p] = x.get(p), sum = add2(sum, y[r][p]);
                s[r] = sum.x + sum.y;
            }
            auto fetch = [&] {
                in.taken();
                in.template fetch<WHOLE>(slot, (unit + AHEAD * stride) * R, rows, place, g);
                ln_commit();
                slot = slot + 1 < AHEAD ? slot + 1 : 0;
            };
            if (!LOOSE) fetch();
            ln_sum<R>(s, MULTI ? 32 : lanes);
            if (LOOSE && !MULTI) fetch();      // when all threads have taken theirs
#pragma unroll
            for (int r = 0; r < R; ++r) {
                mean[r] = s[r] * warp_per;
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    float2 z = add2(y[r][p], both(-mean[r]));
                    if (!place.template in<WHOLE>(2 * p / V)) z.x = 0.f;
                    if (!place.template in<WHOLE>((2 * p + 1) / V)) z.y = 0.f;
                    sum = fma2(z, z, sum);
                    if (!MULTI) y[r][p] = z;
                }
                s[r] = sum.x + sum.y;
            }
            ln_sum<R>(s, MULTI ? 32 : lanes);
            if constexpr (MULTI) {
                const float2 other = ln_exchange(make_float2(mean[0], s[0]), lanes, part, at, 1);
                if (LOOSE) fetch();
                float m[1] = {other.x * count};
                ln_sum<1>(m, warps);
                mean[0] = m[0] * per;
                const float z = other.x - mean[0];
                m[0] = fmaf(z * count, z, other.y);
                ln_sum<1>(m, warps);
                mean[0] = __shfl_sync(0xffffffffu, mean[0], 0), s[0] = __shfl_sync(0xffffffffu, m[0], 0);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const unsigned row = unit * R + r;
                if (row >= rows) continue;
                const float rstd = rsqrtf(fmaf(s[r], per, a.eps));      // (two units in the last place)
                Row x;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const float2 z = MULTI ? add2(y[r][p], both(-mean[r])) : y[r][p];
                    x.set(p, fma2(mul2(z, both(rstd)), w[p], b[p]));
                }
                x.template store<WHOLE>(out + r * a.ld_out, place);
                if (g == 0) {
                    if (a.mean) a.mean[row] = mean[r];
                    if (a.rstd) a.rstd[row] = rstd;
                }
            }
        }
    };
    if (EXACT || (LOOSE && place.whole())) work(std::true_type{});
    else work(std::false_type{});
}

// The gradients; the sums over the rows are gathered by column in registers, joined in shared memory over the block's groups and
// written as the block's part of partial [blocks][2][dim], or, from a single block, as they are.
template <typename T, int V, int N, bool MULTI, bool EXACT>
__global__ void __launch_bounds__(MULTI ? LN_ROW / (N * V) : 256) k_ln_rows_backward(const LayerNormArgs a, float *partial, int lanes) {
    qg_after_prior();
    extern __shared__ __align__(16) unsigned char shared_bytes[];
    __shared__ LnParts part;
    constexpr int E = N * V, R = LN_PAIR<E, MULTI>, AHEAD = LN_AHEAD_BACKWARD<R>;
    using Ahead = LnAhead<T, V, N, R, AHEAD>;
    constexpr bool LOOSE = Ahead::LOOSE;
    using Row = typename Ahead::Row;
    constexpr int P = Row::PAIRS;
    const int groups = blockDim.x / lanes, group = threadIdx.x / lanes, g = threadIdx.x - group * lanes, dim = a.dim;
    const unsigned rows = (unsigned)a.rows, stride = gridDim.x * groups, units = (rows + R - 1) / R;
    const float per = 1.f / (float)dim;
    // weight (zeros outside the row; of a warp's vectors of 8 the first halves, then the second ones, so that its threads read from all
    // banks); the coming rows of x and of the gradient, afterwards the columns' sums [2 P][threads]
    float *const weight = reinterpret_cast<float *>(shared_bytes), *const joined = weight + lanes * E;
    unsigned unit = blockIdx.x * groups + group;
    unsigned char *const rings = reinterpret_cast<unsigned char *>(joined);
    const size_t ring = Ahead::bytes(blockDim.x, lanes);
    Ahead in_x(a.x, a.ld_x, unit, stride, lanes, group, rings), in_u(a.grad, a.ld_grad, unit, stride, lanes, group, rings + ring);
    const LnPlace<V, N, LN_APART<V, N, MULTI>> place(dim, lanes, g);
    auto fetch = [&](auto whole, int slot, unsigned row) {
        in_x.template fetch<decltype(whole)::value>(slot, row, rows, place, g);
        in_u.template fetch<decltype(whole)::value>(slot, row, rows, place, g);
        ln_commit();
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) fetch(std::bool_constant<EXACT>{}, k, (unit + k * stride) * R);
    // mean and rstd: a lane has those of one of the group's next `turns` steps, and of as many after those
    const int turns = lanes < 32 ? lanes : 32, mine = threadIdx.x & (turns - 1);
    float2 stats[R], later[R];
    auto statistics = [&](float2 (&to)[R], unsigned of) {
#pragma unroll
        for (int r = 0; r < R; ++r) to[r] = of * R + r < rows ? make_float2(a.mean[of * R + r], a.rstd[of * R + r]) : make_float2(0.f, 0.f);
    };
    statistics(stats, unit + mine * stride);
    const bool f32 = a.weight_type == QGBDT_F32;
    const int plane = place.apart() * N;      // a warp's vectors
    const float4 *const weights = reinterpret_cast<const float4 *>(weight) + (MULTI ? (g & ~31) * N * (V / 4) + (g & 31) : g);
    for (int c = threadIdx.x; c < lanes * E; c += blockDim.x) {
        const int to = LOOSE ? c : (c / (V * plane) * (V / 4) * plane + c / 4 % (V / 4) * plane + c / V % plane) * 4 + c % 4;
        weight[to] = c < dim ? ln_weight<T>(a.weight, f32, c, 1.f) : 0.f;
    }
    __syncthreads();
    float2 dw[P] = {}, db[P] = {};
    T *out = reinterpret_cast<T *>(a.out) + (int64_t)unit * R * a.ld_out;
    const int64_t out_step = (int64_t)stride * R * a.ld_out;
    const int warps = ln_power(lanes / 32);
    int at = 0, slot = 0, turn = 0;
    auto work = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        for (unsigned base = unit - group; base < units; base += stride, unit += stride, out += out_step) {
            if (turn == 0) statistics(later, unit + (mine + turns) * stride);
            float2 xh[R][P], y[R][P];
            float s[2 * R], rstd[R];
            ln_row_arrived<AHEAD - 1, LOOSE, MULTI>(lanes, 1 + group);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float mean = __shfl_sync(0xffffffffu, stats[r].x, turn, turns);
                rstd[r] = __shfl_sync(0xffffffffu, stats[r].y, turn, turns);
                Row x, u;
                in_x.template take<WHOLE>(x, slot, r, place);
                in_u.template take<WHOLE>(u, slot, r, place);
                float2 sum = make_float2(0.f, 0.f), along = sum;
                if (unit * R + r >= rows) {        // (what its slot holds may be anything)
#pragma unroll
                    for (int i = 0; i < N; ++i) x.v[i] = u.v[i] = typename Row::Vec{};
                }
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const float2 v = u.get(p), h = mul2(add2(x.get(p), both(-mean)), both(rstd[r]));     // v is zero outside the row
                    db[p] = add2(db[p], v);
                    dw[p] = fma2(v, h, dw[p]);
                    float2 w;
                    if constexpr (LOOSE) w = make_float2(weight[place.column(2 * p)], weight[place.column(2 * p + 1)]);
                    else w = reinterpret_cast<const float2 *>(weights + 2 * p % V / 4 * plane + 2 * p / V * place.apart())[p % 2];
                    xh[r][p] = h;
                    y[r][p] = mul2(v, w);
                    sum = add2(sum, y[r][p]);
                    along = fma2(y[r][p], h, along);
                }
                s[2 * r] = sum.x + sum.y, s[2 * r + 1] = along.x + along.y;
            }
            if (++turn == turns) {
                turn = 0;
#pragma unroll
                for (int r = 0; r < R; ++r) stats[r] = later[r];
            }
            auto next = [&] {
                in_x.taken(), in_u.taken();
                fetch(whole, slot, (unit + AHEAD * stride) * R);
                slot = slot + 1 < AHEAD ? slot + 1 : 0;
            };
            if (!LOOSE) next();
            ln_sum<2 * R>(s, MULTI ? 32 : lanes);
            if (LOOSE && !MULTI) next();       // when all threads have taken theirs
            if constexpr (MULTI) {
                const float2 other = ln_exchange(make_float2(s[0], s[1]), lanes, part, at, 1 + group);
                if (LOOSE) next();
                s[0] = other.x, s[1] = other.y;
                ln_sum<2>(s, warps);
                s[0] = __shfl_sync(0xffffffffu, s[0], 0), s[1] = __shfl_sync(0xffffffffu, s[1], 0);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (unit * R + r >= rows) continue;
                const float2 c1 = both(-s[2 * r] * per), c2 = both(-s[2 * r + 1] * per);
                Row x;
#pragma unroll
                for (int p = 0; p < P; ++p) x.set(p, mul2(fma2(xh[r][p], c2, add2(y[r][p], c1)), both(rstd[r])));
                x.template store<WHOLE>(out + r * a.ld_out, place);
            }
        }
    };
    if (EXACT || (LOOSE && place.whole())) work(std::true_type{});
    else work(std::false_type{});
    if (!a.d_weight && !a.d_bias) return;
    ln_arrived<0>();
    for (int which = 0; which < 2; ++which) {
        void *const final = which ? a.d_bias : a.d_weight;
        __syncthreads();
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const float2 v = which ? db[p] : dw[p];
            joined[2 * p * blockDim.x + threadIdx.x] = v.x;
            joined[(2 * p + 1) * blockDim.x + threadIdx.x] = v.y;
        }
        __syncthreads();
        // column c of a group: vector c / V, of a warp's (or of the fewer threads') its `in`-th, of a thread its in / apart-th
        for (int c = threadIdx.x; c < dim; c += blockDim.x) {
            const int apart = place.apart(), warp = c / (apart * N * V), in = c / V - warp * apart * N, i = in / apart;
            const float *const of = joined + (i * V + c % V) * blockDim.x + warp * apart + (in - i * apart);
            float s = 0.f;
            for (int k = 0; k < groups; ++k) s += of[k * lanes];
            if (gridDim.x > 1) partial[((int64_t)blockIdx.x * 2 + which) * dim + c] = s;
            else if (!final) continue;
            else if (f32) reinterpret_cast<float *>(final)[c] = s;
            else reinterpret_cast<T *>(final)[c] = OpsType<T>::store(s);
        }
    }
}

// ---- launches --------------------------------------------------------------------------------------

// Whether all rows start on 16 bytes and are whole vectors of that size.
bool aligned(const LayerNormArgs &a) {
    const int w = qg_type_size(a.type);
    return qg_vec_bytes(a.x, a.ld_x * w, (int64_t)a.dim * w) == 16 && qg_vec_bytes(a.out, a.ld_out * w, (int64_t)a.dim * w) == 16 &&
           (!a.grad || qg_vec_bytes(a.grad, a.ld_grad * w, (int64_t)a.dim * w) == 16);
}

// Of the launches over segments: eight blocks per SM, or one for every segment of every row.
dim3 ln_segments_grid(const qgbdt_ctx *c, int64_t rows, int segments) {
    const int64_t most = ((int64_t)c->sm_count * 8 + segments - 1) / segments;
    return dim3((unsigned)segments, (unsigned)(rows < 1 ? 1 : rows < most ? rows : most));
}

// Blocks of `threads` that the GPU holds at once.
template <typename K>
int ln_resident(qgbdt_ctx *c, K kernel, int threads, size_t smem, int64_t *blocks) {
    int each = 0;
    QG_CUDA(c, cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, threads, smem));
    *blocks = (int64_t)each * c->sm_count;
    return QGBDT_OK;
}

// Leave for a launch that gives a block `smem` bytes.  It is the kernel's, for rows of all widths and for all contexts of the process, so that
// every call asks for the same: a call's own size would take from another thread what it has asked for and not yet launched with.
template <typename K>
int ln_leave(qgbdt_ctx *c, K kernel, size_t smem) {
    if (smem > LN_LEAVE) QG_CUDA(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LN_MOST));
    return QGBDT_OK;
}

template <typename T, int V, int N, bool MULTI, bool EXACT>
int rows_forward(qgbdt_ctx *c, const LayerNormArgs &a, int lanes, cudaStream_t st) {
    constexpr int R = LN_PAIR<N * V, MULTI>;
    constexpr auto kernel = k_ln_rows<T, V, N, MULTI, EXACT>;
    const int threads = MULTI ? lanes : 128, groups = threads / lanes;
    const int64_t want = (a.rows + groups * R - 1) / (groups * R);
    const size_t smem = LnAhead<T, V, N, R, LN_AHEAD<R>>::bytes(threads, lanes);
    QG_RUN(ln_leave(c, kernel, smem));
    int64_t grid = want;
    if (want > c->sm_count) {
        QG_RUN(ln_resident(c, kernel, threads, smem, &grid));
        if (want < grid) grid = want;
    }
    return qg_launch(c, kernel, dim3((unsigned)grid), threads, smem, st, a, lanes);
}

// How a row is cut up: calls `with` with N, MULTI, EXACT and the threads of a row.  Vectors: one per thread up to a warp's worth, then
// LN_EACH elements; single elements: four, eight or LN_EACH; then more warps.
template <int V, int MANY, typename F>
int rows_cut(int dim, F with) {
    constexpr int most = LN_EACH / V, many = MANY / V;
    const int vectors = (dim + V - 1) / V;
    auto choose = [&](auto n, auto multi, int lanes) {
        if constexpr (V > 1)
            if (lanes * n.value * V == dim) return with(n, multi, std::true_type{}, lanes);
        return with(n, multi, std::false_type{}, lanes);
    };
    auto few = [&](auto n) {      // of a warp's lanes
        int lanes = 1;
        while (lanes * n.value < vectors) lanes *= 2;
        return choose(n, std::false_type{}, lanes);
    };
    if constexpr (V > 1) {
        if (vectors <= 32) return few(std::integral_constant<int, 1>{});
    } else {
        if (vectors <= 32 * 4) return few(std::integral_constant<int, 4>{});
        if (vectors <= 32 * 8) return few(std::integral_constant<int, 8>{});
    }
    if (vectors <= 32 * most) return few(std::integral_constant<int, most>{});
    return choose(std::integral_constant<int, many>{}, std::true_type{}, (vectors + 32 * many - 1) / (32 * many) * 32);
}

template <typename T, int V>
int rows_forward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    return rows_cut<V, LN_MANY<T, V>>(a.dim, [&](auto n, auto multi, auto exact, int lanes) { return rows_forward<T, V, n.value, multi.value, exact.value>(c, a, lanes, st); });
}

template <typename T>
int forward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const bool vectors = aligned(a);
    constexpr int most = LN_SHARED / (LN_AHEAD<1> * (int)sizeof(T)) < LN_LONG ? LN_SHARED / (LN_AHEAD<1> * (int)sizeof(T)) / 512 * 512 : LN_LONG;
    if (a.dim <= (vectors ? most : LN_ROW)) {
        return vectors ? rows_forward<T, V>(c, a, st) : rows_forward<T, 1>(c, a, st);
    }
    const int segments = (a.dim + LN_SEGMENT - 1) / LN_SEGMENT;
    QgWorkspace ws;
    QG_RUN(qg_ws_open(c, qg_ws_size((size_t)a.rows * segments, sizeof(float2)), st, &ws));
    float2 *shares = ws.take<float2>((size_t)a.rows * segments);
    const dim3 grid = ln_segments_grid(c, a.rows, segments);
    if (vectors) {
        QG_RUN(qg_launch(c, k_ln_shares<T, V, false>, grid, LN_THREADS, 0, st, a, shares, segments));
        QG_RUN(qg_launch(c, k_ln_segments<T, V>, grid, LN_THREADS, 0, st, a, (const float2 *)shares, segments));
    } else {
        QG_RUN(qg_launch(c, k_ln_shares<T, 1, false>, grid, LN_THREADS, 0, st, a, shares, segments));
        QG_RUN(qg_launch(c, k_ln_segments<T, 1>, grid, LN_THREADS, 0, st, a, (const float2 *)shares, segments));
    }
    return qg_ws_close(c, st);
}

template <typename T, int V, int N, bool MULTI, bool EXACT>
int rows_backward(qgbdt_ctx *c, const LayerNormArgs &a, int lanes, cudaStream_t st) {
    constexpr int R = LN_PAIR<N * V, MULTI>;
    constexpr auto kernel = k_ln_rows_backward<T, V, N, MULTI, EXACT>;
    const int threads = lanes >= 256 ? lanes : 256 / lanes * lanes, groups = threads / lanes;
    const size_t sums_bytes = (size_t)threads * N * V * sizeof(float), ring = 2 * LnAhead<T, V, N, R, LN_AHEAD_BACKWARD<R>>::bytes(threads, lanes);
    const size_t smem = (size_t)lanes * N * V * sizeof(float) + (ring > sums_bytes ? ring : sums_bytes);
    QG_RUN(ln_leave(c, kernel, smem));
    // Few steps: one block, which needs no other launch to join anything.  As many blocks as there are steps up to one per
    // SM; beyond that four rows per group at least, since the partial sums are as large as one and a half.
    const int64_t steps = (a.rows + groups * R - 1) / (groups * R), fours = (a.rows + groups * 4 - 1) / (groups * 4);
    int64_t want = steps < c->sm_count ? steps : c->sm_count;
    if (want < fours) want = fours;
    if (steps <= (V > 1 ? 4 : 2)) want = 1;
    int64_t grid = want;
    if (want > c->sm_count) {
        QG_RUN(ln_resident(c, kernel, threads, smem, &grid));
        if (want < grid) grid = want;
    }
    const bool sums = a.d_weight || a.d_bias;
    if (!sums || grid == 1) return qg_launch(c, kernel, dim3((unsigned)grid), threads, smem, st, a, (float *)nullptr, lanes);
    QgWorkspace ws;
    QG_RUN(qg_ws_open(c, qg_ws_size((size_t)grid * 2 * a.dim, sizeof(float)), st, &ws));
    float *partial = ws.take<float>((size_t)grid * 2 * a.dim);
    QG_RUN(qg_launch(c, kernel, dim3((unsigned)grid), threads, smem, st, a, partial, lanes));
    QG_RUN(ln_join<T>(c, a, partial, (int)grid, st));
    return qg_ws_close(c, st);
}

template <typename T, int V>
int rows_backward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    auto cut = [&](auto n, auto multi, auto exact, int lanes) { return rows_backward<T, V, n.value, multi.value, exact.value>(c, a, lanes, st); };
    if constexpr (V == 4) {
        if (a.dim > LN_WIDE) return rows_cut<V, 8>(a.dim, cut);
    }
    return rows_cut<V, 16>(a.dim, cut);
}

template <typename T>
int backward(qgbdt_ctx *c, const LayerNormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const bool vectors = aligned(a);
    if (a.dim <= LN_ROW) {
        return vectors ? rows_backward<T, V>(c, a, st) : rows_backward<T, 1>(c, a, st);
    }
    const int segments = (a.dim + LN_SEGMENT - 1) / LN_SEGMENT;
    const bool sums = a.d_weight || a.d_bias;
    // two blocks per SM, of four rows each at least
    int64_t slices = ((int64_t)c->sm_count * 2 + segments - 1) / segments, fours = (a.rows + 3) / 4;
    if (slices > fours) slices = fours;
    if (slices < 1) slices = 1;
    QgWorkspace ws;
    QG_RUN(qg_ws_open(c, qg_ws_size((size_t)a.rows * segments, sizeof(float2)) + qg_ws_size((size_t)slices * 2 * a.dim, sizeof(float)), st, &ws));
    float2 *shares = ws.take<float2>((size_t)a.rows * segments);
    float *partial = ws.take<float>((size_t)slices * 2 * a.dim);
    const dim3 grid = ln_segments_grid(c, a.rows, segments), blocks((unsigned)segments, (unsigned)slices);
    if (a.rows > 0) {
        if (vectors) QG_RUN(qg_launch(c, k_ln_shares<T, V, true>, grid, LN_THREADS, 0, st, a, shares, segments));
        else QG_RUN(qg_launch(c, k_ln_shares<T, 1, true>, grid, LN_THREADS, 0, st, a, shares, segments));
    }
    if (vectors) QG_RUN(qg_launch(c, k_ln_segments_backward<T, V>, blocks, LN_THREADS, 0, st, a, (const float2 *)shares, sums ? partial : (float *)nullptr, segments));
    else QG_RUN(qg_launch(c, k_ln_segments_backward<T, 1>, blocks, LN_THREADS, 0, st, a, (const float2 *)shares, sums ? partial : (float *)nullptr, segments));
    if (sums) QG_RUN(ln_join<T>(c, a, partial, (int)slices, st));
    return qg_ws_close(c, st);
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
