// An AdamW step over many tensors, with states in 32 bits or in 8.
//
//   g = grad * coef;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) + eps)
//
// A tensor is cut into blocks of 256 elements from its start, which is what shares exponents where states have 8
// bits; a warp works on one of them at a time.
#include <cmath>

#include "ops_internal.cuh"

namespace {

constexpr int AW_THREADS = 256;
constexpr int AW_BLOCK = 256;                    // elements that share exponents: 8 per lane
constexpr int AW_WARPS = AW_THREADS / 32;
constexpr int AW_SMALL = 32, AW_LARGE = 400;     // tensors per launch (parameters of 2.3 or 28 KB)
constexpr int AW_CODES_M = 897, AW_CODES_V = 769;

// Types in `what`: bits 0-1 parameter, 2-3 gradient, 4-5 copy; bit 6: vectors.
template <int CAP>
struct AdamwTable {
    void *param[CAP];
    const void *grad[CAP];
    void *m[CAP], *v[CAP];
    uint8_t *exponents[CAP];
    void *copy[CAP];
    long long count[CAP];     // elements | what << 48
    unsigned first[CAP];      // first block of 256 of this launch
    int n;
    unsigned blocks;
    unsigned number;          // of the launch's first block within the call
};

struct AdamwFactors {         // the same for all elements
    double lr, beta1, beta2, eps, decay, max_norm, loss_scale;   // max_norm: times loss_scale
    long long step;
    unsigned key;
    const float *d_lr;
    const long long *d_step;
    const float *d_norm;
};

struct AdamwScalars {
    float coef, b1, c1, b2, c2, eps, keep, size, root;   // p = p * keep - size * m / (sqrt(v) * root + eps)
    unsigned key;
    bool skip;
};

__host__ __device__ __forceinline__ unsigned aw_mix(unsigned x) {
    x ^= x >> 16;
    x *= 0x9E3779B9u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

__device__ __forceinline__ AdamwScalars aw_scalars(const AdamwFactors &f) {
    AdamwScalars s;
    s.skip = false;
    double coef = 1.0;
    if (f.d_norm) {
        const float norm = *f.d_norm;
        s.skip = !(norm <= 3.402823466e38f);
        coef = f.max_norm / (double)norm;          // 0 / 0 (nothing to clip, nothing left to keep): 1
        if (!(coef < 1.0)) coef = 1.0;
    }
    const long long step = f.d_step ? *f.d_step : f.step;
    const double lr = f.d_lr ? (double)*f.d_lr : f.lr;
    s.coef = (float)(coef / f.loss_scale);
    s.b1 = (float)f.beta1, s.c1 = (float)(1.0 - f.beta1), s.b2 = (float)f.beta2, s.c2 = (float)(1.0 - f.beta2);
    s.eps = (float)f.eps;
    s.keep = (float)(1.0 - lr * f.decay);
    s.size = (float)(lr / (1.0 - pow(f.beta1, (double)step)));
    s.root = (float)(1.0 / sqrt(1.0 - pow(f.beta2, (double)step)));
    s.key = aw_mix(f.key ^ (unsigned)step);
    return s;
}

__device__ __forceinline__ float aw_load(const void *p, int type, int64_t i) {
    if (type == QGBDT_F32) return reinterpret_cast<const float *>(p)[i];
    if (type == QGBDT_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(reinterpret_cast<const __half *>(p)[i]);
}
__device__ __forceinline__ void aw_store(void *p, int type, int64_t i, float x) {
    if (type == QGBDT_F32) reinterpret_cast<float *>(p)[i] = x;
    else if (type == QGBDT_BF16) reinterpret_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(x);
    else reinterpret_cast<__half *>(p)[i] = __float2half_rn(x);
}

// 2^(E - 127); NaN for E = 255.
__device__ __forceinline__ float aw_power(unsigned e) { return __uint_as_float(e == 255 ? 0x7fc00000u : e ? e << 23 : 0x00400000u); }

__device__ __forceinline__ float aw_decode(unsigned code, unsigned offset, float power) {   // code without its sign
    return (code ? __uint_as_float((code + offset) << 20) : 0.f) * power;
}

// The code of y >= 0, below 2; r: 16 random bits.  From the smallest code's value on the bits below the code's are cut off
// after the random ones have been added to them; below it, it is the smallest code or zero.
template <bool KEEP>
__device__ __forceinline__ unsigned aw_encode(float y, unsigned offset, unsigned r) {
    const float least = __uint_as_float((offset + 1) << 20);
    r = (r << 4) + 8;
    const unsigned code = ((__float_as_uint(y) + r) >> 20) - offset;
    const bool one = KEEP ? y > 0.f : (float)r * (least * 0x1p-20f) < y;
    return y < least ? (one ? 1u : 0u) : code;
}

template <int CAP>
__device__ __forceinline__ int aw_find(const AdamwTable<CAP> &t, unsigned block) {
    int lo = 0, hi = t.n;   // t.first[lo] <= block < t.first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= block) lo = mid;
        else hi = mid;
    }
    return lo;
}

// One element: m, v and p are replaced.
__device__ __forceinline__ void aw_element(const AdamwScalars &s, float g, float &m, float &v, float &p) {
    g = g * s.coef;
    m = m * s.b1 + g * s.c1;
    v = v * s.b2 + (g * s.c2) * g;
    p = fmaf(p, s.keep, -(s.size * m / fmaf(sqrtf(v), s.root, s.eps)));
}

// The exponent of a block's largest magnitude (E; NaN and infinity give 255), from the lanes' largest bits.
__device__ __forceinline__ unsigned aw_exponent(unsigned bits) { return __reduce_max_sync(0xffffffffu, bits) >> 23; }
// 2^(127 - E) for E < 255.
__device__ __forceinline__ float aw_inverse(unsigned e) { return __uint_as_float(e == 254 ? 0x00400000u : (254 - e) << 23); }

template <int CAP, bool PACKED>
__global__ void __launch_bounds__(AW_THREADS) k_adamw(const __grid_constant__ AdamwTable<CAP> t, const AdamwFactors f) {
    qg_after_prior();
    __shared__ AdamwScalars scalars;
    if (threadIdx.x == 0) scalars = aw_scalars(f);
    __syncthreads();
    const AdamwScalars s = scalars;
    if (s.skip) return;
    const int lane = threadIdx.x & 31;
    const unsigned block = blockIdx.x * AW_WARPS + (threadIdx.x >> 5);
    if (block >= t.blocks) return;
    const int i = aw_find(t, block);
    const int what = (int)(t.count[i] >> 48), param_type = what & 3, grad_type = what >> 2 & 3, copy_type = what >> 4 & 3;
    const int64_t base = (int64_t)(block - t.first[i]) * AW_BLOCK, left = (t.count[i] & ((1ll << 48) - 1)) - base;
    const int n = left < AW_BLOCK ? (int)left : AW_BLOCK;
    constexpr int E = AW_BLOCK / 32;
    float m[E], v[E];
    unsigned exponents[2] = {0, 0}, top[2] = {0, 0};
    if constexpr (PACKED) exponents[0] = t.exponents[i][base / AW_BLOCK * 2], exponents[1] = t.exponents[i][base / AW_BLOCK * 2 + 1];
    const float power[2] = {aw_power(exponents[0]), aw_power(exponents[1])};
#pragma unroll
    for (int k = 0; k < E; ++k) {
        const int j = lane + k * 32;
        m[k] = v[k] = 0.f;
        if (j >= n) continue;
        const int64_t at = base + j;
        if constexpr (PACKED) {
            const unsigned cm = reinterpret_cast<const uint8_t *>(t.m[i])[at], cv = reinterpret_cast<const uint8_t *>(t.v[i])[at];
            m[k] = aw_decode(cm & 127, AW_CODES_M, power[0]);
            if (cm > 127) m[k] = -m[k];
            v[k] = aw_decode(cv, AW_CODES_V, power[1]);
        } else {
            m[k] = reinterpret_cast<const float *>(t.m[i])[at], v[k] = reinterpret_cast<const float *>(t.v[i])[at];
        }
        float p = aw_load(t.param[i], param_type, at);
        aw_element(s, aw_load(t.grad[i], grad_type, at), m[k], v[k], p);
        aw_store(t.param[i], param_type, at, p);
        if (t.copy[i]) aw_store(t.copy[i], copy_type, at, p);
        if constexpr (PACKED) {
            top[0] = max(top[0], __float_as_uint(fabsf(m[k])));
            top[1] = max(top[1], __float_as_uint(fabsf(v[k])));
        } else {
            reinterpret_cast<float *>(t.m[i])[at] = m[k], reinterpret_cast<float *>(t.v[i])[at] = v[k];
        }
    }
    if constexpr (PACKED) {
        const unsigned key = aw_mix(s.key ^ (t.number + block));
        const unsigned e0 = aw_exponent(top[0]), e1 = aw_exponent(top[1]);
        const float inverse[2] = {aw_inverse(e0), aw_inverse(e1)};
        if (lane == 0) t.exponents[i][base / AW_BLOCK * 2] = (uint8_t)e0, t.exponents[i][base / AW_BLOCK * 2 + 1] = (uint8_t)e1;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const int j = lane + k * 32;
            if (j >= n) continue;
            const unsigned r = aw_mix(key ^ (unsigned)j);
            unsigned cm = 0, cv = 0;
            if (e0 < 255) {
                cm = aw_encode<false>(fabsf(m[k]) * inverse[0], AW_CODES_M, r >> 16);
                if (cm && m[k] < 0.f) cm |= 128;
            }
            if (e1 < 255) cv = aw_encode<true>(v[k] * inverse[1], AW_CODES_V, r & 0xffffu);
            reinterpret_cast<uint8_t *>(t.m[i])[base + j] = (uint8_t)cm;
            reinterpret_cast<uint8_t *>(t.v[i])[base + j] = (uint8_t)cv;
        }
    }
}

// What packed states stand for.  Of the table: m, v and exponents as above, param and copy for the values of m and v.
template <int CAP>
__global__ void __launch_bounds__(AW_THREADS) k_adamw_values(const __grid_constant__ AdamwTable<CAP> t) {
    qg_after_prior();
    const int lane = threadIdx.x & 31;
    const unsigned block = blockIdx.x * AW_WARPS + (threadIdx.x >> 5);
    if (block >= t.blocks) return;
    const int i = aw_find(t, block);
    const int type = (int)(t.count[i] >> 48) & 3;
    const int64_t base = (int64_t)(block - t.first[i]) * AW_BLOCK, left = (t.count[i] & ((1ll << 48) - 1)) - base;
    const int n = left < AW_BLOCK ? (int)left : AW_BLOCK;
    const float power[2] = {aw_power(t.exponents[i][base / AW_BLOCK * 2]), aw_power(t.exponents[i][base / AW_BLOCK * 2 + 1])};
    for (int j = lane; j < n; j += 32) {
        const int64_t at = base + j;
        const unsigned cm = reinterpret_cast<const uint8_t *>(t.m[i])[at], cv = reinterpret_cast<const uint8_t *>(t.v[i])[at];
        const float m = aw_decode(cm & 127, AW_CODES_M, power[0]);
        aw_store(t.param[i], type, at, cm > 127 ? -m : m);
        aw_store(t.copy[i], type, at, aw_decode(cv, AW_CODES_V, power[1]));
    }
}

// Takes tensors from `at` on into the table, as many as it holds (a large tensor in parts).  `fill` gives tensor i: false if
// it has no elements.
template <int CAP, typename F>
void aw_fill(AdamwTable<CAP> &t, int32_t &at, int64_t &done, int32_t n, unsigned &number, F fill) {
    constexpr int64_t most = 1ll << 30;   // blocks of a launch
    t.n = 0, t.blocks = 0, t.number = number;
    while (at < n && t.n < CAP && t.blocks < most) {
        const int64_t count = fill(t, t.n, at, done);
        if (count > 0) {
            const int64_t blocks = (count + AW_BLOCK - 1) / AW_BLOCK, room = most - t.blocks, here = blocks < room ? blocks : room;
            t.count[t.n] |= here < blocks ? here * AW_BLOCK : count;
            t.first[t.n++] = t.blocks;
            t.blocks += (unsigned)here;
            done += here * AW_BLOCK;
            if (here < blocks) break;
        }
        ++at, done = 0;
    }
    number += t.blocks;
}

template <int CAP, bool PACKED>
int aw_run(qgbdt_ctx *c, const qgbdt_adamw_tensor *in, int32_t n, const AdamwFactors &f, cudaStream_t st) {
    AdamwTable<CAP> t;
    int32_t at = 0;
    int64_t done = 0;
    unsigned number = 0;
    while (at < n) {
        aw_fill(t, at, done, n, number, [in](AdamwTable<CAP> &t, int k, int32_t i, int64_t from) -> int64_t {
            const qgbdt_adamw_tensor &a = in[i];
            const int64_t state = PACKED ? 1 : 4;
            auto moved = [from](const void *p, int64_t width) { return const_cast<char *>(reinterpret_cast<const char *>(p)) + from * width; };
            t.param[k] = moved(a.param, qg_type_size(a.param_type));
            t.grad[k] = moved(a.grad, qg_type_size(a.grad_type));
            t.m[k] = moved(a.exp_avg, state), t.v[k] = moved(a.exp_avg_sq, state);
            t.exponents[k] = PACKED ? a.exponents + from / AW_BLOCK * 2 : nullptr;
            t.copy[k] = a.copy ? moved(a.copy, qg_type_size(a.copy_type)) : nullptr;
            t.count[k] = (long long)(a.param_type | a.grad_type << 2 | (a.copy ? a.copy_type : 0) << 4) << 48;
            return a.count - from;
        });
        if (t.blocks) QG_RUN(qg_launch(c, k_adamw<CAP, PACKED>, dim3((t.blocks + AW_WARPS - 1) / AW_WARPS), AW_THREADS, 0, st, t, f));
    }
    return QGBDT_OK;
}

template <int CAP>
int aw_values(qgbdt_ctx *c, const uint8_t *const *m, const uint8_t *const *v, const uint8_t *const *exponents, void *const *out_m, void *const *out_v,
              const int64_t *counts, int32_t n, int32_t type, cudaStream_t st) {
    AdamwTable<CAP> t;
    int32_t at = 0;
    int64_t done = 0;
    unsigned number = 0;
    while (at < n) {
        aw_fill(t, at, done, n, number, [&](AdamwTable<CAP> &t, int k, int32_t i, int64_t from) -> int64_t {
            const int w = qg_type_size(type);
            t.m[k] = const_cast<uint8_t *>(m[i]) + from, t.v[k] = const_cast<uint8_t *>(v[i]) + from;
            t.exponents[k] = const_cast<uint8_t *>(exponents[i]) + from / AW_BLOCK * 2;
            t.param[k] = reinterpret_cast<char *>(out_m[i]) + from * w, t.copy[k] = reinterpret_cast<char *>(out_v[i]) + from * w;
            t.count[k] = (long long)type << 48;
            return counts[i] - from;
        });
        if (t.blocks) QG_RUN(qg_launch(c, k_adamw_values<CAP>, dim3((t.blocks + AW_WARPS - 1) / AW_WARPS), AW_THREADS, 0, st, t));
    }
    return QGBDT_OK;
}

}  // namespace

int qg_adamw(qgbdt_ctx *c, const qgbdt_adamw_tensor *t, int32_t n, const qgbdt_adamw_options &o, cudaStream_t st) {
    AdamwFactors f;
    f.lr = o.lr, f.beta1 = o.beta1, f.beta2 = o.beta2, f.eps = o.eps, f.decay = o.weight_decay, f.max_norm = o.max_norm * o.loss_scale;
    f.loss_scale = o.loss_scale, f.step = o.step;
    f.key = aw_mix(aw_mix((unsigned)o.seed) ^ (unsigned)(o.seed >> 32));
    f.d_lr = o.d_lr, f.d_step = reinterpret_cast<const long long *>(o.d_step), f.d_norm = o.d_norm;
    if (o.state_bits == 8) return n <= AW_SMALL ? aw_run<AW_SMALL, true>(c, t, n, f, st) : aw_run<AW_LARGE, true>(c, t, n, f, st);
    return n <= AW_SMALL ? aw_run<AW_SMALL, false>(c, t, n, f, st) : aw_run<AW_LARGE, false>(c, t, n, f, st);
}

int qg_adamw_values(qgbdt_ctx *c, const uint8_t *const *m, const uint8_t *const *v, const uint8_t *const *exponents, void *const *out_m,
                    void *const *out_v, const int64_t *counts, int32_t n, int32_t type, cudaStream_t st) {
    return n <= AW_SMALL ? aw_values<AW_SMALL>(c, m, v, exponents, out_m, out_v, counts, n, type, st)
                         : aw_values<AW_LARGE>(c, m, v, exponents, out_m, out_v, counts, n, type, st);
}
