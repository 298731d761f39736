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

struct AdamwScalars {
    float coef, b1, c1, b2, c2, eps, keep, size, root;   // p = p * keep - size * m / (sqrt(v) * root + eps)
    unsigned key;
};

// The same for all elements: worked out on the host, but for what depends on numbers in device memory.
struct AdamwFactors {
    AdamwScalars s;
    double lr, beta1, beta2, decay, max_norm, loss_scale;   // max_norm: times loss_scale
    long long step;
    unsigned seed;             // hashed
    const float *d_lr;
    const long long *d_step;
    const float *d_norm;
};

__host__ __device__ __forceinline__ unsigned aw_mix(unsigned x) {
    x ^= x >> 16;
    x *= 0x9E3779B9u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

__host__ __device__ inline void aw_of_step(AdamwScalars &s, const AdamwFactors &f, double lr, long long step) {
    s.keep = (float)(1.0 - lr * f.decay);
    s.size = (float)(lr / (1.0 - pow(f.beta1, (double)step)));
    s.root = (float)(1.0 / sqrt(1.0 - pow(f.beta2, (double)step)));
    s.key = aw_mix(f.seed ^ (unsigned)step);
}

// One thread's work, for the block; false: the gradients' norm is not finite.
__device__ __noinline__ bool aw_scalars(const AdamwFactors &f, AdamwScalars &s) {
    bool fine = true;
    if (f.d_norm) {
        const float norm = *f.d_norm;
        fine = norm <= 3.402823466e38f;
        double coef = f.max_norm / (double)norm;
        if (!(coef < 1.0)) coef = 1.0;             // 0 / 0 too: nothing to clip
        s.coef = (float)(coef / f.loss_scale);
    }
    if (f.d_lr || f.d_step) aw_of_step(s, f, f.d_lr ? (double)*f.d_lr : f.lr, f.d_step ? *f.d_step : f.step);
    return fine;
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

// One element: m, v and p are replaced.  m and v in operations that are rounded one by one (what is rounded to 8 bits
// afterwards then has the bits of the formula written out); the root and the quotient by the approximations of the
// special function unit, 2^-22 of the change off at most: with the exact ones the update has half as many instructions again.
__device__ __forceinline__ void aw_element(const AdamwScalars &s, float g, float &m, float &v, float &p) {
    g = g * s.coef;
    m = m * s.b1 + g * s.c1;
    v = v * s.b2 + (g * s.c2) * g;
    float root;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
    p = fmaf(p, s.keep, -s.size * __fdividef(m, fmaf(root, s.root, s.eps)));
}

// The exponent of a block's largest magnitude (E; NaN and infinity give 255), from the lanes' largest bits.
__device__ __forceinline__ unsigned aw_exponent(unsigned bits) { return __reduce_max_sync(0xffffffffu, bits) >> 23; }
// 2^(127 - E) for E < 255.
__device__ __forceinline__ float aw_inverse(unsigned e) { return __uint_as_float(e == 254 ? 0x00400000u : (254 - e) << 23); }

// Eight neighbouring elements of a lane: 32 bytes in one access where they have 4 each, 16 or 8 else.
constexpr int AW_EACH = AW_BLOCK / 32;
struct AwRaw {
    unsigned x[8];
};
__device__ __forceinline__ void aw_read32(AwRaw &r, const void *p) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r.x[0]), "=r"(r.x[1]), "=r"(r.x[2]), "=r"(r.x[3]), "=r"(r.x[4]), "=r"(r.x[5]), "=r"(r.x[6]), "=r"(r.x[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void aw_write32(void *p, const AwRaw &r) {
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r.x[0]), "r"(r.x[1]), "r"(r.x[2]), "r"(r.x[3]), "r"(r.x[4]),
                 "r"(r.x[5]), "r"(r.x[6]), "r"(r.x[7]), "l"(p)
                 : "memory");
}
__device__ __forceinline__ void aw_read(AwRaw &r, const void *p, int type, int64_t at) {
    if (type == QGBDT_F32) {
        aw_read32(r, reinterpret_cast<const float *>(p) + at);
    } else {
        const uint4 q = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(p) + at);
        r.x[0] = q.x, r.x[1] = q.y, r.x[2] = q.z, r.x[3] = q.w;
    }
}
__device__ __forceinline__ void aw_unpack(float (&f)[8], const AwRaw &r, int type) {
    if (type == QGBDT_F32) {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = __uint_as_float(r.x[k]);
    } else if (type == QGBDT_BF16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) f[2 * k] = __uint_as_float(r.x[k] << 16), f[2 * k + 1] = __uint_as_float(r.x[k] & 0xffff0000u);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 two = __half22float2(*reinterpret_cast<const __half2 *>(&r.x[k]));
            f[2 * k] = two.x, f[2 * k + 1] = two.y;
        }
    }
}
__device__ __forceinline__ void aw_write(void *p, int type, int64_t at, const float (&f)[8]) {
    AwRaw r;
    if (type == QGBDT_F32) {
#pragma unroll
        for (int k = 0; k < 8; ++k) r.x[k] = __float_as_uint(f[k]);
        aw_write32(reinterpret_cast<float *>(p) + at, r);
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (type == QGBDT_BF16) *reinterpret_cast<__nv_bfloat162 *>(&r.x[k]) = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
        else *reinterpret_cast<__half2 *>(&r.x[k]) = __floats2half2_rn(f[2 * k], f[2 * k + 1]);
    }
    *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(p) + at) = make_uint4(r.x[0], r.x[1], r.x[2], r.x[3]);
}

// A warp takes `per` neighbouring blocks of 256 at a time.  Where addresses allow it and the block is whole, a lane has eight
// neighbouring elements, else every 32nd.
template <int CAP, bool PACKED>
__global__ void __launch_bounds__(AW_THREADS) k_adamw(const __grid_constant__ AdamwTable<CAP> t, const __grid_constant__ AdamwFactors f, int per) {
    qg_after_prior();
    __shared__ AdamwScalars scalars;
    __shared__ bool fine;
    if (f.d_norm || f.d_lr || f.d_step) {
        if (threadIdx.x == 0) scalars = f.s, fine = aw_scalars(f, scalars);
        __syncthreads();
        if (!fine) return;
    } else {
        if (threadIdx.x == 0) scalars = f.s;
        __syncthreads();
    }
    const AdamwScalars s = scalars;
    const int lane = threadIdx.x & 31;
    for (unsigned unit = blockIdx.x * AW_WARPS + (threadIdx.x >> 5); unit * (unsigned)per < t.blocks; unit += gridDim.x * AW_WARPS) {
        unsigned block = unit * per;
        const unsigned end = min(t.blocks, block + per);
        int i = aw_find(t, block);
        for (; block < end; ++block) {
            while (i + 1 < t.n && t.first[i + 1] <= block) ++i;
            const int what = (int)(t.count[i] >> 48), param_type = what & 3, grad_type = what >> 2 & 3, copy_type = what >> 4 & 3;
            const int64_t base = (int64_t)(block - t.first[i]) * AW_BLOCK, left = (t.count[i] & ((1ll << 48) - 1)) - base;
            const int n = left < AW_BLOCK ? (int)left : AW_BLOCK;
            const bool vectors = (what & 64) && n == AW_BLOCK;
            const int64_t at = base + (vectors ? lane * AW_EACH : lane);
            void *const param = t.param[i], *const copy = t.copy[i], *const pm = t.m[i], *const pv = t.v[i];
            uint8_t *const exponents = t.exponents[i] + base / AW_BLOCK * 2;
            float p[AW_EACH], g[AW_EACH], m[AW_EACH], v[AW_EACH];
            uint2 codes[2] = {};
            float power[2] = {};
            if constexpr (PACKED) power[0] = aw_power(exponents[0]), power[1] = aw_power(exponents[1]);
            if (vectors) {
                AwRaw rp, rg, rm, rv;
                aw_read(rp, param, param_type, at);
                aw_read(rg, t.grad[i], grad_type, at);
                if constexpr (PACKED) {
                    codes[0] = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(pm) + at);
                    codes[1] = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(pv) + at);
                } else {
                    aw_read32(rm, reinterpret_cast<const float *>(pm) + at);
                    aw_read32(rv, reinterpret_cast<const float *>(pv) + at);
                    aw_unpack(m, rm, QGBDT_F32);
                    aw_unpack(v, rv, QGBDT_F32);
                }
                aw_unpack(p, rp, param_type);
                aw_unpack(g, rg, grad_type);
            } else {
#pragma unroll
                for (int k = 0; k < AW_EACH; ++k) {
                    p[k] = g[k] = m[k] = v[k] = 0.f;
                    if (lane + 32 * k >= n) continue;
                    p[k] = aw_load(param, param_type, at + 32 * k);
                    g[k] = aw_load(t.grad[i], grad_type, at + 32 * k);
                    if constexpr (PACKED) {
                        (k < 4 ? codes[0].x : codes[0].y) |= (unsigned)reinterpret_cast<const uint8_t *>(pm)[at + 32 * k] << (k & 3) * 8;
                        (k < 4 ? codes[1].x : codes[1].y) |= (unsigned)reinterpret_cast<const uint8_t *>(pv)[at + 32 * k] << (k & 3) * 8;
                    } else {
                        m[k] = reinterpret_cast<const float *>(pm)[at + 32 * k];
                        v[k] = reinterpret_cast<const float *>(pv)[at + 32 * k];
                    }
                }
            }
            unsigned top[2] = {0, 0};
#pragma unroll
            for (int k = 0; k < AW_EACH; ++k) {
                if constexpr (PACKED) {
                    const unsigned cm = (k < 4 ? codes[0].x : codes[0].y) >> (k & 3) * 8, cv = (k < 4 ? codes[1].x : codes[1].y) >> (k & 3) * 8 & 255;
                    m[k] = aw_decode(cm & 127, AW_CODES_M, power[0]);
                    m[k] = __uint_as_float(__float_as_uint(m[k]) | (cm & 128) << 24);
                    v[k] = aw_decode(cv, AW_CODES_V, power[1]);
                }
                aw_element(s, g[k], m[k], v[k], p[k]);
                if constexpr (PACKED) {
                    top[0] = max(top[0], __float_as_uint(fabsf(m[k])));
                    top[1] = max(top[1], __float_as_uint(fabsf(v[k])));
                }
            }
            if constexpr (PACKED) {
                const unsigned key = aw_mix(s.key ^ (t.number + block));
                const unsigned e[2] = {aw_exponent(top[0]), aw_exponent(top[1])};
                const float inverse[2] = {aw_inverse(e[0]), aw_inverse(e[1])};
                codes[0] = codes[1] = make_uint2(0, 0);
#pragma unroll
                for (int k = 0; k < AW_EACH; ++k) {
                    const unsigned r = aw_mix(key ^ (unsigned)(vectors ? lane * AW_EACH + k : lane + 32 * k));
                    unsigned cm = aw_encode<false>(fabsf(m[k]) * inverse[0], AW_CODES_M, r >> 16);
                    if (cm && m[k] < 0.f) cm |= 128;
                    const unsigned cv = aw_encode<true>(v[k] * inverse[1], AW_CODES_V, r & 0xffffu);
                    (k < 4 ? codes[0].x : codes[0].y) |= cm << (k & 3) * 8;
                    (k < 4 ? codes[1].x : codes[1].y) |= cv << (k & 3) * 8;
                }
                if (e[0] == 255) codes[0] = make_uint2(0, 0);
                if (e[1] == 255) codes[1] = make_uint2(0, 0);
                if (lane == 0) exponents[0] = (uint8_t)e[0], exponents[1] = (uint8_t)e[1];
            }
            if (vectors) {
                aw_write(param, param_type, at, p);
                if (copy) aw_write(copy, copy_type, at, p);
                if constexpr (PACKED) {
                    *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(pm) + at) = codes[0];
                    *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(pv) + at) = codes[1];
                } else {
                    aw_write(pm, QGBDT_F32, at, m);
                    aw_write(pv, QGBDT_F32, at, v);
                }
            } else {
#pragma unroll
                for (int k = 0; k < AW_EACH; ++k) {
                    if (lane + 32 * k >= n) continue;
                    aw_store(param, param_type, at + 32 * k, p[k]);
                    if (copy) aw_store(copy, copy_type, at + 32 * k, p[k]);
                    if constexpr (PACKED) {
                        reinterpret_cast<uint8_t *>(pm)[at + 32 * k] = (uint8_t)((k < 4 ? codes[0].x : codes[0].y) >> (k & 3) * 8);
                        reinterpret_cast<uint8_t *>(pv)[at + 32 * k] = (uint8_t)((k < 4 ? codes[1].x : codes[1].y) >> (k & 3) * 8);
                    } else {
                        reinterpret_cast<float *>(pm)[at + 32 * k] = m[k];
                        reinterpret_cast<float *>(pv)[at + 32 * k] = v[k];
                    }
                }
            }
        }
    }
}

// What packed states stand for.  Of the table: m, v and exponents as above, param and copy for the values of m and v.
template <int CAP>
__global__ void __launch_bounds__(AW_THREADS) k_adamw_values(const __grid_constant__ AdamwTable<CAP> t, int per) {
    qg_after_prior();
    const int lane = threadIdx.x & 31;
    for (unsigned unit = blockIdx.x * AW_WARPS + (threadIdx.x >> 5); unit * (unsigned)per < t.blocks; unit += gridDim.x * AW_WARPS) {
        unsigned block = unit * per;
        const unsigned end = min(t.blocks, block + per);
        int i = aw_find(t, block);
        for (; block < end; ++block) {
            while (i + 1 < t.n && t.first[i + 1] <= block) ++i;
            const int what = (int)(t.count[i] >> 48), type = what & 3;
            const int64_t base = (int64_t)(block - t.first[i]) * AW_BLOCK, left = (t.count[i] & ((1ll << 48) - 1)) - base;
            const int n = left < AW_BLOCK ? (int)left : AW_BLOCK;
            const uint8_t *const pm = reinterpret_cast<const uint8_t *>(t.m[i]), *const pv = reinterpret_cast<const uint8_t *>(t.v[i]);
            const float power[2] = {aw_power(t.exponents[i][base / AW_BLOCK * 2]), aw_power(t.exponents[i][base / AW_BLOCK * 2 + 1])};
            if ((what & 64) && n == AW_BLOCK) {
                const int64_t at = base + lane * AW_EACH;
                const uint2 cm = *reinterpret_cast<const uint2 *>(pm + at), cv = *reinterpret_cast<const uint2 *>(pv + at);
                float m[AW_EACH], v[AW_EACH];
#pragma unroll
                for (int k = 0; k < AW_EACH; ++k) {
                    const unsigned one = (k < 4 ? cm.x : cm.y) >> (k & 3) * 8;
                    m[k] = aw_decode(one & 127, AW_CODES_M, power[0]);
                    m[k] = __uint_as_float(__float_as_uint(m[k]) | (one & 128) << 24);
                    v[k] = aw_decode((k < 4 ? cv.x : cv.y) >> (k & 3) * 8 & 255, AW_CODES_V, power[1]);
                }
                aw_write(t.param[i], type, at, m);
                aw_write(t.copy[i], type, at, v);
            } else {
                for (int j = lane; j < n; j += 32) {
                    const unsigned one = pm[base + j];
                    const float m = aw_decode(one & 127, AW_CODES_M, power[0]);
                    aw_store(t.param[i], type, base + j, __uint_as_float(__float_as_uint(m) | (one & 128) << 24));
                    aw_store(t.copy[i], type, base + j, aw_decode(pv[base + j], AW_CODES_V, power[1]));
                }
            }
        }
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

// Whether lanes may read and write eight neighbouring elements of `width` bytes at once.
bool aw_whole(const void *p, int64_t width) { return qg_aligned(p, (int)(8 * width)); }

// Blocks of 256 that a warp takes at a time (it looks for its tensor once for all of them): four where every warp of the GPU has
// that many, one else.  And the grid: what fits on the GPU at once, so that the work in front of the first block is done once.
template <typename K>
int aw_grid(qgbdt_ctx *c, K kernel, unsigned blocks, int *per, unsigned *grid) {
    *per = 1;
    *grid = (blocks + AW_WARPS - 1) / AW_WARPS;
    if (*grid <= (unsigned)c->sm_count) return QGBDT_OK;
    int each = 0;
    QG_CUDA(c, cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, AW_THREADS, 0));
    const unsigned most = (unsigned)(each * c->sm_count);
    *per = blocks >= most * AW_WARPS * 4 ? 4 : 1;
    const unsigned want = (blocks + AW_WARPS * *per - 1) / (AW_WARPS * *per);
    *grid = want < most ? want : most;
    return QGBDT_OK;
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
            const bool vectors = aw_whole(t.param[k], qg_type_size(a.param_type)) && aw_whole(t.grad[k], qg_type_size(a.grad_type)) && aw_whole(t.m[k], state) &&
                                 aw_whole(t.v[k], state) && (!a.copy || aw_whole(t.copy[k], qg_type_size(a.copy_type)));
            t.count[k] = (long long)(a.param_type | a.grad_type << 2 | (a.copy ? a.copy_type : 0) << 4 | (vectors ? 64 : 0)) << 48;
            return a.count - from;
        });
        if (t.blocks == 0) continue;
        int per;
        unsigned grid;
        QG_RUN(aw_grid(c, k_adamw<CAP, PACKED>, t.blocks, &per, &grid));
        QG_RUN(qg_launch(c, k_adamw<CAP, PACKED>, dim3(grid), AW_THREADS, 0, st, t, f, per));
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
            const bool vectors = aw_whole(t.param[k], w) && aw_whole(t.copy[k], w) && aw_whole(t.m[k], 1) && aw_whole(t.v[k], 1);
            t.count[k] = (long long)(type | (vectors ? 64 : 0)) << 48;
            return counts[i] - from;
        });
        if (t.blocks == 0) continue;
        int per;
        unsigned grid;
        QG_RUN(aw_grid(c, k_adamw_values<CAP>, t.blocks, &per, &grid));
        QG_RUN(qg_launch(c, k_adamw_values<CAP>, dim3(grid), AW_THREADS, 0, st, t, per));
    }
    return QGBDT_OK;
}

}  // namespace

int qg_adamw(qgbdt_ctx *c, const qgbdt_adamw_tensor *t, int32_t n, const qgbdt_adamw_options &o, cudaStream_t st) {
    AdamwFactors f;
    f.lr = o.lr, f.beta1 = o.beta1, f.beta2 = o.beta2, f.decay = o.weight_decay, f.max_norm = o.max_norm * o.loss_scale;
    f.loss_scale = o.loss_scale, f.step = o.step;
    f.seed = aw_mix(aw_mix((unsigned)o.seed) ^ (unsigned)(o.seed >> 32));
    f.d_lr = o.d_lr, f.d_step = reinterpret_cast<const long long *>(o.d_step), f.d_norm = o.d_norm;
    f.s.coef = (float)(1.0 / o.loss_scale), f.s.eps = (float)o.eps;
    f.s.b1 = (float)o.beta1, f.s.c1 = (float)(1.0 - o.beta1), f.s.b2 = (float)o.beta2, f.s.c2 = (float)(1.0 - o.beta2);
    aw_of_step(f.s, f, o.d_lr ? 0.0 : o.lr, o.d_step ? 1 : o.step);
    if (o.state_bits == 8) return n <= AW_SMALL ? aw_run<AW_SMALL, true>(c, t, n, f, st) : aw_run<AW_LARGE, true>(c, t, n, f, st);
    return n <= AW_SMALL ? aw_run<AW_SMALL, false>(c, t, n, f, st) : aw_run<AW_LARGE, false>(c, t, n, f, st);
}

int qg_adamw_values(qgbdt_ctx *c, const uint8_t *const *m, const uint8_t *const *v, const uint8_t *const *exponents, void *const *out_m,
                    void *const *out_v, const int64_t *counts, int32_t n, int32_t type, cudaStream_t st) {
    return n <= AW_SMALL ? aw_values<AW_SMALL>(c, m, v, exponents, out_m, out_v, counts, n, type, st)
                         : aw_values<AW_LARGE>(c, m, v, exponents, out_m, out_v, counts, n, type, st);
}
