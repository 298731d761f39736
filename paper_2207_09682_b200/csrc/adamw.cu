// An AdamW step over many tensors, with states in 32 bits or in 8.
//
//   g = grad * coef;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr decay) - lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) + eps)
//
// A tensor is cut into blocks of 256 elements from its start, which is what shares exponents where states have 8
// bits; a warp works on one of them at a time.  One launch for up to 400 tensors.
//
// With states in 32 bits it is bound by memory traffic: 200 M elements with 32-bit gradients and a 16-bit copy, 6.0 GB, take
// 0.96 ms (6.2 TB/s; 19 instructions per element).  With states in 8 bits half the bytes are left and three times the
// instructions (63, 27 of them on the integer pipe): 73.7 M elements with 16-bit gradients and copies, 1.18 GB, take 0.20 ms (5.9 TB/s,
// 69 % of the issue slots); parameters in 16 bits alone, 10 bytes an element, are bound by instructions (30 M: 84 us, 3.6 TB/s; in few
// tensors 80 % of the issue slots and 67 % of the integer pipe, which warps wait for most).
#include <cmath>

#include "ops_internal.cuh"

namespace {

// Threads and resident blocks of an SM, of the update with packed and with plain states: the former waits more for its own
// instructions than for the memory and has 20 warps of 96 registers (16 of 128: 2 % slower), the latter 16 (20: 1 % slower).
template <bool PACKED>
constexpr int AW_THREADS = PACKED ? 128 : 256;
template <bool PACKED>
constexpr int AW_RESIDENT = PACKED ? 5 : 2;
constexpr int AW_BLOCK = 256;                    // elements that share exponents: 8 per lane
constexpr int AW_SMALL = 16, AW_MEDIUM = 56, AW_LARGE = 400;     // tensors per launch (parameters of 1.2, 3.9 or 27 KB)
constexpr unsigned AW_CODES_M = 897, AW_CODES_V = 769;

// A tensor.  Types in the upper bits of `count`: bits 48-49 parameter, 50-51 gradient, 52-53 copy; bit 54: vectors.  (What a warp reads
// of a tensor is neighbouring in the kernel's parameters: it comes from memory, with as many misses as there are lines.)
struct alignas(64) AdamwEntry {
    void *param;
    const void *grad;
    void *m, *v;
    uint8_t *exponents;
    void *copy;
    long long count;
};
template <int CAP>
struct AdamwTable {
    AdamwEntry entry[CAP];
    unsigned first[CAP];      // first block of 256 of this launch
    int n;
    unsigned blocks;
    unsigned number;          // of the launch's first block within the call
};

struct AdamwScalars {
    float coef, b1, c1, b2, c2, keep, root, eps;   // p = p * keep - m / (sqrt(v) * root + eps)
    unsigned key;
};

// The same for all elements: worked out on the host, but for what depends on numbers in device memory.
struct AdamwFactors {
    AdamwScalars s;
    double lr, beta1, beta2, eps, decay, max_norm, loss_scale;   // max_norm: times loss_scale
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
    const double size = lr / (1.0 - pow(f.beta1, (double)step));
    s.keep = (float)(1.0 - lr * f.decay);
    // both infinite without a rate
    s.root = (float)(1.0 / (size * sqrt(1.0 - pow(f.beta2, (double)step))));
    s.eps = size > 0.0 ? (float)(f.eps / size) : s.root;
    s.key = aw_mix(f.seed ^ (unsigned)step);
}

// The gradients' factor x.  Below single precision's normal range it would lose bits that the gradients (of norms near the other end of that
// range) have: they are then taken times 2^k, which the factors behind theirs take back.
__host__ __device__ inline void aw_of_gradients(AdamwScalars &s, const AdamwFactors &f, double x) {
    s.coef = (float)x;
    if (!(x > 0.0 && x < 0x1p-126)) return;
    const int k = x < 0x1p-190 ? 64 : -126 - ilogb(x);
    s.coef = (float)ldexp(x, k);
    s.c1 = (float)ldexp(1.0 - f.beta1, -k), s.c2 = (float)ldexp(1.0 - f.beta2, -2 * k);
}

// One thread's work, for the block; false: the gradients' norm is not finite.
__device__ __noinline__ bool aw_scalars(const AdamwFactors &f, AdamwScalars &s) {
    bool fine = true;
    if (f.d_norm) {
        const float norm = *f.d_norm;
        fine = norm <= 3.402823466e38f;
        double coef = f.max_norm / (double)norm;
        if (!(coef < 1.0)) coef = 1.0;             // 0 / 0 too: nothing to clip
        aw_of_gradients(s, f, coef / f.loss_scale);
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

// 2^(127 - E) for E < 255.
__device__ __forceinline__ float aw_inverse(unsigned e) { return __uint_as_float(e == 254 ? 0x00400000u : (254 - e) << 23); }

// What eight codes stand for, times 2^(127 - E).  Two at once, as halves of a word that hold the upper 16 bits of the values: bits
// (code + offset) << 4, or 0 for code 0.  (Integer instructions have half the rate of the others; sums and shifts are products where
// they can be.)
template <unsigned OFFSET, bool SIGNED>
__device__ __forceinline__ void aw_values_of(const uint2 &codes, float (&x)[8]) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const unsigned word = k < 4 ? codes.x : codes.y, code = SIGNED ? word & 0x7f7f7f7fu : word;
        const unsigned two = __byte_perm(code, 0, k & 2 ? 0x4342 : 0x4140);
        unsigned bits = two * 16u;
        if (SIGNED) bits += __byte_perm(word & 0x80808080u, 0, k & 2 ? 0x3424 : 0x1404);
        bits += __vminu2(two, 0x00010001u) * (OFFSET * 16u);
        x[k] = __uint_as_float(bits << 16);
        x[k + 1] = __uint_as_float(bits & 0xffff0000u);
    }
}

// Code of y (2 > y >= the smallest code's value, or the value at the place of code 0 for zero) in the uppermost byte: the bits below a
// code's, and 8 below those, are rounded by the carry of 16 random bits r << 8.  (What is above the code falls off at the top.)
template <unsigned OFFSET>
__device__ __forceinline__ unsigned aw_encode(unsigned y, unsigned r) { return y * 16u + (128u - (OFFSET << 24)) + r; }

// The uppermost bytes of four words.
__device__ __forceinline__ unsigned aw_bytes(unsigned a, unsigned b, unsigned c, unsigned d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// The code, 0 or 1, of a y below the smallest code's value; r: 16 random bits.
__device__ __forceinline__ unsigned aw_code(float y, unsigned offset, unsigned r) {
    return (float)((r << 4) + 8) * (__uint_as_float((offset + 1) << 20) * 0x1p-20f) < y ? 1u : 0u;
}

// Eight elements' states to codes; `hash`: that of the first one's place, before it is mixed; the places are 2^APART apart.
template <int APART>
__device__ __forceinline__ void aw_round(const float (&m)[8], const float (&v)[8], float inverse_m, float inverse_v, unsigned hash, uint2 (&codes)[2]) {
    constexpr unsigned zero_m = AW_CODES_M << 20, zero_v = AW_CODES_V << 20, least_m = (AW_CODES_M + 1) << 20;
    const unsigned mixed = hash ^ hash >> 16;      // aw_mix's first step, for all eight: their places differ in three bits
    unsigned cm[8], cv[8], ym[8], smallest = ~0u;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        unsigned x = (mixed ^ k << APART) * 0x9E3779B9u;
        x ^= x >> 15;
        x *= 0xBB67AE85u;
        const unsigned upper = __byte_perm(x, 0, 0x4324);    // the upper half, << 8 (the last step leaves it)
        ym[k] = __float_as_uint(fabsf(m[k]) * inverse_m);
        if (k & 1) smallest = __vimin3_u32(smallest, ym[k - 1] - 1, ym[k] - 1);
        cm[k] = aw_encode<AW_CODES_M>(max(ym[k], zero_m), upper);
        // v: above zero it is the smallest code at least, also where the product is zero
        const unsigned yv = __float_as_uint(v[k] * inverse_v);
        cv[k] = aw_encode<AW_CODES_V>(max(yv, min(__float_as_uint(v[k]), 1u) * (1u << 20) + zero_v), __byte_perm(x, 0, 0x4104) ^ upper);
    }
    if (smallest < least_m - 1) {   // rare: an m between zero and the smallest code is one of the two
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float y = fabsf(m[k]) * inverse_m;
            if (y > 0.f && y < __uint_as_float(least_m)) cm[k] = aw_code(y, AW_CODES_M, aw_mix(hash ^ k << APART) >> 16) << 24;
        }
    }
    codes[1].x = aw_bytes(cv[0], cv[1], cv[2], cv[3]);
    codes[1].y = aw_bytes(cv[4], cv[5], cv[6], cv[7]);
    auto bits = [&](int k) { return __float_as_uint(m[k]); };
    codes[0].x = aw_bytes(cm[0], cm[1], cm[2], cm[3]) | (aw_bytes(bits(0), bits(1), bits(2), bits(3)) & 0x80808080u);
    codes[0].y = aw_bytes(cm[4], cm[5], cm[6], cm[7]) | (aw_bytes(bits(4), bits(5), bits(6), bits(7)) & 0x80808080u);
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

// One element: m, v and p are replaced.  b1 and b2 come with the power of two that m and v are to be multiplied with (which
// changes no rounding).  m and v in operations that are rounded one by one (what is rounded to 8 bits afterwards then has the
// bits of the formula written out); the root and the quotient by the approximations of the special function unit, 2^-22 of the
// change off at most: exact ones would be half as many instructions again.  Below 2^-126 they take v for that: by a maximum where eps
// is too small to cover the difference (BARE), else by a sum, which goes to a pipe that has room (30 M bf16, 8 bits, with the values read
// back: 114 instead of 117 us).
template <bool BARE>
__device__ __forceinline__ void aw_element(const AdamwScalars &s, float b1, float b2, float g, float &m, float &v, float &p) {
    g = g * s.coef;
    m = m * b1 + g * s.c1;
    v = v * b2 + (g * s.c2) * g;
    float root, one;
    float x = v + 1.17549435e-38f;
    if (BARE) asm("max.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(v), "f"(1.17549435e-38f));
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root) : "f"(x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(one) : "f"(fmaf(root, s.root, s.eps)));
    p = fmaf(p, s.keep, -(m * one));
}

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
template <bool WIDE>
__device__ __forceinline__ void aw_read(AwRaw &r, const void *p, int64_t at) {
    if constexpr (WIDE) {
        aw_read32(r, reinterpret_cast<const float *>(p) + at);
    } else {
        const uint4 q = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(p) + at);
        r.x[0] = q.x, r.x[1] = q.y, r.x[2] = q.z, r.x[3] = q.w;
    }
}
template <bool WIDE>
__device__ __forceinline__ void aw_unpack(float (&f)[8], const AwRaw &r, bool bf16) {
    if constexpr (WIDE) {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = __uint_as_float(r.x[k]);
    } else if (bf16) {
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
template <bool WIDE>
__device__ __forceinline__ void aw_write(void *p, int64_t at, const float (&f)[8], bool bf16) {
    AwRaw r;
    if constexpr (WIDE) {
#pragma unroll
        for (int k = 0; k < 8; ++k) r.x[k] = __float_as_uint(f[k]);
        aw_write32(reinterpret_cast<float *>(p) + at, r);
    } else {
        if (bf16) {
#pragma unroll
            for (int k = 0; k < 4; ++k) *reinterpret_cast<__nv_bfloat162 *>(&r.x[k]) = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) *reinterpret_cast<__half2 *>(&r.x[k]) = __floats2half2_rn(f[2 * k], f[2 * k + 1]);
        }
        *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(p) + at) = make_uint4(r.x[0], r.x[1], r.x[2], r.x[3]);
    }
}

// The larger of a and two magnitudes; NaN if one is NaN.
__device__ __forceinline__ float aw_largest(float a, float b, float c) {
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Exponent E of the largest of the lanes' values (NaN and infinity: 255).
__device__ __forceinline__ unsigned aw_exponent(float largest) { return __reduce_max_sync(0xffffffffu, __float_as_uint(largest)) >> 23; }

// What a tensor's blocks have in common.
struct AwTensor {
    void *param, *copy, *m, *v;
    const void *grad;
    int param_type, grad_type, copy_type;
};

// A lane's eight neighbouring elements, as they are read.
template <bool PACKED, bool WIDE_P, bool WIDE_G>
struct AwInput {
    AwRaw p, g, m, v;    // 16-bit p and g: four words; packed m and v: two
    __device__ __forceinline__ void read(const AwTensor &t, int64_t at) {
        if constexpr (PACKED) {
            const uint2 a = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(t.m) + at);
            const uint2 b = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(t.v) + at);
            m.x[0] = a.x, m.x[1] = a.y, v.x[0] = b.x, v.x[1] = b.y;
        } else {
            aw_read32(m, reinterpret_cast<const float *>(t.m) + at);
            aw_read32(v, reinterpret_cast<const float *>(t.v) + at);
        }
        aw_read<WIDE_P>(p, t.param, at);
        aw_read<WIDE_G>(g, t.grad, at);
    }
};

// Eight elements of a lane, whose places are 2^APART apart, m and v without the powers of two of the exponents e.  Packed: m and
// v are rounded to codes, e is replaced.
template <bool PACKED, bool BARE, int APART>
__device__ __forceinline__ void aw_eight(const AdamwScalars &s, float (&p)[8], const float (&g)[8], float (&m)[8], float (&v)[8], unsigned hash, unsigned (&e)[2],
                                         uint2 (&codes)[2]) {
    const float b1 = PACKED ? s.b1 * aw_power(e[0]) : s.b1, b2 = PACKED ? s.b2 * aw_power(e[1]) : s.b2;
    float top[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < AW_EACH; ++k) {
        aw_element<BARE>(s, b1, b2, g[k], m[k], v[k], p[k]);
        if (PACKED && (k & 1)) top[0] = aw_largest(top[0], m[k - 1], m[k]), top[1] = aw_largest(top[1], v[k - 1], v[k]);
    }
    if constexpr (PACKED) {
        e[0] = aw_exponent(top[0]), e[1] = aw_exponent(top[1]);
        aw_round<APART>(m, v, aw_inverse(e[0]), aw_inverse(e[1]), hash, codes);
        if (e[0] == 255) codes[0] = make_uint2(0, 0);
        if (e[1] == 255) codes[1] = make_uint2(0, 0);
    }
}

// A whole block whose addresses allow eight neighbouring elements per lane.
template <bool PACKED, bool BARE, bool WIDE_P, bool WIDE_G>
__device__ __forceinline__ void aw_whole_block(const AwTensor &t, const AdamwScalars &s, const AwInput<PACKED, WIDE_P, WIDE_G> &in, int64_t at, unsigned hash,
                                               unsigned (&e)[2]) {
    float p[8], g[8], m[8], v[8];
    uint2 codes[2];
    if constexpr (PACKED) {
        aw_values_of<AW_CODES_M, true>(make_uint2(in.m.x[0], in.m.x[1]), m);
        aw_values_of<AW_CODES_V, false>(make_uint2(in.v.x[0], in.v.x[1]), v);
    } else {
        aw_unpack<true>(m, in.m, false);
        aw_unpack<true>(v, in.v, false);
    }
    aw_unpack<WIDE_P>(p, in.p, t.param_type == QGBDT_BF16);
    aw_unpack<WIDE_G>(g, in.g, t.grad_type == QGBDT_BF16);
    aw_eight<PACKED, BARE, 0>(s, p, g, m, v, hash, e, codes);
    aw_write<WIDE_P>(t.param, at, p, t.param_type == QGBDT_BF16);
    if (t.copy) {
        if (t.copy_type == QGBDT_F32) aw_write<true>(t.copy, at, p, false);
        else aw_write<false>(t.copy, at, p, t.copy_type == QGBDT_BF16);
    }
    if constexpr (PACKED) {
        *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(t.m) + at) = codes[0];
        *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(t.v) + at) = codes[1];
    } else {
        aw_write<true>(t.m, at, m, false);
        aw_write<true>(t.v, at, v, false);
    }
}

// Any other block, of n elements: a lane has every 32nd, from its own on.
template <bool PACKED, bool BARE>
__device__ __forceinline__ void aw_ragged_block(const AwTensor &t, const AdamwScalars &s, int64_t at, int n, unsigned hash, unsigned (&e)[2]) {
    float p[8], g[8], m[8], v[8];
    uint2 codes[2] = {};
#pragma unroll
    for (int k = 0; k < AW_EACH; ++k) {
        p[k] = g[k] = m[k] = v[k] = 0.f;
        if (32 * k >= n) continue;
        const int64_t i = at + 32 * k;
        p[k] = aw_load(t.param, t.param_type, i);
        g[k] = aw_load(t.grad, t.grad_type, i);
        if constexpr (PACKED) {
            (k < 4 ? codes[0].x : codes[0].y) |= (unsigned)reinterpret_cast<const uint8_t *>(t.m)[i] << (k & 3) * 8;
            (k < 4 ? codes[1].x : codes[1].y) |= (unsigned)reinterpret_cast<const uint8_t *>(t.v)[i] << (k & 3) * 8;
        } else {
            m[k] = reinterpret_cast<const float *>(t.m)[i], v[k] = reinterpret_cast<const float *>(t.v)[i];
        }
    }
    if constexpr (PACKED) {
        aw_values_of<AW_CODES_M, true>(codes[0], m);
        aw_values_of<AW_CODES_V, false>(codes[1], v);
    }
    aw_eight<PACKED, BARE, 5>(s, p, g, m, v, hash, e, codes);
#pragma unroll
    for (int k = 0; k < AW_EACH; ++k) {
        if (32 * k >= n) continue;
        const int64_t i = at + 32 * k;
        aw_store(t.param, t.param_type, i, p[k]);
        if (t.copy) aw_store(t.copy, t.copy_type, i, p[k]);
        if constexpr (PACKED) {
            reinterpret_cast<uint8_t *>(t.m)[i] = (uint8_t)((k < 4 ? codes[0].x : codes[0].y) >> (k & 3) * 8);
            reinterpret_cast<uint8_t *>(t.v)[i] = (uint8_t)((k < 4 ? codes[1].x : codes[1].y) >> (k & 3) * 8);
        } else {
            reinterpret_cast<float *>(t.m)[i] = m[k], reinterpret_cast<float *>(t.v)[i] = v[k];
        }
    }
}

// The first blocks of a run, the whole ones; `held`: the run's exponents, a byte per lane (replaced); `number`: of the first block.
template <bool PACKED, bool BARE, bool WIDE_P, bool WIDE_G>
__device__ __forceinline__ void aw_whole_blocks(const AwTensor &t, const AdamwScalars &s, int64_t at, int whole, unsigned number, int lane, unsigned &held) {
    at += lane * AW_EACH;
    AwInput<PACKED, WIDE_P, WIDE_G> next;
    if (PACKED) next.read(t, at);
#pragma unroll 1
    for (int k = 0; k < whole; ++k, at += AW_BLOCK) {
        unsigned e[2] = {};
        if constexpr (PACKED) {
            const unsigned key = aw_mix(s.key ^ (number + k));
            e[0] = __shfl_sync(0xffffffffu, held, 2 * k), e[1] = __shfl_sync(0xffffffffu, held, 2 * k + 1);
            const AwInput<PACKED, WIDE_P, WIDE_G> now = next;
            if (k + 1 < whole) next.read(t, at + AW_BLOCK);   // under this block's work
            aw_whole_block<PACKED, BARE, WIDE_P, WIDE_G>(t, s, now, at, key ^ (lane * AW_EACH), e);
            held = lane == 2 * k ? e[0] : lane == 2 * k + 1 ? e[1] : held;
        } else {
            next.read(t, at);   // four times the bytes in flight as it is
            aw_whole_block<PACKED, BARE, WIDE_P, WIDE_G>(t, s, next, at, 0, e);
        }
    }
}

// A warp takes `per` (AW_RUN at most) neighbouring blocks of 256 at a time.  Their exponents are read together and written
// together, a byte per lane: single ones would have warps wait for one another's sectors.
constexpr int AW_RUN = 16;

template <int CAP, bool PACKED, bool BARE>
__global__ void __launch_bounds__(AW_THREADS<PACKED>, AW_RESIDENT<PACKED>) k_adamw(const __grid_constant__ AdamwTable<CAP> t, const __grid_constant__ AdamwFactors f, int per) {
    qg_after_prior();
    __shared__ AdamwScalars scalars;
    __shared__ bool fine;
    if (threadIdx.x == 0) {
        scalars = f.s;
        fine = !(f.d_norm || f.d_lr || f.d_step) || aw_scalars(f, scalars);
    }
    __syncthreads();
    if (!fine) return;
    const AdamwScalars s = scalars;
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);   // (so that the compiler sees one for all lanes)
    constexpr int warps = AW_THREADS<PACKED> / 32;
    for (unsigned unit = blockIdx.x * warps + warp; unit * (unsigned)per < t.blocks; unit += gridDim.x * warps) {
        unsigned block = unit * per;
        const unsigned end = min(t.blocks, block + per);
        for (int i = aw_find(t, block); block < end; ++i) {
            const int run = (int)((i + 1 < t.n ? min(end, t.first[i + 1]) : end) - block);   // of this tensor's blocks
            const int what = (int)(t.entry[i].count >> 48);
            const AwTensor one{t.entry[i].param, t.entry[i].copy, t.entry[i].m, t.entry[i].v, t.entry[i].grad, what & 3, what >> 2 & 3, what >> 4 & 3};
            const int64_t at = (int64_t)(block - t.first[i]) * AW_BLOCK, count = (t.entry[i].count & ((1ll << 48) - 1)) - at;
            const int whole = !(what & 64) ? 0 : count >= (int64_t)run * AW_BLOCK ? run : (int)(count / AW_BLOCK);
            uint8_t *const exponents = t.entry[i].exponents + at / AW_BLOCK * 2 + lane;
            unsigned held = PACKED && lane < 2 * run ? *exponents : 0;
            const unsigned number = t.number + block;
            if (whole > 0) {
                if (one.param_type == QGBDT_F32) {
                    if (one.grad_type == QGBDT_F32) aw_whole_blocks<PACKED, BARE, true, true>(one, s, at, whole, number, lane, held);
                    else aw_whole_blocks<PACKED, BARE, true, false>(one, s, at, whole, number, lane, held);
                } else {
                    if (one.grad_type == QGBDT_F32) aw_whole_blocks<PACKED, BARE, false, true>(one, s, at, whole, number, lane, held);
                    else aw_whole_blocks<PACKED, BARE, false, false>(one, s, at, whole, number, lane, held);
                }
            }
#pragma unroll 1
            for (int k = whole; k < run; ++k) {
                unsigned e[2] = {};
                if constexpr (PACKED) e[0] = __shfl_sync(0xffffffffu, held, 2 * k), e[1] = __shfl_sync(0xffffffffu, held, 2 * k + 1);
                const int64_t left = count - (int64_t)k * AW_BLOCK;
                aw_ragged_block<PACKED, BARE>(one, s, at + (int64_t)k * AW_BLOCK + lane, (left < AW_BLOCK ? (int)left : AW_BLOCK) - lane, aw_mix(s.key ^ (number + k)) ^ lane, e);
                if constexpr (PACKED) held = lane == 2 * k ? e[0] : lane == 2 * k + 1 ? e[1] : held;
            }
            if (PACKED && lane < 2 * run) *exponents = (uint8_t)held;
            block += run;
        }
    }
}

// What packed states stand for.  Of the table: m, v and exponents as above, param and copy for the values of m and v.
template <int CAP>
__global__ void __launch_bounds__(AW_THREADS<false>) k_adamw_values(const __grid_constant__ AdamwTable<CAP> t, int per) {
    qg_after_prior();
    const int lane = threadIdx.x & 31;
    constexpr int warps = AW_THREADS<false> / 32;
    for (unsigned unit = blockIdx.x * warps + __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0); unit * (unsigned)per < t.blocks; unit += gridDim.x * warps) {
        unsigned block = unit * per;
        const unsigned end = min(t.blocks, block + per);
        for (int i = aw_find(t, block); block < end; ++i) {
            const int run = (int)((i + 1 < t.n ? min(end, t.first[i + 1]) : end) - block);
            const int what = (int)(t.entry[i].count >> 48), type = what & 3;
            const uint8_t *const pm = reinterpret_cast<const uint8_t *>(t.entry[i].m), *const pv = reinterpret_cast<const uint8_t *>(t.entry[i].v);
            int64_t at = (int64_t)(block - t.first[i]) * AW_BLOCK;
            const int64_t count = (t.entry[i].count & ((1ll << 48) - 1)) - at;
            const unsigned held = lane < 2 * run ? t.entry[i].exponents[at / AW_BLOCK * 2 + lane] : 0;
#pragma unroll 2
            for (int k = 0; k < run; ++k, at += AW_BLOCK) {
                const int64_t left = count - (int64_t)k * AW_BLOCK;
                const int n = left < AW_BLOCK ? (int)left : AW_BLOCK;
                const bool vectors = (what & 64) && n == AW_BLOCK;
                const int64_t mine = at + (vectors ? lane * AW_EACH : lane);
                uint2 codes[2] = {};
                float m[AW_EACH], v[AW_EACH];
                if (vectors) {
                    codes[0] = *reinterpret_cast<const uint2 *>(pm + mine), codes[1] = *reinterpret_cast<const uint2 *>(pv + mine);
                } else {
#pragma unroll
                    for (int j = 0; j < AW_EACH; ++j) {
                        if (lane + 32 * j >= n) continue;
                        (j < 4 ? codes[0].x : codes[0].y) |= (unsigned)pm[mine + 32 * j] << (j & 3) * 8;
                        (j < 4 ? codes[1].x : codes[1].y) |= (unsigned)pv[mine + 32 * j] << (j & 3) * 8;
                    }
                }
                aw_values_of<AW_CODES_M, true>(codes[0], m);
                aw_values_of<AW_CODES_V, false>(codes[1], v);
                const float power[2] = {aw_power(__shfl_sync(0xffffffffu, held, 2 * k)), aw_power(__shfl_sync(0xffffffffu, held, 2 * k + 1))};
#pragma unroll
                for (int j = 0; j < AW_EACH; ++j) m[j] *= power[0], v[j] *= power[1];
                if (vectors) {
                    if (type == QGBDT_F32) aw_write<true>(t.entry[i].param, mine, m, false), aw_write<true>(t.entry[i].copy, mine, v, false);
                    else aw_write<false>(t.entry[i].param, mine, m, true), aw_write<false>(t.entry[i].copy, mine, v, true);
                } else {
#pragma unroll
                    for (int j = 0; j < AW_EACH; ++j) {
                        if (lane + 32 * j >= n) continue;
                        aw_store(t.entry[i].param, type, mine + 32 * j, m[j]);
                        aw_store(t.entry[i].copy, type, mine + 32 * j, v[j]);
                    }
                }
            }
            block += run;
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
            t.entry[t.n].count |= here < blocks ? here * AW_BLOCK : count;
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

// The grid is what fits on the GPU at once, so that the work in front of the first block is done once.  A warp takes up to AW_RUN
// neighbouring blocks of 256 at a time, as many as let all warps end with the same number of turns.
template <typename K>
int aw_grid(qgbdt_ctx *c, K kernel, int threads, unsigned blocks, int *per, unsigned *grid) {
    const unsigned each = threads / 32;   // warps
    *per = 1;
    *grid = (blocks + each - 1) / each;
    if (*grid <= (unsigned)c->sm_count) return QGBDT_OK;
    int resident = 0;
    QG_CUDA(c, cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, threads, 0));
    const unsigned most = (unsigned)(resident * c->sm_count), warps = most * each, turns = (blocks + warps * AW_RUN - 1) / (warps * AW_RUN);
    *per = (int)((blocks + warps * turns - 1) / (warps * turns));
    const unsigned want = (blocks + each * *per - 1) / (each * *per);
    *grid = want < most ? want : most;
    return QGBDT_OK;
}

template <int CAP, bool PACKED, bool BARE>
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
            t.entry[k].param = moved(a.param, qg_type_size(a.param_type));
            t.entry[k].grad = moved(a.grad, qg_type_size(a.grad_type));
            t.entry[k].m = moved(a.exp_avg, state), t.entry[k].v = moved(a.exp_avg_sq, state);
            t.entry[k].exponents = PACKED ? a.exponents + from / AW_BLOCK * 2 : nullptr;
            t.entry[k].copy = a.copy ? moved(a.copy, qg_type_size(a.copy_type)) : nullptr;
            const bool vectors = aw_whole(t.entry[k].param, qg_type_size(a.param_type)) && aw_whole(t.entry[k].grad, qg_type_size(a.grad_type)) && aw_whole(t.entry[k].m, state) &&
                                 aw_whole(t.entry[k].v, state) && (!a.copy || aw_whole(t.entry[k].copy, qg_type_size(a.copy_type)));
            t.entry[k].count = (long long)(a.param_type | a.grad_type << 2 | (a.copy ? a.copy_type : 0) << 4 | (vectors ? 64 : 0)) << 48;
            return a.count - from;
        });
        if (t.blocks == 0) continue;
        int per;
        unsigned grid;
        QG_RUN(aw_grid(c, k_adamw<CAP, PACKED, BARE>, AW_THREADS<PACKED>, t.blocks, &per, &grid));
        QG_RUN(qg_launch(c, k_adamw<CAP, PACKED, BARE>, dim3(grid), AW_THREADS<PACKED>, 0, st, t, f, per));
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
            t.entry[k].m = const_cast<uint8_t *>(m[i]) + from, t.entry[k].v = const_cast<uint8_t *>(v[i]) + from;
            t.entry[k].exponents = const_cast<uint8_t *>(exponents[i]) + from / AW_BLOCK * 2;
            t.entry[k].param = reinterpret_cast<char *>(out_m[i]) + from * w, t.entry[k].copy = reinterpret_cast<char *>(out_v[i]) + from * w;
            const bool vectors = aw_whole(t.entry[k].param, w) && aw_whole(t.entry[k].copy, w) && aw_whole(t.entry[k].m, 1) && aw_whole(t.entry[k].v, 1);
            t.entry[k].count = (long long)(type | (vectors ? 64 : 0)) << 48;
            return counts[i] - from;
        });
        if (t.blocks == 0) continue;
        int per;
        unsigned grid;
        QG_RUN(aw_grid(c, k_adamw_values<CAP>, AW_THREADS<false>, t.blocks, &per, &grid));
        QG_RUN(qg_launch(c, k_adamw_values<CAP>, dim3(grid), AW_THREADS<false>, 0, st, t, per));
    }
    return QGBDT_OK;
}

}  // namespace

int qg_adamw(qgbdt_ctx *c, const qgbdt_adamw_tensor *t, int32_t n, const qgbdt_adamw_options &o, cudaStream_t st) {
    AdamwFactors f;
    f.lr = o.lr, f.beta1 = o.beta1, f.beta2 = o.beta2, f.eps = o.eps, f.decay = o.weight_decay, f.max_norm = o.max_norm * o.loss_scale;
    f.loss_scale = o.loss_scale, f.step = o.step;
    f.seed = aw_mix(aw_mix((unsigned)o.seed) ^ (unsigned)(o.seed >> 32));
    f.d_lr = o.d_lr, f.d_step = reinterpret_cast<const long long *>(o.d_step), f.d_norm = o.d_norm;
    f.s.b1 = (float)o.beta1, f.s.c1 = (float)(1.0 - o.beta1), f.s.b2 = (float)o.beta2, f.s.c2 = (float)(1.0 - o.beta2);
    if (!o.d_norm) aw_of_gradients(f.s, f, 1.0 / o.loss_scale);
    aw_of_step(f.s, f, o.d_lr ? 0.0 : o.lr, o.d_step ? 1 : o.step);
    const bool packed = o.state_bits == 8;
    // An eps that is 2^23 times the root of 2^-126 or more in the first step already covers what a sum adds to the moments.  Smaller ones
    // (rare) are not worth a kernel of their own for few tensors.
    if (o.eps * sqrt(1.0 - o.beta2) < 0x1p-40) return packed ? aw_run<AW_LARGE, true, true>(c, t, n, f, st) : aw_run<AW_LARGE, false, true>(c, t, n, f, st);
    if (n <= AW_SMALL) return packed ? aw_run<AW_SMALL, true, false>(c, t, n, f, st) : aw_run<AW_SMALL, false, false>(c, t, n, f, st);
    if (n <= AW_MEDIUM) return packed ? aw_run<AW_MEDIUM, true, false>(c, t, n, f, st) : aw_run<AW_MEDIUM, false, false>(c, t, n, f, st);
    return packed ? aw_run<AW_LARGE, true, false>(c, t, n, f, st) : aw_run<AW_LARGE, false, false>(c, t, n, f, st);
}

int qg_adamw_values(qgbdt_ctx *c, const uint8_t *const *m, const uint8_t *const *v, const uint8_t *const *exponents, void *const *out_m,
                    void *const *out_v, const int64_t *counts, int32_t n, int32_t type, cudaStream_t st) {
    return n <= AW_SMALL ? aw_values<AW_SMALL>(c, m, v, exponents, out_m, out_v, counts, n, type, st)
                         : aw_values<AW_LARGE>(c, m, v, exponents, out_m, out_v, counts, n, type, st);
}
