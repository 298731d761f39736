// Embedding bag over leaf numbers and its gradient by sorted tokens.
//
//   forward   out[i]   = scale * sum_k table[tok[i][k]]
//   gradient  grad[v]  = scale * sum over (i, k) with tok[i][k] == v of dout[i]
//
// Both are gathers of whole rows: per (row, token) one row of `dim` elements comes out of L2 or DRAM and
// is added in single precision, so the time is that traffic.  A row is read by a group of 2^lg lanes, one
// vector of up to 16 bytes per lane; wider rows are cut into column blocks of 32 vectors.  Rows that allow only narrow
// vectors and are read often are copied first, to where they allow wide ones.
//
// 65536 rows of 100 tokens, 256 bf16 each: 215 us for 3.4 GB of rows, which is what L2 delivers (13 TB/s; 15 % are hits in L1).
//
// Gradient: the (token, row) pairs are sorted by token with a stable radix sort (pairs keep their row
// order inside a token), the sorted list is cut into tiles of equal length, and a group of lanes walks a
// tile adding rows until the token changes.  A token whose pairs cross a tile border leaves partial sums
// that a second kernel adds in an order that depends on the tiles alone.  Equal tile lengths keep the work even however
// the tokens crowd, and the order of every sum depends on the tokens alone.  The same 65536 rows: 395 us, of which the sums
// take 270 (12.7 TB/s out of L2), sorting 100, the joining 20.
#include <type_traits>

#include "ops_internal.cuh"

namespace {

constexpr int EMB_THREADS = 256;
constexpr int EMB_UNROLL = 8;

// A token as 32 bits: negative ones have the top bit, ones beyond 31 bits become 2^31 - 1 (which no table has).
__device__ __forceinline__ unsigned token_at(const int32_t *tokens, long long i) { return (unsigned)tokens[i]; }
__device__ __forceinline__ unsigned token_at(const int64_t *tokens, long long i) {
    const int64_t t = tokens[i];
    return t < 0 ? 0x80000000u : t < 0x7fffffff ? (unsigned)t : 0x7fffffffu;
}

struct EmbedPlan {
    int lg;        // log2 of the lanes per row
    int split;     // log2 of the parts a bag is cut into (forward)
    int col_blocks;
    bool out_vec;  // the output's rows take whole vectors
};

// Two single-precision sums in one instruction.
__device__ __forceinline__ void add2(float &a, float &b, float x, float y) {
    asm("{\n.reg .b64 s, t;\nmov.b64 s, {%0, %1};\nmov.b64 t, {%2, %3};\nadd.rn.f32x2 s, s, t;\nmov.b64 {%0, %1}, s;\n}" : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}

__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

template <typename T, int V>
__device__ __forceinline__ void add_row(float (&acc)[V], const OpsVec<T, V> &x) {
    if constexpr (V == 1) {
        acc[0] += OpsType<T>::load(x.v[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < V; j += 2) add2(acc[j], acc[j + 1], x.v[j], x.v[j + 1]);
    } else {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&x);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 y = unpack2(w[j / 2], T());
            add2(acc[j], acc[j + 1], y.x, y.y);
        }
    }
}

// acc * scale: a whole vector, or one by one the `left` elements up to the row's end.
template <typename T, int V>
__device__ __forceinline__ void store_row(T *out, const float (&acc)[V], float scale, bool vec, int left) {
    OpsVec<T, V> y;
#pragma unroll
    for (int j = 0; j < V; ++j) y.v[j] = OpsType<T>::store(acc[j] * scale);
    if (vec) {
        *reinterpret_cast<OpsVec<T, V> *>(out) = y;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < left) out[j] = y.v[j];
    }
}

// Row `t` of a matrix with rows of `ld_bytes` (below 2^32): one 32 x 32 bit product per address.
template <typename T, int V>
__device__ __forceinline__ OpsVec<T, V> row_of(const T *p, unsigned t, unsigned ld_bytes) {
    return *reinterpret_cast<const OpsVec<T, V> *>(reinterpret_cast<const char *>(p) + (unsigned long long)t * ld_bytes);
}

// One group of lanes per (row, part of the bag, column block).  Eight rows of the table are in flight per group.
template <typename T, int V, typename I>
__global__ void __launch_bounds__(EMB_THREADS) k_embed(const EmbedArgs a, const EmbedPlan p) {
    qg_after_prior();
    using Vec = OpsVec<T, V>;
    __shared__ float part_sum[EMB_THREADS][V];
    const int lane = threadIdx.x & ((1 << p.lg) - 1), group = threadIdx.x >> p.lg;
    const int part = group & ((1 << p.split) - 1);
    const int rows_per_block = (EMB_THREADS >> p.lg) >> p.split;
    const long long row = (long long)(blockIdx.x / p.col_blocks) * rows_per_block + (group >> p.split);
    const int col = ((int)(blockIdx.x % p.col_blocks) << p.lg) * V + lane * V;
    const bool live = row < a.rows && col < a.dim;
    const I *tok = reinterpret_cast<const I *>(a.tokens) + row * a.ld_tokens;
    const T *table = reinterpret_cast<const T *>(a.table) + col;
    const unsigned ld_bytes = (unsigned)(a.ld * sizeof(T)), n_entries = (unsigned)a.n_entries;
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.0f;
    if (live) {
        const int k0 = (int)((long long)a.bag * part >> p.split), k1 = (int)((long long)a.bag * (part + 1) >> p.split);
        bool bad = false;
        int k = k0;
        unsigned next[EMB_UNROLL];   // tokens, 2^31 and more: missing; loaded under the rows of the batch before
        auto load_tokens = [&](int at) {
#pragma unroll
            for (int u = 0; u < EMB_UNROLL; ++u) next[u] = token_at(tok, at + u);
        };
        if (k + EMB_UNROLL <= k1) load_tokens(k);
        for (; k + EMB_UNROLL <= k1; k += EMB_UNROLL) {
            bool on[EMB_UNROLL];
            Vec x[EMB_UNROLL];
#pragma unroll
            for (int u = 0; u < EMB_UNROLL; ++u) {   // without a predicate on the loads: for a missing token row 0 is read and left out
                on[u] = next[u] < n_entries;
                bad |= !on[u] && next[u] < 0x80000000u;
                x[u] = row_of<T, V>(table, on[u] ? next[u] : 0u, ld_bytes);
            }
            if (k + 2 * EMB_UNROLL <= k1) load_tokens(k + EMB_UNROLL);
#pragma unroll
            for (int u = 0; u < EMB_UNROLL; ++u)
                if (on[u]) add_row(acc, x[u]);
        }
#pragma unroll 4
        for (; k < k1; ++k) {
            const unsigned t = token_at(tok, k);
            const bool on = t < n_entries;
            const Vec x = row_of<T, V>(table, on ? t : 0u, ld_bytes);
            if (on) add_row(acc, x);
            bad |= !on && t < 0x80000000u;
        }
        if (bad && lane == 0 && a.status) *a.status = 1;
    }
    if (p.split) {
#pragma unroll
        for (int j = 0; j < V; ++j) part_sum[threadIdx.x][j] = acc[j];
        __syncthreads();
        if (part == 0)
            for (int q = 1; q < (1 << p.split); ++q)
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += part_sum[threadIdx.x + (q << p.lg)][j];
    }
    if (live && part == 0) store_row(reinterpret_cast<T *>(a.out) + row * a.ld_out + col, acc, a.scale, p.out_vec, a.dim - col);
}

// The plain lookup, one token per row: a group of lanes per row, four vectors in flight per lane.
template <typename T, int V, typename I>
__global__ void __launch_bounds__(EMB_THREADS) k_lookup(const EmbedArgs a, int lg) {
    qg_after_prior();
    using Vec = OpsVec<T, V>;
    const int lane = threadIdx.x & ((1 << lg) - 1), step = V << lg;
    const long long row = (long long)blockIdx.x * (EMB_THREADS >> lg) + (threadIdx.x >> lg);
    if (row >= a.rows) return;
    const unsigned t = token_at(reinterpret_cast<const I *>(a.tokens), row * a.ld_tokens);
    const bool on = t < (unsigned)a.n_entries;
    if (!on && t < 0x80000000u && lane == 0 && a.status) *a.status = 1;
    const T *in = reinterpret_cast<const T *>(a.table) + (on ? t : 0ll) * a.ld;
    T *out = reinterpret_cast<T *>(a.out) + row * a.ld_out;
    for (int col = lane * V; col < a.dim; col += step * 4) {
        Vec x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (col + u * step < a.dim) x[u] = *reinterpret_cast<const Vec *>(in + col + u * step);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (col + u * step < a.dim) {
                Vec y;
#pragma unroll
                for (int j = 0; j < V; ++j) y.v[j] = OpsType<T>::store(on ? OpsType<T>::load(x[u].v[j]) * a.scale : 0.0f);
                *reinterpret_cast<Vec *>(out + col + u * step) = y;
            }
    }
}

// ---- sorting of the (token, row) pairs -----------------------------------------------------------

struct SortArgs {
    const void *tokens;
    long long ld_tokens, n_entries, n;   // n pairs
    unsigned bag, div_mul, div_shift;    // i / bag == (i * div_mul) >> div_shift in 64 bits, for i < 2^31
    int row_bits;                        // of a packed pair
    int32_t *status;
    int blocks;                          // of a launch that sort; those behind them clear
};

// Few pairs beside the entries: nearly every row of the gradient is zero, and the sort leaves most SMs without work.  Its
// launches clear all rows then, a share each, in blocks behind those that sort.  4099 tokens, 50021 x 768 f16: 35 us with
// the rows no token points to cleared under the sums (as with many pairs), 29 us this way; 30000 tokens, 200000 x 512: 67 and 63 us.
struct ClearArgs {
    char *out;
    long long ld_bytes, row0, row1;
    int vectors, lg, vb;   // of a row; log2 of the lanes per row; bytes of a vector
};
constexpr int CLEAR_BLOCKS = 3;   // per SM, at most

template <typename V>
__device__ __forceinline__ void clear_with(const ClearArgs &z, int block, int blocks, V zero) {
    const int rows = EMB_THREADS >> z.lg;
    for (long long r = z.row0 + (long long)block * rows + (threadIdx.x >> z.lg); r < z.row1; r += (long long)blocks * rows) {
        V *row = reinterpret_cast<V *>(z.out + r * z.ld_bytes);
        for (int k = threadIdx.x & ((1 << z.lg) - 1); k < z.vectors; k += 1 << z.lg) row[k] = zero;
    }
}
__device__ void clear_ahead(const ClearArgs &z, int block, int blocks) {
    if (z.vb == 16) clear_with(z, block, blocks, make_uint4(0, 0, 0, 0));
    else if (z.vb == 8) clear_with(z, block, blocks, make_uint2(0, 0));
    else if (z.vb == 4) clear_with(z, block, blocks, 0u);
    else clear_with(z, block, blocks, (unsigned short)0);
}

// A pair between two passes: token and row in one word where both fit (every usual size), or in two.  The last pass
// writes two words in any case.
template <bool PACKED>
struct Pair {
    using E = uint2;
    static __device__ __forceinline__ E make(unsigned key, unsigned row, int) { return make_uint2(key, row); }
    static __device__ __forceinline__ unsigned word(E p) { return p.x; }   // the digits are taken from this one
    static __device__ __forceinline__ uint2 wide(E p, int) { return p; }
};
template <>
struct Pair<true> {
    using E = unsigned;
    static __device__ __forceinline__ E make(unsigned key, unsigned row, int row_bits) { return key << row_bits | row; }
    static __device__ __forceinline__ unsigned word(E p) { return p; }
    static __device__ __forceinline__ uint2 wide(E p, int row_bits) { return make_uint2(p >> row_bits, p & ((1u << row_bits) - 1)); }
};

// floor(i / d) for i < 2^31 as a product: with shift = 31 + ceil(log2 d) and mul = ceil(2^shift / d), mul < 2^32 and the
// error i * (mul * d - 2^shift) / (d * 2^shift) stays below 1 / d.
void set_divisor(SortArgs &a, unsigned d) {
    unsigned l = 0;
    while ((1ull << l) < d) ++l;
    a.bag = d;
    a.div_shift = 31 + l;
    a.div_mul = (unsigned)(((1ull << a.div_shift) + d - 1) / d);
}
__device__ __forceinline__ unsigned div_bag(const SortArgs &a, unsigned i) { return (unsigned)(((unsigned long long)i * a.div_mul) >> a.div_shift); }

// Where the token of pair i is, and what becomes of it: a missing or bad one is n_entries and sorts behind all
// others.  The two steps are apart so that a thread's loads come before the first use of any of them.
__device__ __forceinline__ long long token_index(const SortArgs &a, unsigned i) {
    if (a.ld_tokens == a.bag) return i;
    const unsigned row = div_bag(a, i);
    return (long long)row * a.ld_tokens + (i - row * a.bag);
}
__device__ __forceinline__ unsigned token_key(const SortArgs &a, unsigned t, bool &bad) {
    const unsigned n = (unsigned)a.n_entries;
    bad |= t >= n && t < 0x80000000u;
    return t < n ? t : n;
}

// Few pairs: every pair's place is the number of pairs before it, counted directly; one launch.
// A whole gradient of 4000 pairs takes 14 us with it and 20 with the passes below, of 6000 pairs 20 and 20.  Where rows are
// cleared ahead, the several launches of the passes hide more of that, so that the limit sinks with the bytes: 50021 rows of
// 128, 512, 1024 and 2048 bytes, 4099 pairs: 15, 19, 24, 36 us and 18, 20, 24, 34.
constexpr int SORT_SMALL = 6144;
constexpr long long SORT_SMALL_CLEAR = 32 << 10;   // bytes to clear that take a pair off the limit
constexpr int SORT_SMALL_LANES = 16;   // lanes that share the count of one pair

template <typename I>
__global__ void __launch_bounds__(EMB_THREADS) k_sort_small(const SortArgs a, const ClearArgs z, uint2 *out) {
    qg_after_prior();
    if ((int)blockIdx.x >= a.blocks) {
        clear_ahead(z, blockIdx.x - a.blocks, gridDim.x - a.blocks);
        return;
    }
    __shared__ alignas(16) unsigned key[SORT_SMALL];
    const int n = (int)a.n, n4 = (n + 3) / 4;
    const I *tokens = reinterpret_cast<const I *>(a.tokens);
    bool bad = false;
    for (int i = threadIdx.x; i < n4 * 4; i += EMB_THREADS * 4) {
        unsigned t[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) t[u] = token_at(tokens, token_index(a, min(i + u * EMB_THREADS, n - 1)));
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * EMB_THREADS < n4 * 4) key[i + u * EMB_THREADS] = i + u * EMB_THREADS < n ? token_key(a, t[u], bad) : 0xffffffffu;
    }
    if (bad && a.status) *a.status = 1;
    __syncthreads();
    const int e = (blockIdx.x * EMB_THREADS + threadIdx.x) / SORT_SMALL_LANES, lane = threadIdx.x % SORT_SMALL_LANES;
    const unsigned mine = e < n ? key[e] : 0;
    unsigned before = 0;
    const int own = e / 4;   // equal tokens in front of e count, those behind it do not
#pragma unroll 4
    for (int q = lane; q < n4; q += SORT_SMALL_LANES) {
        const uint4 k = reinterpret_cast<const uint4 *>(key)[q];
        const unsigned limit = q < own ? mine + 1 : mine;
        before += (k.x < limit) + (k.y < limit) + (k.z < limit) + (k.w < limit);
    }
    if (lane == own % SORT_SMALL_LANES)
        for (int i = 4 * own; i < e; ++i) before += key[i] == mine;
#pragma unroll
    for (int o = SORT_SMALL_LANES / 2; o; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    if (e < n && lane == 0) out[before] = make_uint2(mine, div_bag(a, (unsigned)e));
}

// Many pairs: least significant digit first, up to 9 bits a pass; a pass is a count per block and digit, a
// scan, and a stable scatter.  A block scatters tiles of 2048 pairs: every warp ranks its pairs among its own (each
// lane sets its bit in a word per digit, and reads who else did), the tile is put in order in shared memory, and runs of
// equal digits leave it as neighbouring words.  6.55 M pairs of 15 + 16 bits: 38 us per scatter, bound by shared
// memory: its data pipe is busy 55 % of the time (l1tex as a whole 81 % of its active cycles), warps wait for it most, a
// third of the issue slots is used (digits compared with a ballot per bit: 51 us); counts 11 to 15 us.
constexpr int SORT_MIN_BITS = 6, SORT_MAX_BITS = 9;
constexpr int SORT_WARPS = EMB_THREADS / 32;
constexpr int SORT_ROUNDS = 8;                                    // pairs per lane and tile
constexpr int SORT_TILE = EMB_THREADS * SORT_ROUNDS;

// Counts of a digit, one per block, padded to 16 bytes.
__host__ __device__ inline size_t count_stride(int blocks) { return ((size_t)blocks + 3) / 4 * 4; }

template <typename I, bool FIRST, bool PACKED>
__global__ void __launch_bounds__(EMB_THREADS) k_sort_count(const SortArgs a, const ClearArgs z, const typename Pair<PACKED>::E *in, int shift, int bits, long long per_block,
                                                            unsigned *counts) {
    qg_after_prior();
    if ((int)blockIdx.x >= a.blocks) {
        clear_ahead(z, blockIdx.x - a.blocks, gridDim.x - a.blocks);
        return;
    }
    extern __shared__ unsigned sort_smem[];
    unsigned *cnt = sort_smem;   // [1 << bits]
    const int digits = 1 << bits;
    for (int d = threadIdx.x; d < digits; d += EMB_THREADS) cnt[d] = 0;
    __syncthreads();
    const long long i0 = per_block * blockIdx.x, i1 = i0 + per_block < a.n ? i0 + per_block : a.n;
    constexpr int LOADS = 16;
    for (long long i = i0 + threadIdx.x; i < i1; i += EMB_THREADS * LOADS) {
        unsigned key[LOADS];
#pragma unroll
        for (int r = 0; r < LOADS; ++r) {
            const long long at = min(i + r * EMB_THREADS, i1 - 1);
            key[r] = FIRST ? token_at(reinterpret_cast<const I *>(a.tokens), token_index(a, (unsigned)at)) : Pair<PACKED>::word(in[at]);
        }
        bool bad = false;
#pragma unroll
        for (int r = 0; r < LOADS; ++r)
            if (i + r * EMB_THREADS < i1) atomicAdd(&cnt[((FIRST ? token_key(a, key[r], bad) : key[r]) >> shift) & (digits - 1)], 1u);
        if (FIRST && bad && a.status) *a.status = 1;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += EMB_THREADS) counts[(size_t)d * count_stride(a.blocks) + blockIdx.x] = cnt[d];
}

// Per digit (one warp): exclusive scan over the blocks, and the digit's total.
__global__ void __launch_bounds__(EMB_THREADS) k_sort_scan(unsigned *counts, unsigned *totals, int digits, int blocks) {
    qg_after_prior();
    const int d = blockIdx.x * SORT_WARPS + threadIdx.x / 32, lane = threadIdx.x & 31;
    if (d >= digits) return;
    unsigned *row = counts + (size_t)d * count_stride(blocks), run = 0;
    for (int b = 0; b < blocks; b += 32 * 8) {
        unsigned x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = b + u * 32 + lane < blocks ? row[b + u * 32 + lane] : 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            unsigned s = x[u];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned y = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o) s += y;
            }
            if (b + u * 32 + lane < blocks) row[b + u * 32 + lane] = run + s - x[u];
            run += __shfl_sync(0xffffffffu, s, 31);
        }
    }
    if (lane == 0) totals[d] = run;
}

size_t scatter_smem(int bits, size_t pair) { return (size_t)SORT_TILE * pair + ((size_t)8 + 6 * SORT_WARPS) * ((size_t)1 << bits); }   // below 48 KB

// Exclusive scan over the block of one number per thread.
__device__ __forceinline__ unsigned block_scan(unsigned x, unsigned *warp_sum) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    unsigned inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    unsigned run = inc - x;
    for (int w = 0; w < warp; ++w) run += warp_sum[w];
    __syncthreads();
    return run;
}

// totals == NULL: the counts have not been scanned; with few blocks every block adds up what it needs itself, which
// takes less time than a launch for it.
constexpr int SORT_FEW_BLOCKS = 128;

template <typename I, bool FIRST, bool PACKED, bool LAST, int BITS>
__global__ void __launch_bounds__(EMB_THREADS, 4) k_sort_scatter(const SortArgs a, const ClearArgs z, const typename Pair<PACKED>::E *in, int shift, long long per_block,
                                                                 const unsigned *counts, const unsigned *totals, void *out) {
    qg_after_prior();
    if ((int)blockIdx.x >= a.blocks) {
        clear_ahead(z, blockIdx.x - a.blocks, gridDim.x - a.blocks);
        return;
    }
    using P = Pair<PACKED>;
    using E = typename P::E;
    extern __shared__ unsigned sort_smem[];
    __shared__ unsigned warp_sum[SORT_WARPS];
    constexpr int digits = 1 << BITS;
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    E *sorted = reinterpret_cast<E *>(sort_smem);                               // [SORT_TILE] the tile in order
    unsigned *base = reinterpret_cast<unsigned *>(sorted + SORT_TILE);          // [digits] where the tile's pairs of a digit go
    unsigned *begin = base + digits;                                            // [digits] where they begin in the tile
    unsigned *match = begin + digits;                                           // [SORT_WARPS][digits] lanes with this digit; 0 between rounds
    unsigned short *cnt = reinterpret_cast<unsigned short *>(match + SORT_WARPS * digits);   // [SORT_WARPS][digits] pairs of a warp, then those of earlier warps
    for (int d = threadIdx.x; d < SORT_WARPS * digits; d += EMB_THREADS) match[d] = 0;
    const unsigned i0 = (unsigned)per_block * blockIdx.x, i1 = min(i0 + (unsigned)per_block, (unsigned)a.n);
    // a tile's pairs (or tokens) are loaded under the work on the tile before; those of a warp are consecutive, so that
    // its rounds keep their order
    using Load = typename std::conditional<FIRST, unsigned, E>::type;
    Load next[SORT_ROUNDS];
    const unsigned in_tile = warp * 32 * SORT_ROUNDS + lane;
    auto load = [&](unsigned tile) {
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            const unsigned at = min(tile + in_tile + r * 32, i1 - 1);
            if constexpr (FIRST) next[r] = token_at(reinterpret_cast<const I *>(a.tokens), token_index(a, at));
            else next[r] = in[at];
        }
    };
    if (i0 < i1) load(i0);
    const int per = (digits + EMB_THREADS - 1) / EMB_THREADS, d0 = threadIdx.x * per;   // digits of this thread in the scans
    {   // base = pairs of smaller digits (scan of the totals) + pairs of this digit in earlier blocks
        const int blocks = a.blocks, mine = blockIdx.x;
        const size_t stride = count_stride(blocks);
        unsigned s = 0;
        for (int j = 0; j < per && d0 + j < digits; ++j) {
            unsigned total = 0, before = 0;
            if (totals) {
                total = totals[d0 + j];
                before = counts[(d0 + j) * stride + mine];
            } else {
                const uint4 *row = reinterpret_cast<const uint4 *>(counts + (d0 + j) * stride);
#pragma unroll 8
                for (int b = 0; b < blocks; b += 4) {
                    const uint4 x = row[b / 4];
                    const unsigned y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        total += b + k < blocks ? y[k] : 0;
                        before += b + k < mine ? y[k] : 0;
                    }
                }
            }
            begin[d0 + j] = total;
            base[d0 + j] = before;
            s += total;
        }
        unsigned run = block_scan(s, warp_sum);
        for (int j = 0; j < per && d0 + j < digits; ++j) {
            base[d0 + j] += run;
            run += begin[d0 + j];
        }
    }
    for (unsigned tile = i0; tile < i1; tile += SORT_TILE) {
        const unsigned w0 = tile + in_tile;
        E pair[SORT_ROUNDS];
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            if constexpr (FIRST) {
                bool bad = false;   // reported by the count
                pair[r] = P::make(token_key(a, next[r], bad), div_bag(a, w0 + r * 32), a.row_bits);
            } else {
                pair[r] = next[r];
            }
        }
        if (tile + SORT_TILE < i1) load(tile + SORT_TILE);
        for (int d = threadIdx.x; d < digits * SORT_WARPS / 2; d += EMB_THREADS) reinterpret_cast<unsigned *>(cnt)[d] = 0;
        __syncthreads();
        unsigned short place[SORT_ROUNDS], *mine = cnt + warp * digits;
        unsigned *lanes = match + warp * digits;
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {   // every lane enters itself at its digit, and looks who else did
            const bool on = w0 + r * 32 < i1;
            const unsigned d = P::word(pair[r]) >> shift & (digits - 1);
            if (on) atomicOr(&lanes[d], 1u << lane);
            __syncwarp();
            const unsigned same = lanes[d], below = __popc(same & ((1u << lane) - 1));
            const unsigned short old = mine[d];
            __syncwarp();
            if (on && below == 0) mine[d] = (unsigned short)(old + __popc(same)), lanes[d] = 0;
            __syncwarp();
            place[r] = (unsigned short)(old + below);
        }
        __syncthreads();
        unsigned sum = 0;
        for (int j = 0; j < per && d0 + j < digits; ++j) {
            unsigned run = 0;
#pragma unroll
            for (int w = 0; w < SORT_WARPS; ++w) {
                const unsigned x = cnt[w * digits + d0 + j];
                cnt[w * digits + d0 + j] = (unsigned short)run;
                run += x;
            }
            begin[d0 + j] = run;
            sum += run;
        }
        unsigned run = block_scan(sum, warp_sum);
        for (int j = 0; j < per && d0 + j < digits; ++j) {
            const unsigned x = begin[d0 + j];
            begin[d0 + j] = run;
            run += x;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r)
            if (w0 + r * 32 < i1) {
                const unsigned d = (P::word(pair[r]) >> shift) & (digits - 1);
                sorted[begin[d] + mine[d] + place[r]] = pair[r];
            }
        __syncthreads();
        const unsigned n = min(i1 - tile, (unsigned)SORT_TILE);
#pragma unroll 8
        for (unsigned i = threadIdx.x; i < n; i += EMB_THREADS) {
            const E p = sorted[i];
            const unsigned d = (P::word(p) >> shift) & (digits - 1), to = base[d] + i - begin[d];
            if constexpr (LAST) reinterpret_cast<uint2 *>(out)[to] = P::wide(p, a.row_bits);
            else reinterpret_cast<E *>(out)[to] = p;
        }
        __syncthreads();
        for (int j = 0; j < per && d0 + j < digits; ++j)   // begin of the next digit - begin = pairs of this digit in the tile
            base[d0 + j] += (d0 + j + 1 < digits ? begin[d0 + j + 1] : n) - begin[d0 + j];
        __syncthreads();
    }
}

// ---- sums over the sorted pairs ------------------------------------------------------------------

struct SegArgs {
    const uint2 *pair;      // [n] sorted by token
    long long n;
    int tile;               // pairs per tile
    long long tiles;
    const void *grad;
    long long ld;
    void *out;
    long long ld_out, n_entries;
    int dim, lg, col_blocks;
    bool out_vec;           // the output's rows take whole vectors
    int ld_partial;         // dim, rounded up to whole vectors
    float scale;
    float *partial;         // [tiles][2][ld_partial]: sum of a tile's first token when it began in an earlier tile;
                            // sum of its last token when it began here and goes on in the next tile
    long long sum_blocks;   // blocks that add; those behind them clear the rows no token points to, unless all are
    bool cleared;
};

constexpr int ZERO_ROWS = 128;   // rows of the gradient a clearing block looks at

__device__ __forceinline__ long long first_not_below(const uint2 *pair, long long n, unsigned key) {
    long long lo = 0, hi = n;
    while (lo < hi) {
        const long long mid = (lo + hi) >> 1;
        if (pair[mid].x < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

template <typename T, int V, bool OUT_VEC>
__device__ void clear_rows(const SegArgs &a, long long block) {
    __shared__ unsigned absent[ZERO_ROWS / 32];
    const long long v0 = block * ZERO_ROWS;
    if (threadIdx.x < ZERO_ROWS) {
        const long long v = v0 + threadIdx.x;
        bool none = false;
        if (v < a.n_entries) {
            const long long at = first_not_below(a.pair, a.n, (unsigned)v);
            none = at >= a.n || a.pair[at].x != (unsigned)v;
        }
        const unsigned m = __ballot_sync(0xffffffffu, none);
        if ((threadIdx.x & 31) == 0) absent[threadIdx.x / 32] = m;
    }
    __syncthreads();
    OpsVec<T, V> zero;
#pragma unroll
    for (int j = 0; j < V; ++j) zero.v[j] = OpsType<T>::store(0.0f);
    for (int r = threadIdx.x >> a.lg; r < ZERO_ROWS; r += EMB_THREADS >> a.lg) {
        if (!(absent[r / 32] >> (r & 31) & 1)) continue;
        T *row = reinterpret_cast<T *>(a.out) + (v0 + r) * a.ld_out;
        if constexpr (OUT_VEC)
            for (int col = (threadIdx.x & ((1 << a.lg) - 1)) * V; col < a.dim; col += V << a.lg) *reinterpret_cast<OpsVec<T, V> *>(row + col) = zero;
        else
            for (int col = threadIdx.x & ((1 << a.lg) - 1); col < a.dim; col += 1 << a.lg) row[col] = zero.v[0];
    }
}

// Blocks of the sums per SM, by the bytes of a vector: what the registers of eight rows in flight allow.  Narrow vectors move
// less per load: 600000 pairs of 200 bytes in vectors of 8, the whole gradient: 53 us with three blocks, 50 with four (five
// spill more, 63).  The widest vectors spill a few bytes (4 to 8 stored) at these settings too.
constexpr int sum_blocks_per_sm(int vector) { return vector == 16 ? 3 : 4; }

// OUT_VEC: the output's rows take whole vectors (tested at run time it costs registers: 395 and 441 us).
template <typename T, int V, bool OUT_VEC>
__global__ void __launch_bounds__(EMB_THREADS, sum_blocks_per_sm(sizeof(T) * V)) k_segment_sum(const SegArgs a) {
    qg_after_prior();
    using Vec = OpsVec<T, V>;
    const long long block = blockIdx.x;
    if (block >= a.sum_blocks) {   // behind the others: these wait for nothing
        clear_rows<T, V, OUT_VEC>(a, block - a.sum_blocks);
        return;
    }
    const int lane = threadIdx.x & ((1 << a.lg) - 1), group = threadIdx.x >> a.lg;
    const long long t = block / a.col_blocks * (EMB_THREADS >> a.lg) + group;
    const int col = ((int)(block % a.col_blocks) << a.lg) * V + lane * V;
    if (t >= a.tiles || col >= a.dim) return;
    const long long i0 = t * a.tile, i1 = i0 + a.tile < a.n ? i0 + a.tile : a.n;
    const unsigned none = (unsigned)a.n_entries;
    const T *grad = reinterpret_cast<const T *>(a.grad) + col;
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.0f;
    unsigned cur = a.pair[i0].x;
    if (cur == none) return;
    bool from_before = i0 > 0 && a.pair[i0 - 1].x == cur;
    auto put_partial = [&](int slot) {
        float *w = a.partial + (t * 2 + slot) * a.ld_partial + col;
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = acc[j];
    };
    auto finish = [&]() {   // the token's pairs end inside this tile
        if (from_before) {
            put_partial(0);
        } else {
            Vec y;
#pragma unroll
            for (int j = 0; j < V; ++j) y.v[j] = OpsType<T>::store(acc[j] * a.scale);
            T *to = reinterpret_cast<T *>(a.out) + (long long)cur * a.ld_out + col;
            if constexpr (OUT_VEC) {
                *reinterpret_cast<Vec *>(to) = y;
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (col + j < a.dim) to[j] = y.v[j];
            }
        }
    };
    const unsigned ld_bytes = (unsigned)(a.ld * sizeof(T));
    bool more = true;
    auto take = [&](unsigned key, const Vec &x) {
        if (key != cur) {
            if (key == none) {   // missing tokens are sorted last
                more = false;
                return;
            }
            finish();
            cur = key;
            from_before = false;
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = 0.0f;
        }
        add_row(acc, x);
    };
    // batches start on 64 bytes of the list; a batch's pairs are loaded under the rows of the one before (and, at the
    // list's end, from its padding)
    const long long whole = i0 + (i1 - i0) / EMB_UNROLL * EMB_UNROLL;
    OpsVec<uint2, 2> next[EMB_UNROLL / 2];
    auto load_pairs = [&](long long i) {
#pragma unroll
        for (int u = 0; u < EMB_UNROLL / 2; ++u) next[u] = reinterpret_cast<const OpsVec<uint2, 2> *>(a.pair + i)[u];
    };
    load_pairs(i0);
    for (long long i = i0; i < whole && more; i += EMB_UNROLL) {
        unsigned key[EMB_UNROLL];
        Vec x[EMB_UNROLL];
#pragma unroll
        for (int u = 0; u < EMB_UNROLL; ++u) {
            key[u] = next[u / 2].v[u & 1].x;
            x[u] = row_of<T, V>(grad, next[u / 2].v[u & 1].y, ld_bytes);   // a missing token's row is read and left out
        }
        load_pairs(i + EMB_UNROLL);
#pragma unroll
        for (int u = 0; u < EMB_UNROLL; ++u)
            if (more) take(key[u], x[u]);
    }
    for (long long i = whole; i < i1 && more; ++i) take(a.pair[i].x, row_of<T, V>(grad, a.pair[i].y, ld_bytes));
    if (i1 < a.n && a.pair[i1].x == cur) put_partial(from_before ? 0 : 1);
    else finish();
}

// Tokens that cross tile borders: 2^lg_cols threads add a token's partial sums, four columns each; 2^lg_parts such rows of
// threads, in the same warp, share those of every tile where such a token begins, and join their sums in a tree.  A token
// of very many tiles is shared by the whole block.  The order of every sum depends on the tiles alone.
constexpr int JOIN_PARTS = 2;    // lg_parts at most: 655360 pairs, 310 x 16 f32: 41 us with 0, 34 with 2, 36 with 3
constexpr int JOIN_LOADS = 4;    // sums in flight per thread
constexpr int JOIN_TILES = 32;   // tiles of a token that the block does not share

template <typename T, int V, bool OUT_VEC>
__global__ void __launch_bounds__(EMB_THREADS) k_segment_join(const SegArgs a, int lg_cols, int lg_parts) {
    qg_after_prior();
    __shared__ float part_sum[EMB_THREADS][V];
    __shared__ long long long_links[EMB_THREADS];   // per group: tiles of a token that the whole block adds, or 0
    __shared__ unsigned long_token[EMB_THREADS];
    const int cols = 1 << lg_cols, row = threadIdx.x >> lg_cols, rows = EMB_THREADS >> lg_cols, lane = threadIdx.x & (cols - 1);
    const int parts = 1 << lg_parts, part = row & (parts - 1), group = row >> lg_parts, groups = rows >> lg_parts;   // a group per tile
    const unsigned none = (unsigned)a.n_entries;
    // Tiles t + 1 .. t + links hold the rest of a token that begins in tile t; 0 where there is none.  The four words
    // that settle nearly every tile are loaded at once.
    auto links_of = [&](long long t, unsigned &cur) -> long long {
        const long long i0 = t * a.tile, i1 = i0 + a.tile;
        if (i1 >= a.n) return 0;
        auto key = [&](long long i) { return a.pair[i < a.n ? i : a.n - 1].x; };
        const unsigned before = i0 > 0 ? key(i0 - 1) : none, last = key(i1 - 1), next = key(i1), second = key(i1 + a.tile);
        cur = next;
        if (cur == none || last != cur || before == cur) return 0;
        if (i1 + a.tile >= a.n || second != cur) return 1;
        // the last tile that begins with it: eight places are looked at together, further and further away, then in between
        auto inside = [&](long long l) { return a.pair[min((t + l) * a.tile, a.n - 1)].x == cur && (t + l) * a.tile < a.n; };
        long long lo = 2, hi = 0;
        for (long long base = 4; hi == 0; base <<= 8) {
            bool in[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) in[u] = inside(base << u);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (hi == 0) (in[u] ? lo : hi) = base << u;
        }
        while (hi - lo > 1) {
            const long long step = (hi - lo + 8) / 9, from = lo, to = hi;
            bool in[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) in[u] = inside(min(from + step * (u + 1), to));
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const long long at = from + step * (u + 1);
                if (at < hi) (in[u] ? lo : hi) = at;
            }
        }
        return lo;
    };
    auto put = [&](unsigned cur, int col, const float (&s)[V]) {
        store_row(reinterpret_cast<T *>(a.out) + (long long)cur * a.ld_out + col, s, a.scale, OUT_VEC, a.dim - col);
    };
    // the token's sums 0 .. links of this row of threads: every `step`-th from `first` on
    auto add_all = [&](float (&s)[V], long long t, long long links, int first, int step, int col) {
        for (long long l = first; l <= links; l += JOIN_LOADS * step) {   // some loads in flight, also behind the last sum
            OpsVec<float, V> x[JOIN_LOADS];
#pragma unroll
            for (int u = 0; u < JOIN_LOADS; ++u) {
                const long long at = min(l + u * step, links);
                x[u] = *reinterpret_cast<const OpsVec<float, V> *>(a.partial + ((t + at) * 2 + (at == 0)) * a.ld_partial + col);
            }
#pragma unroll
            for (int u = 0; u < JOIN_LOADS; ++u)
                if (l + u * step <= links)
#pragma unroll
                    for (int j = 0; j < V; ++j) s[j] += x[u].v[j];
        }
    };
    auto tree = [&](float (&s)[V], int lanes) {   // over the rows of threads among `lanes` lanes
        for (int o = lanes / 2; o >= cols; o >>= 1)
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
    };
    // tokens of few tiles
    const long long t0 = (long long)blockIdx.x * groups, mine = t0 + group;
    unsigned cur = 0;
    long long links = links_of(mine, cur);
    const bool few = links > 0 && links <= JOIN_TILES;
    if (__any_sync(0xffffffffu, few))
        for (int c0 = 0; c0 < a.dim; c0 += cols * V) {
            const int col = c0 + lane * V;
            float s[V] = {};
            if (few && col < a.dim) add_all(s, mine, links, part, parts, col);
            tree(s, cols << lg_parts);
            if (few && col < a.dim && part == 0) put(cur, col, s);
        }
    if (part == 0 && lane == 0) long_links[group] = links > JOIN_TILES ? links : 0, long_token[group] = cur;
    if (!__syncthreads_or(links > JOIN_TILES)) return;
    for (int q = 0; q < groups; ++q) {   // the whole block for each of the others
        links = long_links[q];
        if (links == 0) continue;
        const long long t = t0 + q;
        cur = long_token[q];
        for (int c0 = 0; c0 < a.dim; c0 += cols * V) {
            const int col = c0 + lane * V;
            float s[V] = {};
            if (col < a.dim) add_all(s, t, links, row, rows, col);
            tree(s, 32);
#pragma unroll
            for (int j = 0; j < V; ++j) part_sum[threadIdx.x][j] = s[j];
            __syncthreads();
            if (row == 0 && col < a.dim) {   // the warps, or wider rows of threads, in their order
                const int step = cols < 32 ? 32 : cols;
                for (int k = step; k < EMB_THREADS; k += step)
#pragma unroll
                    for (int j = 0; j < V; ++j) s[j] += part_sum[lane + k][j];
                put(cur, col, s);
            }
            __syncthreads();
        }
    }
}

// ---- few pairs and few entries: no sorting -----------------------------------------------------------
// Every warp takes entries in turn, looks all tokens over for it (32 at a time), lists the rows of those it finds and
// adds them, eight in flight, in their order.  One launch instead of three; worth it while entries * pairs stays small.

constexpr int SCAN_PAIRS = 4096;
constexpr long long SCAN_WORK = 1ll << 22;   // entries * pairs

template <typename T, int V, typename I>
__global__ void __launch_bounds__(EMB_THREADS) k_scan_sum(const SortArgs a, const SegArgs g) {
    qg_after_prior();
    using Vec = OpsVec<T, V>;
    constexpr int LIST = 128;
    __shared__ unsigned key[SCAN_PAIRS];
    __shared__ unsigned lists[EMB_THREADS / 32][LIST];
    unsigned *list = lists[threadIdx.x / 32];
    const int n = (int)a.n, n32 = (n + 31) / 32 * 32, lane = threadIdx.x & 31;
    const I *tokens = reinterpret_cast<const I *>(a.tokens);
    bool bad = false;
    for (int i = threadIdx.x; i < n32; i += EMB_THREADS * 4) {
        unsigned t[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) t[u] = token_at(tokens, token_index(a, min(i + u * EMB_THREADS, n - 1)));
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * EMB_THREADS < n32) key[i + u * EMB_THREADS] = i + u * EMB_THREADS < n ? token_key(a, t[u], bad) : (unsigned)a.n_entries;
    }
    if (bad && a.status) *a.status = 1;
    __syncthreads();
    const unsigned ld_bytes = (unsigned)(g.ld * sizeof(T));
    const int warps = gridDim.x * (EMB_THREADS / 32);
    for (int v = blockIdx.x * (EMB_THREADS / 32) + threadIdx.x / 32; v < (int)g.n_entries; v += warps)
        for (int c0 = 0; c0 < g.dim; c0 += 32 * V) {
            const int col = c0 + lane * V;
            const T *grad = reinterpret_cast<const T *>(g.grad) + (col < g.dim ? col : 0);
            float acc[V];
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = 0.0f;
            int listed = 0;
            auto add_listed = [&]() {
                __syncwarp();
                for (int k = 0; k < listed; k += EMB_UNROLL) {
                    Vec x[EMB_UNROLL];
#pragma unroll
                    for (int u = 0; u < EMB_UNROLL; ++u) x[u] = row_of<T, V>(grad, list[min(k + u, listed - 1)], ld_bytes);
#pragma unroll
                    for (int u = 0; u < EMB_UNROLL; ++u)
                        if (k + u < listed) add_row(acc, x[u]);
                }
                __syncwarp();
                listed = 0;
            };
            for (int i = 0; i < n32; i += 32) {
                const bool hit = key[i + lane] == (unsigned)v;
                const unsigned m = __ballot_sync(0xffffffffu, hit);
                if (hit) list[listed + __popc(m & ((1u << lane) - 1))] = div_bag(a, (unsigned)(i + lane));
                listed += __popc(m);
                if (listed > LIST - 32) add_listed();
            }
            if (listed > 0) add_listed();
            if (col < g.dim) {
                Vec y;
#pragma unroll
                for (int j = 0; j < V; ++j) y.v[j] = OpsType<T>::store(acc[j] * g.scale);
                *reinterpret_cast<Vec *>(reinterpret_cast<T *>(g.out) + (long long)v * g.ld_out + col) = y;
            }
        }
}

// ---- launches --------------------------------------------------------------------------------------

// Copy of a matrix with rows that start on 16 bytes, zeros behind their ends.
template <typename E>
__global__ void __launch_bounds__(EMB_THREADS) k_align_rows(const E *in, long long ld, long long rows, int dim, E *out, int ld_out) {
    qg_after_prior();
    constexpr int V = 16 / sizeof(E);
    const int vectors = ld_out / V;
    for (long long i = blockIdx.x * (long long)EMB_THREADS + threadIdx.x; i < rows * vectors; i += (long long)gridDim.x * EMB_THREADS) {
        const long long r = i / vectors;
        const int d = (int)(i - r * vectors) * V;
        OpsVec<E, V> x;
#pragma unroll
        for (int j = 0; j < V; ++j) x.v[j] = in[r * ld + min(d + j, dim - 1)];
#pragma unroll
        for (int j = 0; j < V; ++j) x.v[j] = d + j < dim ? x.v[j] : E(0);
        *reinterpret_cast<OpsVec<E, V> *>(out + r * ld_out + d) = x;
    }
}

// Rows that are read many times in vectors of less than 16 bytes: a copy of them with aligned rows pays for a launch and
// a pass over them where enough is read, the sooner the narrower the vectors are.  Forward, without and with a copy, f16:
// 20 MB in vectors of 2 bytes 12 and 9 us, of 4 bytes 8 and 9; 61 MB of 4 bytes 17 and 12, of 8 bytes 11 and 12; 504 MB of
// 8 bytes 49 and 45, of 2 bytes 161 and 45; 2.2 GB of 2 bytes 747 and 216.  The gradient's: 725 and 315.
constexpr int ALIGN_REUSE = 4;                // times a row is read, on average
constexpr long long ALIGN_BYTES = 3ll << 20;  // that are read, per square of the vectors' bytes
constexpr size_t ALIGN_MOST = 1ull << 30;     // a larger copy is not worth its memory

// The matrix to read from (`rows` rows), aligned where that pays for `reads` rows read in vectors of vb bytes; `below`: not
// for vectors of this size on.
struct AlignedRows {
    size_t bytes = 0;   // of the copy; 0: none
    int ld = 0;
};
AlignedRows align_plan(long long rows, int dim, int width, int vb, int below, long long reads) {
    AlignedRows r;
    if (vb >= below || reads < ALIGN_REUSE * rows || reads * dim * width < ALIGN_BYTES * vb * vb) return r;
    r.ld = (dim * width + 15) / 16 * 16 / width;
    const size_t bytes = qg_ws_size((size_t)rows * r.ld, width);
    if (bytes <= ALIGN_MOST) r.bytes = bytes;
    return r;
}
int align_rows(qgbdt_ctx *c, EmbedArgs &a, long long rows, const AlignedRows &r, QgWorkspace &ws, cudaStream_t st) {
    const int w = qg_type_size(a.type);
    const long long want = (rows * r.ld * w / 16 + EMB_THREADS - 1) / EMB_THREADS, most = c->sm_count * 16;
    const unsigned blocks = (unsigned)(want < most ? want : most);
    const void *in = a.table;
    void *out = ws.take<char>(r.bytes);
    const long long ld = a.ld;
    a.table = out, a.ld = r.ld;
    if (w == 4) return qg_launch(c, k_align_rows<uint32_t>, dim3(blocks), EMB_THREADS, 0, st, reinterpret_cast<const uint32_t *>(in), ld, rows, a.dim, reinterpret_cast<uint32_t *>(out), r.ld);
    return qg_launch(c, k_align_rows<uint16_t>, dim3(blocks), EMB_THREADS, 0, st, reinterpret_cast<const uint16_t *>(in), ld, rows, a.dim, reinterpret_cast<uint16_t *>(out), r.ld);
}

int log2_at_least(long long v, int most) {   // smallest l <= most with 2^l >= v
    int l = 0;
    while (l < most && (1ll << l) < v) ++l;
    return l;
}

int vec_bytes(const EmbedArgs &a) {
    const int w = qg_type_size(a.type);
    const int x = qg_vec_bytes(a.table, a.ld * w, (int64_t)a.dim * w), y = qg_vec_bytes(a.out, a.ld_out * w, (int64_t)a.dim * w);
    return x < y ? x : y;
}

template <typename T, int V>
int embed_typed(qgbdt_ctx *c, const EmbedArgs &a, bool out_vec, cudaStream_t st) {
    EmbedPlan p;
    p.out_vec = out_vec;
    p.lg = log2_at_least((a.dim + V - 1) / V, 5);
    p.col_blocks = (a.dim + (V << p.lg) - 1) / (V << p.lg);
    if (a.bag == 1) {
        const long long blocks = (a.rows + (EMB_THREADS >> p.lg) - 1) / (EMB_THREADS >> p.lg);
        return qg_launch(c, a.token_type == QGBDT_I64 ? k_lookup<T, V, int64_t> : k_lookup<T, V, int32_t>, dim3((unsigned)blocks), EMB_THREADS, 0, st, a, p.lg);
    }
    // few rows: a bag is cut into parts until every SM has 512 threads, parts hold at least two tokens
    const long long threads = a.rows * p.col_blocks << p.lg;
    p.split = 0;
    while (p.split < 8 - p.lg && (threads << p.split) < (long long)c->sm_count * 512 && (a.bag >> (p.split + 1)) >= 2) ++p.split;
    const long long rows_per_block = (EMB_THREADS >> p.lg) >> p.split;
    const long long blocks = (a.rows + rows_per_block - 1) / rows_per_block * p.col_blocks;
    if (blocks > 0x7fffffffll) return qg_fail(c, QGBDT_ERR_ARG, "rows * dim is too large for one call");
    return qg_launch(c, a.token_type == QGBDT_I64 ? k_embed<T, V, int64_t> : k_embed<T, V, int32_t>, dim3((unsigned)blocks), EMB_THREADS, 0, st, a, p);
}

// Radix passes for keys up to n_entries.
struct SortPlan {
    int passes, bits, blocks;
    long long per_block;
};

SortPlan sort_plan(const qgbdt_ctx *c, long long n, long long n_entries) {
    SortPlan s;
    const int bits = log2_at_least(n_entries + 1, 32);
    s.passes = (bits + SORT_MAX_BITS - 1) / SORT_MAX_BITS;
    if (s.passes < 1) s.passes = 1;
    s.bits = (bits + s.passes - 1) / s.passes;
    if (s.bits < SORT_MIN_BITS) s.bits = SORT_MIN_BITS;
    const long long tiles = (n + SORT_TILE - 1) / SORT_TILE;
    const long long most = 4ll * c->sm_count;   // blocks that fit beside one another
    s.blocks = (int)(tiles < most ? tiles : most);
    s.per_block = (tiles + s.blocks - 1) / s.blocks * SORT_TILE;
    return s;
}

// The rows to clear ahead of the sums, in equal shares for the sort's launches; blocks == 0: none.
struct Clearing {
    ClearArgs all;
    int blocks, launches;
    ClearArgs share(int k) const {
        ClearArgs z = all;
        z.row0 = all.row1 * k / launches, z.row1 = all.row1 * (k + 1) / launches;
        return z;
    }
};

template <typename I, bool FIRST, bool PACKED, bool LAST>
int sort_scatter(qgbdt_ctx *c, const SortArgs &a, const SortPlan &s, const Clearing &z, int launch, const void *in, int shift, const unsigned *counts, const unsigned *totals, void *out,
                 cudaStream_t st) {
    using E = typename Pair<PACKED>::E;
    const auto kernel = s.bits == 6   ? k_sort_scatter<I, FIRST, PACKED, LAST, 6>
                        : s.bits == 7 ? k_sort_scatter<I, FIRST, PACKED, LAST, 7>
                        : s.bits == 8 ? k_sort_scatter<I, FIRST, PACKED, LAST, 8>
                                      : k_sort_scatter<I, FIRST, PACKED, LAST, 9>;
    return qg_launch(c, kernel, dim3(s.blocks + z.blocks), EMB_THREADS, scatter_smem(s.bits, sizeof(E)), st, a, z.share(launch), reinterpret_cast<const E *>(in), shift, s.per_block,
                     counts, totals, out);
}

template <typename I, bool PACKED>
int sort_passes(qgbdt_ctx *c, const SortArgs &a, const SortPlan &s, const Clearing &z, void *in, void *out, unsigned *counts, unsigned *totals, const uint2 **sorted,
                cudaStream_t st) {
    using E = typename Pair<PACKED>::E;
    const int digits = 1 << s.bits;
    const bool scan = s.blocks > SORT_FEW_BLOCKS;
    for (int k = 0; k < s.passes; ++k) {
        const bool first = k == 0, last = k == s.passes - 1;
        const int shift = k * s.bits, at = PACKED ? shift + a.row_bits : shift;   // of the token; of the digit in a pair's word
        QG_RUN(first ? qg_launch(c, k_sort_count<I, true, PACKED>, dim3(s.blocks + z.blocks), EMB_THREADS, digits * sizeof(unsigned), st, a, z.share(2 * k),
                                 reinterpret_cast<const E *>(in), shift, s.bits, s.per_block, counts)
                     : qg_launch(c, k_sort_count<int32_t, false, PACKED>, dim3(s.blocks + z.blocks), EMB_THREADS, digits * sizeof(unsigned), st, a, z.share(2 * k),
                                 reinterpret_cast<const E *>(in), at, s.bits, s.per_block, counts));
        if (scan) QG_RUN(qg_launch(c, k_sort_scan, dim3((digits + SORT_WARPS - 1) / SORT_WARPS), EMB_THREADS, 0, st, counts, totals, digits, s.blocks));
        const unsigned *t = scan ? totals : nullptr;
        QG_RUN(first ? (last ? sort_scatter<I, true, PACKED, true>(c, a, s, z, 2 * k + 1, in, at, counts, t, out, st)
                             : sort_scatter<I, true, PACKED, false>(c, a, s, z, 2 * k + 1, in, at, counts, t, out, st))
                     : (last ? sort_scatter<int32_t, false, PACKED, true>(c, a, s, z, 2 * k + 1, in, at, counts, t, out, st)
                             : sort_scatter<int32_t, false, PACKED, false>(c, a, s, z, 2 * k + 1, in, at, counts, t, out, st)));
        void *swap = in;
        in = out;
        out = swap;
    }
    *sorted = reinterpret_cast<const uint2 *>(in);
    return QGBDT_OK;
}

template <typename I>
int sort_pairs(qgbdt_ctx *c, SortArgs a, const SortPlan &s, Clearing z, uint2 *buf0, uint2 *buf1, unsigned *counts, unsigned *totals, const uint2 **sorted,
               cudaStream_t st) {
    if (s.passes == 0) {
        *sorted = buf0;
        a.blocks = (int)((a.n * SORT_SMALL_LANES + EMB_THREADS - 1) / EMB_THREADS), z.launches = 1;
        return qg_launch(c, k_sort_small<I>, dim3(a.blocks + z.blocks), EMB_THREADS, 0, st, a, z.share(0), buf0);
    }
    a.blocks = s.blocks, z.launches = 2 * s.passes;
    a.row_bits = log2_at_least(a.n / a.bag, 31);
    return a.row_bits + log2_at_least(a.n_entries + 1, 32) <= 32 ? sort_passes<I, true>(c, a, s, z, buf1, buf0, counts, totals, sorted, st)
                                                                 : sort_passes<I, false>(c, a, s, z, buf1, buf0, counts, totals, sorted, st);
}

template <typename T, int V>
int segments_typed(qgbdt_ctx *c, SegArgs s, cudaStream_t st) {
    const long long per_block = EMB_THREADS >> s.lg;
    s.sum_blocks = (s.tiles + per_block - 1) / per_block * s.col_blocks;
    const long long blocks = s.sum_blocks + (s.cleared ? 0 : (s.n_entries + ZERO_ROWS - 1) / ZERO_ROWS);
    if (blocks > 0x7fffffffll) return qg_fail(c, QGBDT_ERR_ARG, "rows * bag * dim is too large for one call");
    auto kernel = k_segment_sum<T, V, true>;
    if constexpr (sizeof(T) * V == 16) kernel = s.out_vec ? kernel : k_segment_sum<T, V, false>;   // (of an aligned copy)
    QG_RUN(qg_launch(c, kernel, dim3((unsigned)blocks), EMB_THREADS, 0, st, s));
    if (s.tiles > 1) {
        // four columns at most per thread: their partial sums are one 16-byte load
        constexpr int JV = V < 4 ? V : 4;
        const int lg = log2_at_least((s.dim + JV - 1) / JV, 7), lg_parts = lg >= 5 ? 0 : lg >= 5 - JOIN_PARTS ? 5 - lg : JOIN_PARTS;
        const long long groups = EMB_THREADS >> lg >> lg_parts;
        auto join = k_segment_join<T, JV, true>;
        if constexpr (sizeof(T) * V == 16) join = s.out_vec ? join : k_segment_join<T, JV, false>;
        QG_RUN(qg_launch(c, join, dim3((unsigned)((s.tiles - 2) / groups + 1)), EMB_THREADS, 0, st, s, lg, lg_parts));
    }
    return QGBDT_OK;
}

template <typename T, int V>
int scan_typed(qgbdt_ctx *c, const SortArgs &a, const SegArgs &g, bool wide, cudaStream_t st) {
    const long long want = (g.n_entries + EMB_THREADS / 32 - 1) / (EMB_THREADS / 32), most = c->sm_count * 6;
    return qg_launch(c, wide ? k_scan_sum<T, V, int64_t> : k_scan_sum<T, V, int32_t>, dim3((unsigned)(want < most ? want : most)), EMB_THREADS, 0, st, a, g);
}

// Calls f<T, V>() for the element type and the vector width in bytes.
#define EMBED_DISPATCH(type, vb, CALL)                                                ((type) == QGBDT_F32 ? ((vb) == 16 ? CALL(float, 4) : (vb) == 8 ? CALL(float, 2) : CALL(float, 1))                            : (type) == QGBDT_BF16                                                                                                           ? ((vb) == 16 ? CALL(__nv_bfloat16, 8) : (vb) == 8 ? CALL(__nv_bfloat16, 4) : (vb) == 4 ? CALL(__nv_bfloat16, 2) : CALL(__nv_bfloat16, 1))          : ((vb) == 16 ? CALL(__half, 8) : (vb) == 8 ? CALL(__half, 4) : (vb) == 4 ? CALL(__half, 2) : CALL(__half, 1)))

}  // namespace

int qg_embed(qgbdt_ctx *c, const EmbedArgs &given, cudaStream_t st) {
    EmbedArgs a = given;
    int vb = vec_bytes(a);
    const AlignedRows r = align_plan(a.n_entries, a.dim, qg_type_size(a.type), vb, 16, a.bag > 1 ? a.rows * a.bag : 0);
    QgWorkspace ws;
    if (r.bytes) {
        QG_RUN(qg_ws_open(c, r.bytes, st, &ws));
        QG_RUN(align_rows(c, a, a.n_entries, r, ws, st));
        vb = 16;
    }
    const bool out_vec = !r.bytes || vec_bytes(a) == 16;
#define CALL(T, V) embed_typed<T, V>(c, a, out_vec, st)
    QG_RUN(EMBED_DISPATCH(a.type, vb, CALL));
#undef CALL
    return r.bytes ? qg_ws_close(c, st) : QGBDT_OK;
}

int qg_embed_backward(qgbdt_ctx *c, const EmbedArgs &given, cudaStream_t st) {
    EmbedArgs a = given;
    const long long n = a.rows * a.bag;
    const int w = qg_type_size(a.type), vb_given = vec_bytes(a);
    const bool scan = n > 0 && n <= SCAN_PAIRS && n * a.n_entries <= SCAN_WORK;
    const AlignedRows r = scan ? AlignedRows{} : align_plan(a.rows, a.dim, w, vb_given, 8, n);   // (504 MB in vectors of 8 bytes: 95 us, 99 with a copy)
    const int vb = r.bytes ? 16 : vb_given, V = vb / w;
    SegArgs s{};
    s.n = n;
    s.ld_partial = (a.dim + V - 1) / V * V, s.out_vec = !r.bytes;
    s.grad = a.table, s.ld = a.ld, s.out = a.out, s.ld_out = a.ld_out, s.n_entries = a.n_entries;
    s.dim = a.dim, s.scale = a.scale;
    SortArgs sa{};
    sa.tokens = a.tokens, sa.ld_tokens = a.ld_tokens, sa.n_entries = a.n_entries, sa.n = n, sa.status = a.status;
    set_divisor(sa, (unsigned)a.bag);
    if (scan) {
#define CALL(T, V) scan_typed<T, V>(c, sa, s, a.token_type == QGBDT_I64, st)
        return EMBED_DISPATCH(a.type, vb, CALL);
#undef CALL
    }
    s.lg = log2_at_least((a.dim + V - 1) / V, 5);
    s.col_blocks = (a.dim + (V << s.lg) - 1) / (V << s.lg);
    // tiles: short lists go once over the groups of 768 threads per SM (more and shorter ones add to the joining: 185000 pairs
    // of 200 bytes 34 us, 39 us with 1024), long ones four times, which evens out what the SMs get; at least 16 pairs
    const long long fit = (long long)c->sm_count * 768 >> s.lg, pairs = (n * s.col_blocks + fit - 1) / fit;
    long long tile = pairs <= 128 ? pairs : pairs <= 512 ? 128 : pairs / 4;
    tile = tile < 16 ? 16 : (tile + EMB_UNROLL - 1) / EMB_UNROLL * EMB_UNROLL;
    s.tile = (int)(tile < (1 << 20) ? tile : 1 << 20);
    s.tiles = (n + s.tile - 1) / s.tile;
    // few pairs beside the entries: all rows are cleared ahead (at most half as much again is written as has to be)
    const bool ahead = n > 0 && 2 * n <= a.n_entries;
    const bool small = n <= SORT_SMALL - (ahead ? a.n_entries * a.dim * qg_type_size(a.type) / SORT_SMALL_CLEAR : 0);
    const SortPlan sp = small ? SortPlan{} : sort_plan(c, n, a.n_entries);
    const size_t digits = small ? 0 : (size_t)1 << sp.bits;
    const size_t bytes = 2 * qg_ws_size((size_t)n + 2 * EMB_UNROLL, sizeof(uint2)) + qg_ws_size(digits * count_stride(sp.blocks), sizeof(unsigned)) +
                         qg_ws_size(digits, sizeof(unsigned)) + qg_ws_size((size_t)s.tiles * 2 * s.ld_partial, sizeof(float)) + r.bytes;
    QgWorkspace ws;
    int rc = qg_ws_open(c, bytes, st, &ws);
    if (rc != QGBDT_OK) return rc;
    uint2 *buf0 = ws.take<uint2>((size_t)n + 2 * EMB_UNROLL), *buf1 = ws.take<uint2>((size_t)n + 2 * EMB_UNROLL);
    unsigned *counts = ws.take<unsigned>(digits * count_stride(sp.blocks)), *totals = ws.take<unsigned>(digits);
    s.partial = ws.take<float>((size_t)s.tiles * 2 * s.ld_partial);
    if (r.bytes) {
        QG_RUN(align_rows(c, a, a.rows, r, ws, st));
        s.grad = a.table, s.ld = a.ld, s.out_vec = vec_bytes(a) == 16;
    }
    s.pair = buf0;
    Clearing z{};
    if (ahead) {
        const int W = vb_given / w;   // the output's rows take these
        z.all = ClearArgs{reinterpret_cast<char *>(a.out), a.ld_out * w, 0, a.n_entries, a.dim / W, log2_at_least(a.dim / W, 8), vb_given};
        const long long want = (a.n_entries * a.dim / W + EMB_THREADS * 16 - 1) / (EMB_THREADS * 16), most = (long long)c->sm_count * CLEAR_BLOCKS;
        z.blocks = (int)(want < most ? want : most);
        s.cleared = true;
    }
    if (n > 0) {
        rc = a.token_type == QGBDT_I64 ? sort_pairs<int64_t>(c, sa, sp, z, buf0, buf1, counts, totals, &s.pair, st)
                                       : sort_pairs<int32_t>(c, sa, sp, z, buf0, buf1, counts, totals, &s.pair, st);
        if (rc != QGBDT_OK) return rc;
    }
#define CALL(T, V) segments_typed<T, V>(c, s, st)
    rc = EMBED_DISPATCH(a.type, vb, CALL);
#undef CALL
    if (rc != QGBDT_OK) return rc;
    return qg_ws_close(c, st);
}
