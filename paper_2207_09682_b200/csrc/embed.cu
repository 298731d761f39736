// Embedding bag over leaf numbers and its gradient by sorted tokens.
//
//   forward   out[i]   = scale * sum_k table[tok[i][k]]
//   gradient  grad[v]  = scale * sum over (i, k) with tok[i][k] == v of dout[i]
//
// Both are gathers of whole rows: per (row, token) one row of `dim` elements comes out of L2 or DRAM and
// is added in single precision, so the time is that traffic.  A row is read by a group of 2^lg lanes, one
// vector of up to 16 bytes per lane; wider rows are cut into column blocks of 32 vectors.
//
// Gradient: the (token, row) pairs are sorted by token with a stable radix sort (pairs keep their row
// order inside a token), the sorted list is cut into tiles of equal length, and a group of lanes walks a
// tile adding rows until the token changes.  A token whose pairs cross a tile border leaves partial sums
// that a second kernel adds in tile order.  Equal tile lengths keep the work even however the tokens
// crowd, and the order of every sum depends on the tokens alone.
#include "ops_internal.cuh"

namespace {

constexpr int EMB_THREADS = 256;
constexpr int EMB_UNROLL = 8;

template <typename I>
__device__ __forceinline__ long long token_at(const I *tokens, long long i) { return (long long)tokens[i]; }

struct EmbedPlan {
    int lg;        // log2 of the lanes per row
    int split;     // log2 of the parts a bag is cut into (forward)
    int col_blocks;
};

template <typename T, int V>
__device__ __forceinline__ void add_row(float (&acc)[V], const OpsVec<T, V> &x) {
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] += OpsType<T>::load(x.v[j]);
}

// One group of lanes per (row, part of the bag, column block).  Eight rows of the table are in flight per group.
template <typename T, int V, typename I>
__global__ void __launch_bounds__(EMB_THREADS) k_embed(const EmbedArgs a, const EmbedPlan p) {
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
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.0f;
    if (live) {
        const int k0 = (int)((long long)a.bag * part >> p.split), k1 = (int)((long long)a.bag * (part + 1) >> p.split);
        bool bad = false;
        for (int k = k0; k < k1; k += EMB_UNROLL) {
            long long t[EMB_UNROLL];
            Vec x[EMB_UNROLL];
#pragma unroll
            for (int u = 0; u < EMB_UNROLL; ++u) t[u] = k + u < k1 ? token_at(tok, k + u) : -1;
#pragma unroll
            for (int u = 0; u < EMB_UNROLL; ++u) {
                if (t[u] >= a.n_entries) bad = true, t[u] = -1;
                if (t[u] >= 0) x[u] = *reinterpret_cast<const Vec *>(table + t[u] * a.ld);
            }
#pragma unroll
            for (int u = 0; u < EMB_UNROLL; ++u)
                if (t[u] >= 0) add_row(acc, x[u]);
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
    if (live && part == 0) {
        Vec y;
#pragma unroll
        for (int j = 0; j < V; ++j) y.v[j] = OpsType<T>::store(acc[j] * a.scale);
        *reinterpret_cast<Vec *>(reinterpret_cast<T *>(a.out) + row * a.ld_out + col) = y;
    }
}

// ---- sorting of the (token, row) pairs -----------------------------------------------------------

struct SortArgs {
    const void *tokens;
    long long ld_tokens, n_entries, n;   // n pairs
    int bag;
    int32_t *status;
};

// Token and row of pair i; a missing or bad token becomes n_entries and sorts behind all others.
template <typename I>
__device__ __forceinline__ uint2 pair_at(const SortArgs &a, long long i) {
    const unsigned row = (unsigned)i / (unsigned)a.bag, k = (unsigned)i - row * (unsigned)a.bag;
    const long long t = token_at(reinterpret_cast<const I *>(a.tokens), (long long)row * a.ld_tokens + k);
    if (t >= a.n_entries && a.status) *a.status = 1;
    return make_uint2(t >= 0 && t < a.n_entries ? (unsigned)t : (unsigned)a.n_entries, row);
}

// Few pairs: every pair's place is the number of pairs before it, counted directly; one launch.
constexpr int SORT_SMALL = 4096;
constexpr int SORT_SMALL_LANES = 8;   // lanes that share the count of one pair

template <typename I>
__global__ void __launch_bounds__(EMB_THREADS) k_sort_small(const SortArgs a, uint2 *out) {
    __shared__ alignas(16) unsigned key[SORT_SMALL];
    const int n = (int)a.n, n4 = (n + 3) / 4;
    for (int i = threadIdx.x; i < n4 * 4; i += EMB_THREADS) key[i] = i < n ? pair_at<I>(a, i).x : 0xffffffffu;
    __syncthreads();
    const int e = (blockIdx.x * EMB_THREADS + threadIdx.x) / SORT_SMALL_LANES, lane = threadIdx.x % SORT_SMALL_LANES;
    const unsigned mine = e < n ? key[e] : 0;
    unsigned before = 0;
    for (int q = lane; q < n4; q += SORT_SMALL_LANES) {
        const uint4 k = reinterpret_cast<const uint4 *>(key)[q];
        before += (k.x < mine || (k.x == mine && 4 * q < e)) + (k.y < mine || (k.y == mine && 4 * q + 1 < e)) +
                  (k.z < mine || (k.z == mine && 4 * q + 2 < e)) + (k.w < mine || (k.w == mine && 4 * q + 3 < e));
    }
#pragma unroll
    for (int o = SORT_SMALL_LANES / 2; o; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    if (e < n && lane == 0) out[before] = make_uint2(mine, (unsigned)e / (unsigned)a.bag);
}

// Many pairs: least significant digit first, up to 11 bits a pass; a pass is a count per block and digit, a
// scan, and a stable scatter.
constexpr int SORT_MAX_BITS = 11;
constexpr int SORT_WARPS = EMB_THREADS / 32;
constexpr int SORT_ROUNDS = 16;                                    // pairs per lane and tile
constexpr int SORT_TILE = EMB_THREADS * SORT_ROUNDS;

template <typename I, bool FIRST>
__device__ __forceinline__ uint2 sort_load(const SortArgs &a, const uint2 *in, long long i) {
    return FIRST ? pair_at<I>(a, i) : in[i];
}

template <typename I, bool FIRST>
__global__ void __launch_bounds__(EMB_THREADS) k_sort_count(const SortArgs a, const uint2 *in, int shift, int bits, long long per_block,
                                                            unsigned *counts) {
    __shared__ unsigned cnt[1 << SORT_MAX_BITS];
    const int digits = 1 << bits;
    for (int d = threadIdx.x; d < digits; d += EMB_THREADS) cnt[d] = 0;
    __syncthreads();
    const long long i0 = per_block * blockIdx.x, i1 = i0 + per_block < a.n ? i0 + per_block : a.n;
    for (long long i = i0 + threadIdx.x; i < i1; i += EMB_THREADS)
        atomicAdd(&cnt[(sort_load<I, FIRST>(a, in, i).x >> shift) & (digits - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += EMB_THREADS) counts[(size_t)d * gridDim.x + blockIdx.x] = cnt[d];
}

// Per digit (one warp): exclusive scan over the blocks, and the digit's total.
__global__ void __launch_bounds__(EMB_THREADS) k_sort_scan(unsigned *counts, unsigned *totals, int digits, int blocks) {
    const int d = blockIdx.x * SORT_WARPS + threadIdx.x / 32, lane = threadIdx.x & 31;
    if (d >= digits) return;
    unsigned *row = counts + (size_t)d * blocks, run = 0;
    for (int b = 0; b < blocks; b += 32) {
        const unsigned x = b + lane < blocks ? row[b + lane] : 0;
        unsigned s = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        if (b + lane < blocks) row[b + lane] = run + s - x;
        run += __shfl_sync(0xffffffffu, s, 31);
    }
    if (lane == 0) totals[d] = run;
}

template <typename I, bool FIRST>
__global__ void __launch_bounds__(EMB_THREADS) k_sort_scatter(const SortArgs a, const uint2 *in, int shift, int bits, long long per_block,
                                                              const unsigned *counts, const unsigned *totals, uint2 *out) {
    __shared__ unsigned short cnt[SORT_WARPS][1 << SORT_MAX_BITS];   // per warp and digit: pairs so far in this tile, then those of earlier warps
    __shared__ unsigned base[1 << SORT_MAX_BITS];                    // where the next pair of a digit goes
    __shared__ unsigned warp_sum[SORT_WARPS];
    const int digits = 1 << bits, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    // base = pairs of smaller digits (scan of the totals) + pairs of this digit in earlier blocks
    {
        const int per = (digits + EMB_THREADS - 1) / EMB_THREADS, d0 = threadIdx.x * per;
        unsigned s = 0;
        for (int j = 0; j < per && d0 + j < digits; ++j) s += totals[d0 + j];
        unsigned inc = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned y = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += y;
        }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        unsigned run = inc - s;
        for (int w = 0; w < warp; ++w) run += warp_sum[w];
        for (int j = 0; j < per && d0 + j < digits; ++j) {
            base[d0 + j] = run + counts[(size_t)(d0 + j) * gridDim.x + blockIdx.x];
            run += totals[d0 + j];
        }
    }
    const long long i0 = per_block * blockIdx.x, i1 = i0 + per_block < a.n ? i0 + per_block : a.n;
    for (long long tile = i0; tile < i1; tile += SORT_TILE) {
        for (int d = threadIdx.x; d < digits * SORT_WARPS; d += EMB_THREADS) cnt[d >> bits][d & (digits - 1)] = 0;
        __syncthreads();
        const long long w0 = tile + (long long)warp * 32 * SORT_ROUNDS;   // a warp's pairs are consecutive: its rounds keep their order
        uint2 pair[SORT_ROUNDS];
        unsigned short place[SORT_ROUNDS];
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            const long long i = w0 + r * 32 + lane;
            if (i < i1) pair[r] = sort_load<I, FIRST>(a, in, i);
        }
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            const bool on = w0 + r * 32 + lane < i1;
            const unsigned d = on ? (pair[r].x >> shift) & (digits - 1) : 0xffffffffu;
            const unsigned same = __match_any_sync(0xffffffffu, d), below = __popc(same & ((1u << lane) - 1));
            unsigned short old = 0;
            if (on) old = cnt[warp][d];
            __syncwarp();
            if (on && below == 0) cnt[warp][d] = (unsigned short)(old + __popc(same));
            __syncwarp();
            place[r] = (unsigned short)(old + below);
        }
        __syncthreads();
        unsigned add[(1 << SORT_MAX_BITS) / EMB_THREADS];
#pragma unroll
        for (int j = 0; j < (1 << SORT_MAX_BITS) / EMB_THREADS; ++j) {
            const int d = threadIdx.x + j * EMB_THREADS;
            unsigned run = 0;
            if (d < digits) {
#pragma unroll
                for (int w = 0; w < SORT_WARPS; ++w) {
                    const unsigned x = cnt[w][d];
                    cnt[w][d] = (unsigned short)run;
                    run += x;
                }
            }
            add[j] = run;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r)
            if (w0 + r * 32 + lane < i1) {
                const unsigned d = (pair[r].x >> shift) & (digits - 1);
                out[base[d] + cnt[warp][d] + place[r]] = pair[r];
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < (1 << SORT_MAX_BITS) / EMB_THREADS; ++j) {
            const int d = threadIdx.x + j * EMB_THREADS;
            if (d < digits) base[d] += add[j];
        }
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
    float scale;
    float *partial;         // [tiles][2][dim]: sum of a tile's first token when it began in an earlier tile;
                            // sum of its last token when it began here and goes on in the next tile
    long long zero_blocks;  // blocks that clear the rows no token points to
};

constexpr int ZERO_ROWS = 32;   // rows of the gradient a clearing block looks at

__device__ __forceinline__ long long first_not_below(const uint2 *pair, long long n, unsigned key) {
    long long lo = 0, hi = n;
    while (lo < hi) {
        const long long mid = (lo + hi) >> 1;
        if (pair[mid].x < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

template <typename T, int V>
__device__ void clear_rows(const SegArgs &a, long long block) {
    __shared__ unsigned absent;
    const long long v0 = block * ZERO_ROWS;
    if (threadIdx.x < 32) {
        const long long v = v0 + threadIdx.x;
        bool none = false;
        if (v < a.n_entries) {
            const long long at = first_not_below(a.pair, a.n, (unsigned)v);
            none = at >= a.n || a.pair[at].x != (unsigned)v;
        }
        const unsigned m = __ballot_sync(0xffffffffu, none);
        if (threadIdx.x == 0) absent = m;
    }
    __syncthreads();
    OpsVec<T, V> zero;
#pragma unroll
    for (int j = 0; j < V; ++j) zero.v[j] = OpsType<T>::store(0.0f);
    for (unsigned m = absent; m; m &= m - 1) {
        T *row = reinterpret_cast<T *>(a.out) + (v0 + __ffs(m) - 1) * a.ld_out;
        for (int col = threadIdx.x * V; col < a.dim; col += EMB_THREADS * V) *reinterpret_cast<OpsVec<T, V> *>(row + col) = zero;
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(EMB_THREADS) k_segment_sum(const SegArgs a) {
    using Vec = OpsVec<T, V>;
    if ((long long)blockIdx.x < a.zero_blocks) {
        clear_rows<T, V>(a, blockIdx.x);
        return;
    }
    const long long block = (long long)blockIdx.x - a.zero_blocks;
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
        float *w = a.partial + (t * 2 + slot) * a.dim + col;
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
            *reinterpret_cast<Vec *>(reinterpret_cast<T *>(a.out) + (long long)cur * a.ld_out + col) = y;
        }
    };
    for (long long i = i0; i < i1; i += EMB_UNROLL) {
        uint2 p[EMB_UNROLL];
        Vec x[EMB_UNROLL];
#pragma unroll
        for (int u = 0; u < EMB_UNROLL; ++u) p[u] = i + u < i1 ? a.pair[i + u] : make_uint2(none, 0);
#pragma unroll
        for (int u = 0; u < EMB_UNROLL; ++u)
            if (p[u].x != none) x[u] = *reinterpret_cast<const Vec *>(grad + (long long)p[u].y * a.ld);
#pragma unroll
        for (int u = 0; u < EMB_UNROLL; ++u) {
            if (p[u].x == none) continue;   // behind the tile's end, or a missing token (these are sorted last)
            if (p[u].x != cur) {
                finish();
                cur = p[u].x;
                from_before = false;
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] = 0.0f;
            }
            add_row(acc, x[u]);
        }
    }
    if (i1 < a.n && a.pair[i1].x == cur) put_partial(from_before ? 0 : 1);
    else finish();
}

// Tokens that cross tile borders: the block of the tile where such a token begins adds its partial sums
// in tile order (cut into 256 / columns runs that are added in order as well).
template <typename T>
__global__ void __launch_bounds__(EMB_THREADS) k_segment_join(const SegArgs a, int lg_cols) {
    __shared__ float part_sum[EMB_THREADS];
    const long long t = blockIdx.x;
    const long long i0 = t * a.tile, i1 = i0 + a.tile;
    if (i1 >= a.n) return;
    const unsigned cur = a.pair[i1].x;
    if (cur == (unsigned)a.n_entries || a.pair[i1 - 1].x != cur || (a.pair[i0].x == cur && i0 > 0 && a.pair[i0 - 1].x == cur)) return;
    const long long last = first_not_below(a.pair, a.n, cur + 1) - 1;   // the token's last pair
    const long long links = last / a.tile - t;                           // slot 0 of tiles t + 1 .. t + links
    const int cols = 1 << lg_cols, parts = EMB_THREADS >> lg_cols, part = threadIdx.x >> lg_cols;
    const long long l0 = links * part / parts, l1 = links * (part + 1) / parts;
    for (int c0 = 0; c0 < a.dim; c0 += cols) {
        const int col = c0 + (threadIdx.x & (cols - 1));
        float s = 0.0f;
        if (col < a.dim) {
            if (part == 0) s = a.partial[(t * 2 + 1) * a.dim + col];
#pragma unroll 4
            for (long long l = l0; l < l1; ++l) s += a.partial[((t + 1 + l) * 2) * a.dim + col];
        }
        part_sum[threadIdx.x] = s;
        __syncthreads();
        if (part == 0 && col < a.dim) {
            for (int q = 1; q < parts; ++q) s += part_sum[threadIdx.x + (q << lg_cols)];
            reinterpret_cast<T *>(a.out)[(long long)cur * a.ld_out + col] = OpsType<T>::store(s * a.scale);
        }
        __syncthreads();
    }
}

// ---- launches --------------------------------------------------------------------------------------

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
int embed_typed(qgbdt_ctx *c, const EmbedArgs &a, cudaStream_t st) {
    EmbedPlan p;
    p.lg = log2_at_least((a.dim + V - 1) / V, 5);
    p.col_blocks = (a.dim + (V << p.lg) - 1) / (V << p.lg);
    // few rows: a bag is cut into parts until every SM has 512 threads, parts hold at least two tokens
    const long long threads = a.rows * p.col_blocks << p.lg;
    p.split = 0;
    while (p.split < 8 - p.lg && (threads << p.split) < (long long)c->sm_count * 512 && (a.bag >> (p.split + 1)) >= 2) ++p.split;
    const long long rows_per_block = (EMB_THREADS >> p.lg) >> p.split;
    const long long blocks = (a.rows + rows_per_block - 1) / rows_per_block * p.col_blocks;
    if (blocks > 0x7fffffffll) return qg_fail(c, QGBDT_ERR_ARG, "rows * dim is too large for one call");
    if (a.token_type == QGBDT_I64) k_embed<T, V, int64_t><<<(unsigned)blocks, EMB_THREADS, 0, st>>>(a, p);
    else k_embed<T, V, int32_t><<<(unsigned)blocks, EMB_THREADS, 0, st>>>(a, p);
    QG_LAUNCH_CHECK(c);
    return QGBDT_OK;
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
    if (s.bits < 1) s.bits = 1;
    const long long tiles = (n + SORT_TILE - 1) / SORT_TILE;
    s.blocks = (int)(tiles < 2 * c->sm_count ? tiles : 2 * c->sm_count);
    s.per_block = (tiles + s.blocks - 1) / s.blocks * SORT_TILE;
    return s;
}

template <typename I>
int sort_pairs(qgbdt_ctx *c, const SortArgs &a, const SortPlan &s, uint2 *buf0, uint2 *buf1, unsigned *counts, unsigned *totals,
               const uint2 **sorted, cudaStream_t st) {
    if (a.n <= SORT_SMALL) {
        k_sort_small<I><<<(unsigned)((a.n * SORT_SMALL_LANES + EMB_THREADS - 1) / EMB_THREADS), EMB_THREADS, 0, st>>>(a, buf0);
        QG_LAUNCH_CHECK(c);
        *sorted = buf0;
        return QGBDT_OK;
    }
    const int digits = 1 << s.bits;
    uint2 *in = buf1, *out = buf0;
    for (int k = 0; k < s.passes; ++k) {
        const int shift = k * s.bits;
        if (k == 0) k_sort_count<I, true><<<s.blocks, EMB_THREADS, 0, st>>>(a, in, shift, s.bits, s.per_block, counts);
        else k_sort_count<I, false><<<s.blocks, EMB_THREADS, 0, st>>>(a, in, shift, s.bits, s.per_block, counts);
        QG_LAUNCH_CHECK(c);
        k_sort_scan<<<(digits + SORT_WARPS - 1) / SORT_WARPS, EMB_THREADS, 0, st>>>(counts, totals, digits, s.blocks);
        QG_LAUNCH_CHECK(c);
        if (k == 0) k_sort_scatter<I, true><<<s.blocks, EMB_THREADS, 0, st>>>(a, in, shift, s.bits, s.per_block, counts, totals, out);
        else k_sort_scatter<I, false><<<s.blocks, EMB_THREADS, 0, st>>>(a, in, shift, s.bits, s.per_block, counts, totals, out);
        QG_LAUNCH_CHECK(c);
        uint2 *swap = in;
        in = out;
        out = swap;
    }
    *sorted = in;
    return QGBDT_OK;
}

template <typename T, int V>
int segments_typed(qgbdt_ctx *c, SegArgs s, cudaStream_t st) {
    const long long per_block = EMB_THREADS >> s.lg;
    const long long blocks = s.zero_blocks + (s.tiles + per_block - 1) / per_block * s.col_blocks;
    if (blocks > 0x7fffffffll) return qg_fail(c, QGBDT_ERR_ARG, "rows * bag * dim is too large for one call");
    k_segment_sum<T, V><<<(unsigned)blocks, EMB_THREADS, 0, st>>>(s);
    QG_LAUNCH_CHECK(c);
    if (s.tiles > 1) {
        k_segment_join<T><<<(unsigned)(s.tiles - 1), EMB_THREADS, 0, st>>>(s, log2_at_least(s.dim, 8));
        QG_LAUNCH_CHECK(c);
    }
    return QGBDT_OK;
}

// Calls f<T, V>() for the element type and the vector width in bytes.
#define EMBED_DISPATCH(type, vb, CALL)                                                ((type) == QGBDT_F32 ? ((vb) == 16 ? CALL(float, 4) : (vb) == 8 ? CALL(float, 2) : CALL(float, 1))                            : (type) == QGBDT_BF16                                                                                                           ? ((vb) == 16 ? CALL(__nv_bfloat16, 8) : (vb) == 8 ? CALL(__nv_bfloat16, 4) : (vb) == 4 ? CALL(__nv_bfloat16, 2) : CALL(__nv_bfloat16, 1))          : ((vb) == 16 ? CALL(__half, 8) : (vb) == 8 ? CALL(__half, 4) : (vb) == 4 ? CALL(__half, 2) : CALL(__half, 1)))

}  // namespace

int qg_embed(qgbdt_ctx *c, const EmbedArgs &a, cudaStream_t st) {
    const int vb = vec_bytes(a);
#define CALL(T, V) embed_typed<T, V>(c, a, st)
    return EMBED_DISPATCH(a.type, vb, CALL);
#undef CALL
}

int qg_embed_backward(qgbdt_ctx *c, const EmbedArgs &a, cudaStream_t st) {
    const long long n = a.rows * a.bag;
    const int vb = vec_bytes(a), V = vb / qg_type_size(a.type);
    SegArgs s{};
    s.n = n;
    s.grad = a.table, s.ld = a.ld, s.out = a.out, s.ld_out = a.ld_out, s.n_entries = a.n_entries;
    s.dim = a.dim, s.scale = a.scale;
    s.lg = log2_at_least((a.dim + V - 1) / V, 5);
    s.col_blocks = (a.dim + (V << s.lg) - 1) / (V << s.lg);
    s.zero_blocks = (a.n_entries + ZERO_ROWS - 1) / ZERO_ROWS;
    // tiles: about two rounds of resident groups, at least 16 pairs each
    const long long target = (long long)c->sm_count * 2048 * 2 >> s.lg;
    long long tile = (n * s.col_blocks + target - 1) / target;
    tile = tile < 16 ? 16 : (tile + EMB_UNROLL - 1) / EMB_UNROLL * EMB_UNROLL;
    s.tile = (int)(tile < (1 << 20) ? tile : 1 << 20);
    s.tiles = (n + s.tile - 1) / s.tile;
    const bool small = n <= SORT_SMALL;
    const SortPlan sp = small ? SortPlan{} : sort_plan(c, n, a.n_entries);
    const size_t digits = small ? 0 : (size_t)1 << sp.bits;
    const size_t bytes = 2 * qg_ws_size((size_t)n, sizeof(uint2)) + qg_ws_size(digits * (sp.blocks + 1), sizeof(unsigned)) +
                         qg_ws_size(digits, sizeof(unsigned)) + qg_ws_size((size_t)s.tiles * 2 * a.dim, sizeof(float));
    QgWorkspace ws;
    int rc = qg_ws_open(c, bytes, st, &ws);
    if (rc != QGBDT_OK) return rc;
    uint2 *buf0 = ws.take<uint2>((size_t)n), *buf1 = ws.take<uint2>((size_t)n);
    unsigned *counts = ws.take<unsigned>(digits * sp.blocks), *totals = ws.take<unsigned>(digits);
    s.partial = ws.take<float>((size_t)s.tiles * 2 * a.dim);
    s.pair = buf0;
    if (n > 0) {
        const SortArgs sa{a.tokens, a.ld_tokens, a.n_entries, n, a.bag, a.status};
        rc = a.token_type == QGBDT_I64 ? sort_pairs<int64_t>(c, sa, sp, buf0, buf1, counts, totals, &s.pair, st)
                                       : sort_pairs<int32_t>(c, sa, sp, buf0, buf1, counts, totals, &s.pair, st);
        if (rc != QGBDT_OK) return rc;
    }
#define CALL(T, V) segments_typed<T, V>(c, s, st)
    rc = EMBED_DISPATCH(a.type, vb, CALL);
#undef CALL
    if (rc != QGBDT_OK) return rc;
    return qg_ws_close(c, st);
}
