// Softmax cross entropy of a linear classifier over many classes, without stored logits, and its gradients.
//
//   z = H W^T + b,   lse_i = log sum_v exp z_iv,   loss = mean of lse_i - z_i,label
//   g_iv = exp(z_iv - lse_i) - [v == label i],   dH = s g W,   dW = s g^T H,   db = s sum_i g_i
//
// with s = grad_loss / (rows with a label).  Four matrix products on the tensor cores: z once for the loss,
// z again for the gradients, and the two products with g.  8 * rows * classes * dim operations in all; a step that
// kept the logits would need 6.  Keeping them would cost 4 bytes per logit out of and into DRAM (z has more bits than
// the inputs' type: half that would round it), which at dim 1024 takes as long as working them out again (0.65 ms for
// 537 million), at smaller dim longer, and memory for all of them (2 GB there); what is kept instead is a maximum and
// a sum per row and 128 classes, 8 bytes.
//
// One kernel carries all four: a persistent grid whose pairs of CTAs take tiles of 256 rows by 256 columns.  One
// warp fills a ring of operand tiles with tiled copies, one thread issues the matrix instructions, eight warps
// empty the accumulators, of which tensor memory holds two, so that the epilogue of a tile runs under the
// products of the next.  What the epilogues do:
//   LOSS  per row of the tile: maximum and sum of exponentials; the label's logit.  No logit leaves the SM.
//   GRAD  g of a piece of the classes, rounded to the inputs' type (relative error 2^-9 in bf16, 2^-12 in f16, of
//         each g on its own: as much as the outputs' own rounding, averaged down by the sums that follow; operands of
//         the tensor cores have no more bits, and two of them per g would double the products), and its column sums in
//         single precision for the bias.  Half precision holds 2^15 g: |g| <= 1 leaves it that much room, and without
//         it classes of a probability below 2^-14 would lose bits and below 2^-25 vanish.  With it the error above
//         holds from |g| = 2^-29 on; below it is 2^-40 at most.  The scale s, with 2^-15 in it, is applied behind the
//         sums, to numbers in single precision.
//   DH    the piece's contribution to dH, in single precision.
//   DW    rows of dW, complete with every piece, written in the output type.
//
// Measured (7373 labelled rows x 65536 classes x 1024, bf16, single launches from cold caches): LOSS 671 us, 1.48
// PFLOP/s; GRAD 0.70 ms (its epilogue writes 1 GB of g), DH 0.67 ms, DW 0.64 ms; the whole step in a stream 3.15 ms.
// The tensor cores are busy 75 to 83 % of a launch's time; they and power bound LOSS (1000 W: in a loop 1.25-1.3 PFLOP/s,
// what library products of these shapes reach), what L2 delivers (about 12 TB/s) DH and DW.  With dim below about 400 the
// epilogues bound LOSS and GRAD (dim 64: 537 million logits in 222 us, of which 120 us are what the exponentials alone
// need at 16 per clock and SM; the rest is the latency of an epilogue's steps).
//
// Rows without a label are taken out first, but for the loss at small sizes (DIRECT_PRODUCTS): the labelled rows are
// packed to the front of a copy of H (which also gives the copies their alignment), and nothing is computed for the
// others.  Where the rows are taken as they are, a row's products meet its own statistics alone, and nobody reads those of
// a row without a label: what it holds, infinities included, reaches no result either way.
#include <math.h>

#include <type_traits>

#include "ops_internal.cuh"
#include "tensor_core.cuh"

namespace {

constexpr int CG = 2;                       // CTAs per tile: a pair halves what each SM loads of the second operand
constexpr int BM = 128 * CG, BN = 256, BK = 64;
constexpr int A_BYTES = 128 * BK * 2, B_ROWS = BN / CG, B_BYTES = B_ROWS * BK * 2;
constexpr int EPI_WARPS = 8, THREADS = 128 + EPI_WARPS * 32;
constexpr int STORE_BYTES = 32 * 128;       // staging buffer of a warp: 32 rows of 128 bytes
constexpr int TMEM_COLS = 512, ACC_COLS = 256;
constexpr int GROUP_M = 16;                 // row tiles that go through all column tiles together
constexpr float LOG2E = 1.44269504088896340736f;
constexpr float F16_UP = 32768.0f;          // g in half precision is held as this multiple

enum Mode { LOSS, GRAD, DH, DW };

// NB: accumulators of 256 columns that a tile has.  One: tensor memory holds two tiles, and a tile's epilogue runs
// under the products of the next.  Two (DH and DW with long products): a tile of 512 columns fills tensor memory, the
// epilogue has nothing to run under, but a quarter less comes out of L2 per product, which is what bounds the products
// of 256 columns (32 KB per block of 64 and SM, 12 TB/s).
//
// Shared memory: a ring of operand tiles and the warps' staging buffers.  GRAD stages every tile it makes, so it has two
// buffers per warp and one operand tile less (8192 rows x 16384 classes x 64: 94 us with one, 82 us with two).
template <int MODE, int NB>
struct Layout {
    static constexpr int BUFFERS = MODE == GRAD ? 2 : 1, STAGES = NB == 2 ? 4 : MODE == GRAD ? 5 : 6;
    static constexpr int STAGE_BYTES = A_BYTES + NB * B_BYTES, ACCS = NB == 2 ? 1 : 2;
    static constexpr int BYTES = 1024 + STAGES * STAGE_BYTES + EPI_WARPS * BUFFERS * STORE_BYTES;
};

// The caller's labels.
struct RawLabels {
    const void *p;
    int type, classes;
    __device__ __forceinline__ long long raw(int i) const {
        return type == QGBDT_I64 ? reinterpret_cast<const long long *>(p)[i] : (long long)reinterpret_cast<const int *>(p)[i];
    }
};

struct GemmArgs {
    const int *count;           // labelled rows; NULL: all rows are taken as they are (LOSS)
    int all_rows;
    int m_tiles, n_tiles;       // tiles (LOSS, GRAD, DH: row tiles for all rows; only those with labelled rows are taken)
    int kb;                     // blocks of 64 along the products' length (DW: taken from the count)
    int classes;                // all classes
    int v0;                     // first class of the piece
    int dim;
    int bf16;
    int *fault;
    // LOSS and GRAD
    const float *bias;          // [classes] or NULL
    int bias_vec;               // it is 16-byte aligned
    const int *label;           // [labelled rows], or NULL with all rows:
    RawLabels labels;
    float2 *stat;               // [row][n_tiles * 2] maximum, sum of exp(z - maximum) over 128 columns
    float *z_label;             // [row]
    const float *lse;           // [row]
    float *bias_part;           // [m_tiles * BM / 32][n_tiles * 256] column sums of g over 32 rows
    // DH and DW
    int gang, gangs, rounds;    // units of a gang, gangs, column tiles / gang rounded up
    bool split;                 // tiles may be cut (the same for every launch of a call)
    int add;                    // DH: add to the fragments of the pieces before
    uint16_t *out;              // DW
    int rows;                   // its rows in this piece
    long long ld_out;
    int out_map;                // its rows are 16-byte aligned: tiled copies write them
    const float *grad_loss;
};

__device__ __forceinline__ float out_scale(const float *grad_loss, int count) {
    return (grad_loss ? *grad_loss : 1.0f) / (float)(count > 0 ? count : 1);
}
// The same for sums of products with g as it is held.
__device__ __forceinline__ float product_scale(const float *grad_loss, int count, bool bf16) {
    return out_scale(grad_loss, count) * (bf16 ? 1.0f : 1.0f / F16_UP);
}

// The tiles of LOSS and GRAD in the order in which they are taken: groups of GROUP_M row tiles, in a group all row
// tiles of a column tile before the next, so that CTAs that run together share both operands in L2.  A unit's next tile
// is `step` further on; kept as group and place in it, since divisions would stand in front of every tile's epilogue.
struct TileWalk {
    int m0, rows, place, size;   // first row tile of the group, its row tiles; place in the group, its tiles
    int m_live, n_tiles, step;
    __device__ TileWalk(int m_live_, int n_tiles_, int first, int step_) : m0(0), place(first), m_live(m_live_), n_tiles(n_tiles_), step(step_) { group(); }
    __device__ __forceinline__ void group() { rows = min(GROUP_M, m_live - m0), size = rows * n_tiles; }
    __device__ __forceinline__ bool next(int &m, int &n) {
        while (m0 < m_live && place >= size) place -= size, m0 += GROUP_M, group();
        if (m0 >= m_live) return false;
        n = rows == GROUP_M ? place / GROUP_M : place / rows;
        m = m0 + place - n * rows;
        place += step;
        return true;
    }
};

// DH and DW have few tiles and long products, so whole tiles would leave SMs idle in the last round, and their
// first operand, g, is larger than L2.  Units (pairs of CTAs) work in gangs: the units of a gang take neighbouring
// column tiles of the same rows and walk along the products together, so that a block of g comes out of DRAM once
// for all of them.  All blocks of all row tiles (once per round of column tiles), one after the other, are a line
// that is cut into equal runs, one per gang; a tile that a cut falls into is summed from its fragments afterwards,
// in the order of the gangs.  Short products (below SPLIT_KB blocks) are not cut: joining fragments costs about as
// long as 30 blocks take, so that their runs are whole tiles.
constexpr int SPLIT_KB = 32;
struct Line {
    long long length;   // rounds * row tiles * kb
    int kb, runs;       // gangs that get a run (of four blocks or more)
    bool split;
    __device__ Line(int lines, int kb_, int gangs, bool split_) : length((long long)lines * kb_), kb(kb_), split(split_) {
        const long long most = split ? length / 4 : lines;
        runs = most < 1 ? 1 : most < gangs ? (int)most : gangs;
    }
    // a * b / c; in 32 bits where the line is short enough for that (a 64-bit division takes a hundred instructions)
    __device__ __forceinline__ long long scaled(long long a, int b, long long c) const {
        return length < (1 << 24) && runs < 256 ? (long long)((unsigned)a * (unsigned)b / (unsigned)c) : a * b / c;
    }
    __device__ __forceinline__ long long start(int g) const { return split ? scaled(length, g, runs) : scaled(length / kb, g, runs) * kb; }
    __device__ __forceinline__ int gang_of(long long pos) const {   // the gang whose run holds block pos
        // the last g with floor(length * g / runs) <= pos
        const long long at = split ? pos : pos / kb, all = split ? length : length / kb;
        return (int)(length < (1 << 24) && runs < 256 ? (((unsigned)at + 1) * (unsigned)runs - 1) / (unsigned)all : ((at + 1) * runs - 1) / all);
    }
};

// What a unit works on next.
struct Work {
    int m, n, kb0, kb1;
    int cols;            // columns of the tile; the last ones of DH and DW are cut to a multiple of 128
    int fragment;        // DH, and DW where the tile is not whole: which part buffer
    bool whole;
};
template <int MODE, int NB>
struct Schedule {
    int m_live, n_tiles, dim, kb, unit, gang, member, size;
    TileWalk walk;
    int place, m, round, k;   // DH and DW: the tile the run has come to, its row tile and round, the block in it
    long long left;           // blocks of the run still to come
    __device__ Schedule(const GemmArgs &a, int count, int cta, int ctas)
        : m_live(MODE == DW ? a.m_tiles : (count + BM - 1) / BM), n_tiles(a.n_tiles), dim(a.dim), walk(m_live, n_tiles, cta / CG, ctas / CG) {
        kb = MODE == DW ? (count + BK - 1) / BK : a.kb;
        unit = cta / CG;
        left = 0;
        if (MODE == DH || MODE == DW) {
            size = a.gang, gang = unit / size, member = unit - gang * size;
            const Line line(a.rounds * m_live, kb, a.gangs, a.split);
            if (line.length > 0 && gang < line.runs) {
                const long long pos = line.start(gang);
                left = line.start(gang + 1) - pos;
                place = (int)(pos / kb), k = (int)(pos - (long long)place * kb);
                round = place / m_live, m = place - round * m_live;   // row tiles of round 0, of round 1, ...
            }
        }
    }
    __device__ __forceinline__ bool next(Work &w) {
        if (MODE == LOSS || MODE == GRAD) {
            w.kb0 = 0, w.kb1 = kb, w.cols = BN;
            return walk.next(w.m, w.n);
        } else {
            while (left > 0) {
                w.m = m;
                w.n = round * size + member;
                w.kb0 = k;
                w.kb1 = (int)min((long long)kb, k + left);
                w.whole = w.kb0 == 0 && w.kb1 == kb;
                w.cols = min(BN * NB, (dim - w.n * BN * NB + 127) / 128 * 128);
                w.fragment = MODE == DH ? (place + gang) * size + member : 2 * unit + (w.kb0 == 0);
                left -= w.kb1 - w.kb0;
                k = 0, ++place;
                if (++m == m_live) m = 0, ++round;
                if (w.n < n_tiles) return true;   // the last round may have fewer column tiles than the gang units
            }
            return false;
        }
    }
};

// x[j] summed over the warp's 32 lanes, for j = lane.
__device__ __forceinline__ float column_sums(float (&x)[32], int lane) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < o; ++i) {
            const float give = up ? x[i] : x[i + o], keep = up ? x[i + o] : x[i];
            x[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    return x[0];
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi, bool bf16) {
    if (bf16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// 16 bytes of this lane's row of the staging buffer, in the 128-byte swizzle.
__device__ __forceinline__ void stage16(uint32_t buf, int lane, int chunk, uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + (((uint32_t)chunk ^ (lane & 7)) << 4)), "r"(w0), "r"(w1), "r"(w2),
                 "r"(w3)
                 : "memory");
}

template <int MODE, int NB>
struct Epilogue {
    const GemmArgs &a;
    const CUtensorMap *map_out, *map_part;
    uint32_t buf;          // this warp's staging buffer
    int lane, count;
    Work c;
    int row_in, row;       // the warp's first row, this thread's
    int col0;              // first of the warp's columns (128, with two accumulators 256)
    bool live;
    int label;
    float lse, scale;

    __device__ Epilogue(const GemmArgs &a_, const CUtensorMap *o, const CUtensorMap *p, uint32_t b, int l, int n)
        : a(a_), map_out(o), map_part(p), buf(b), lane(l), count(n) {
        if (MODE == DW) scale = product_scale(a.grad_loss, count, a.bf16);
    }

    // What the next tile's rows need from memory, loaded under this tile's work and not looked at before begin().
    // The bias of the warp's 128 columns: four per lane, minus infinity behind the last class.
    int label_lo, label_hi;
    float lse_next;
    float4 bias_next, bias_now;
    __device__ __forceinline__ void fetch(const Work &w, int rank, int quarter, int half) {
        if (MODE != LOSS && MODE != GRAD) return;
        if (a.bias) {
            const int v = a.v0 + w.n * BN + half * 128 + lane * 4;
            if (a.bias_vec && v + 4 <= a.classes) {
                bias_next = __ldg(reinterpret_cast<const float4 *>(a.bias + v));
            } else {
                bias_next.x = v < a.classes ? __ldg(a.bias + v) : -INFINITY;
                bias_next.y = v + 1 < a.classes ? __ldg(a.bias + v + 1) : -INFINITY;
                bias_next.z = v + 2 < a.classes ? __ldg(a.bias + v + 2) : -INFINITY;
                bias_next.w = v + 3 < a.classes ? __ldg(a.bias + v + 3) : -INFINITY;
            }
        }
        const int r = w.m * BM + rank * 128 + quarter * 32 + lane;
        label_lo = label_hi = -1;
        if (r >= count) return;
        if (a.label) {
            label_lo = a.label[r];
        } else if (a.labels.type == QGBDT_I64) {
            label_lo = reinterpret_cast<const int *>(a.labels.p)[2ll * r], label_hi = reinterpret_cast<const int *>(a.labels.p)[2ll * r + 1];
        } else {
            label_lo = reinterpret_cast<const int *>(a.labels.p)[r];
        }
        if (MODE == GRAD) lse_next = a.lse[r];
    }

    __device__ __forceinline__ void begin(const Work &w, int rank, int quarter, int half) {
        c = w;
        row_in = w.m * BM + rank * 128 + quarter * 32;
        row = row_in + lane;
        col0 = w.n * BN * NB + half * (BN * NB / 2);
        live = row < count;
        if (MODE == LOSS || MODE == GRAD) {   // a label that is none, or out of range, meets no column
            label = live && (unsigned)label_lo < (unsigned)a.classes ? label_lo : -1;
            if (!a.label && a.labels.type == QGBDT_I64 && label_hi != 0) label = -1;
        }
        if (MODE == GRAD) lse = live ? lse_next : 0.0f;
        if ((MODE == LOSS || MODE == GRAD) && a.bias) {
            bias_now = bias_next;
            if (MODE == LOSS) {   // LOSS does not stage anything else: all lanes read the bias from there
                __syncwarp();
                asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 16), "f"(bias_now.x), "f"(bias_now.y), "f"(bias_now.z), "f"(bias_now.w)
                             : "memory");
                __syncwarp();
            }
        }
    }

    // The staging buffer may be written: the copy out of it has been read.
    __device__ __forceinline__ void stage_open() {
        if (lane == 0) tc_store_wait_read<0>();
        __syncwarp();
    }
    // Rows of the buffer are complete: the caller's copy may start (lane 0).
    __device__ __forceinline__ void stage_close() {
        tc_fence_async_smem();
        __syncwarp();
    }
    __device__ __forceinline__ void stage_half(const float (&x)[32], int h) {   // 32 columns as 16-bit elements, left or right half of the buffer
#pragma unroll
        for (int i = 0; i < 4; ++i)
            stage16(buf, lane, h * 4 + i, pack2(x[8 * i], x[8 * i + 1], a.bf16), pack2(x[8 * i + 2], x[8 * i + 3], a.bf16),
                    pack2(x[8 * i + 4], x[8 * i + 5], a.bf16), pack2(x[8 * i + 6], x[8 * i + 7], a.bf16));
    }

    // x = exp(x - base).  The difference first: base * log2(e) would overflow for classes masked by the type's lowest value.
    template <int N>
    __device__ __forceinline__ void exponentials(float (&x)[N], float base) {
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            tc_add2(x[j], x[j + 1], -base, -base);
            tc_mul2(x[j], x[j + 1], LOG2E);
            x[j] = tc_ex2(x[j]), x[j + 1] = tc_ex2(x[j + 1]);
        }
    }

    // Bias, or minus infinity behind the last class, for N logits from the warp's column j0 on.
    template <int N>
    __device__ __forceinline__ void logits(float (&x)[N], int j0) {
        const int v = a.v0 + col0 + j0;
        if (a.bias) {
#pragma unroll
            for (int j = 0; j < N; j += 4) {
                float4 b;
                if (MODE == LOSS) {
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w) : "r"(buf + (j0 + j) * 4));
                } else {
                    const int from = (j0 + j) / 4;
                    b.x = __shfl_sync(0xffffffffu, bias_now.x, from), b.y = __shfl_sync(0xffffffffu, bias_now.y, from);
                    b.z = __shfl_sync(0xffffffffu, bias_now.z, from), b.w = __shfl_sync(0xffffffffu, bias_now.w, from);
                }
                tc_add2(x[j], x[j + 1], b.x, b.y);
                tc_add2(x[j + 2], x[j + 3], b.z, b.w);
            }
        } else if (v + N > a.classes) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (v + j >= a.classes) x[j] = -INFINITY;
        }
    }

    // LOSS: all 128 columns of the warp at once; no logit waits for a running maximum.
    __device__ __forceinline__ void row_statistics(float (&x)[128], int half) {
        const int lj = label - (a.v0 + col0);
        logits(x, 0);
        const bool mine = lj >= 0 && lj < 128;
        if (__any_sync(0xffffffffu, mine)) {
            float z[64];   // x[lj], by the bits of lj
#pragma unroll
            for (int j = 0; j < 64; ++j) z[j] = lj & 64 ? x[j + 64] : x[j];
#pragma unroll
            for (int o = 32; o; o >>= 1)
#pragma unroll
                for (int j = 0; j < o; ++j) z[j] = lj & o ? z[j + o] : z[j];
            if (mine) a.z_label[row] = z[0];
        }
        float t[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int j = 4; j < 124; j += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) t[k] = tc_max3(t[k], x[j + 2 * k], x[j + 2 * k + 1]);
        const float top = fmaxf(fmaxf(tc_max3(t[0], x[124], x[125]), tc_max3(t[1], x[126], x[127])), fmaxf(t[2], t[3])), base = top == -INFINITY ? 0.0f : top;
        exponentials(x, base);
        float s[8] = {};
#pragma unroll
        for (int j = 0; j < 128; j += 8)
#pragma unroll
            for (int k = 0; k < 8; k += 2) tc_add2(s[k], s[k + 1], x[j + k], x[j + k + 1]);
        if (live) a.stat[((long long)row * a.n_tiles + c.n) * 2 + half] = make_float2(top, ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
    }

    // GRAD: 64 columns, left or right half of the warp's.
    __device__ __forceinline__ void gradients(float (&x)[64], int h) {
        const int col = col0 + h * 64, lj = label - (a.v0 + col);
        const bool mine = lj >= 0 && lj < 64;
        logits(x, h * 64);
        exponentials(x, lse);
        if (__any_sync(0xffffffffu, mine)) {
#pragma unroll
            for (int j = 0; j < 64; ++j)
                if (lj == j) x[j] -= 1.0f;
        }
        if (row_in + 32 > count) {
#pragma unroll
            for (int j = 0; j < 64; ++j) x[j] = live ? x[j] : 0.0f;
        }
        if (!a.bf16) {
#pragma unroll
            for (int j = 0; j < 64; j += 2) tc_mul2(x[j], x[j + 1], F16_UP);
        }
        const uint32_t to = buf + h * STORE_BYTES;
        if (lane == 0) tc_store_wait_read<1>();   // the copy out of this buffer has been read
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            stage16(to, lane, i, pack2(x[8 * i], x[8 * i + 1], a.bf16), pack2(x[8 * i + 2], x[8 * i + 3], a.bf16), pack2(x[8 * i + 4], x[8 * i + 5], a.bf16),
                    pack2(x[8 * i + 6], x[8 * i + 7], a.bf16));
        stage_close();
        if (lane == 0) {
            tc_store_2d(map_out, col, row_in, to);
            tc_store_commit();
        }
        if (a.bias_part) {
            float *sums = a.bias_part + (long long)(row_in / 32) * (a.n_tiles * BN) + col + lane;
#pragma unroll
            for (int k = 0; k < 64; k += 32) {
                float y[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) y[j] = x[k + j];
                sums[k] = column_sums(y, lane) * (a.bf16 ? 1.0f : 1.0f / F16_UP);
            }
        }
    }

    // DH and DW: 32 columns, chunk cc of four from column c0 of the warp's on.
    __device__ __forceinline__ void chunk(const uint32_t (&r)[32], int c0, int cc) {
        float x[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j] = __uint_as_float(r[j]);
        const int col = col0 + c0 + cc * 32;
        if (MODE == DW && c.whole) {
            const int v_in = a.v0 + row_in;
            if ((cc & 1) == 0) stage_open();
#pragma unroll
            for (int j = 0; j < 32; ++j) x[j] *= scale;
            stage_half(x, cc & 1);
            if ((cc & 1) == 0) return;
            stage_close();
            const int first = col - 32;   // of 64 columns
            if (a.out_map) {
                if (lane == 0 && first < a.dim && v_in < a.classes) {
                    tc_store_2d(map_out, first, v_in, buf);
                    tc_store_commit();
                }
            } else {   // two columns per lane, row after row
                const int d = first + 2 * lane;
                for (int i = 0; i < 32 && v_in + i < a.classes; ++i) {
                    uint32_t w;
                    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(buf + i * 128 + ((((uint32_t)lane >> 2) ^ (i & 7)) << 4) + (lane & 3) * 4) : "memory");
                    uint16_t *o = a.out + (v_in + i) * a.ld_out + d;
                    if (d < a.dim) o[0] = (uint16_t)w;
                    if (d + 1 < a.dim) o[1] = (uint16_t)(w >> 16);
                }
                __syncwarp();
            }
            return;
        }
        // a fragment, single precision, to its part buffer
        stage_open();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            stage16(buf, lane, i, __float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
        stage_close();
        if (lane == 0) {
            const int y = c.fragment * BM + row_in - c.m * BM, xx = col - c.n * BN * NB;
            if (MODE == DH && a.add) tc_add_2d(map_part, xx, y, buf);
            else tc_store_2d(map_part, xx, y, buf);
            tc_store_commit();
        }
    }
};

// CTA `cta` of `ctas` that work on a product.
template <int MODE, int NB>
__device__ __forceinline__ void softmax_gemm(const GemmArgs &a, const CUtensorMap &map_a, const CUtensorMap &map_b, const CUtensorMap &map_out,
                                             const CUtensorMap &map_part, int cta, int ctas) {
    constexpr bool A_MN = MODE == DW, B_MN = MODE == DH || MODE == DW;   // operand rows run along the products' length
    extern __shared__ char smem_raw[];
    constexpr int STAGES = Layout<MODE, NB>::STAGES, STAGE_BYTES = Layout<MODE, NB>::STAGE_BYTES, ACCS = Layout<MODE, NB>::ACCS;
    __shared__ alignas(8) unsigned long long bars[2 * STAGES + 4 + 1];
    __shared__ uint32_t tmem_base;
    __shared__ int stop;
    const uint32_t tiles_at = (tc_smem(smem_raw) + 1023) & ~1023u, store_at = tiles_at + STAGES * STAGE_BYTES;
    const uint32_t bar0 = tc_smem(bars);
    auto full = [&](int s) { return bar0 + 8 * s; };
    auto empty = [&](int s) { return bar0 + 8 * (STAGES + s); };
    auto acc_full = [&](int b) { return bar0 + 8 * (2 * STAGES + b); };
    auto acc_empty = [&](int b) { return bar0 + 8 * (2 * STAGES + 2 + b); };
    const uint32_t drained = bar0 + 8 * (2 * STAGES + 4);
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0 : tc_cta_rank();

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) tc_bar_init(full(s), 1), tc_bar_init(empty(s), 1);
        for (int b = 0; b < 2; ++b) tc_bar_init(acc_full(b), 1), tc_bar_init(acc_empty(b), EPI_WARPS * CG);
        tc_bar_init(drained, 1);
        tc_bar_init_fence();
        stop = 0;
    }
    if (warp == 2) tc_alloc<CG>(tc_smem(&tmem_base), TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_group_sync<CG>();
    tc_fence_after();
    const uint32_t tmem = *(volatile uint32_t *)&tmem_base;

    qg_after_prior();   // what is above touches no memory of the device
    const int count = a.count ? *a.count : a.all_rows;
    Schedule<MODE, NB> todo(a, count, cta, ctas);
    Work c;
    bool ok = true;

    if (warp == 0 && lane == 0) {
        // ---- copies
        int it = 0;
        while (ok && todo.next(c)) {
            for (int k = c.kb0; k < c.kb1; ++k, ++it) {
                const int s = it % STAGES;
                if (!(ok = tc_bar_wait(empty(s), (it / STAGES & 1) ^ 1, &stop))) break;
                const uint32_t bar = CG == 1 ? full(s) : tc_map_rank(full(s), 0);
                if (rank == 0) tc_bar_expect(full(s), CG * A_BYTES + c.cols * BK * 2);
                const uint32_t at = tiles_at + s * STAGE_BYTES, bt = at + A_BYTES;
                const int am = c.m * BM + rank * 128;
                if (A_MN) {
                    for (int j = 0; j < 2; ++j) tc_load_2d<CG>(at + j * 8192, &map_a, am + 64 * j, k * BK, bar);
                } else {
                    tc_load_2d<CG>(at, &map_a, k * BK, am, bar);
                }
                if (B_MN) {
                    const int y = (MODE == DH ? a.v0 : 0) + k * BK;
                    for (int h = 0; h < NB; ++h) {   // this CTA's part of every accumulator's columns
                        const int part = min(BN, c.cols - h * BN) / CG, x = c.n * BN * NB + h * BN + rank * part;
                        for (int j = 0; j < part / 64; ++j) tc_load_2d<CG>(bt + h * B_BYTES + j * 8192, &map_b, x + 64 * j, y, bar);
                    }
                } else {
                    tc_load_2d<CG>(bt, &map_b, k * BK, a.v0 + c.n * BN + rank * B_ROWS, bar);
                }
            }
        }
        if (!ok) {
            // gave up: the copies under way must land before the CTA ends
            stop = 1;
            *a.fault = 1;
            int never = 0;
            if (rank == 0)
                for (int i = it > STAGES ? it - STAGES : 0; i < it; ++i) tc_bar_wait(full(i % STAGES), i / STAGES & 1, &never);
        }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ---- matrix instructions
        int it = 0, n_acc = 0;
        while (ok && todo.next(c)) {
            uint32_t idesc[NB];
#pragma unroll
            for (int h = 0; h < NB; ++h) idesc[h] = tc_idesc(BM, min(BN, max(c.cols - h * BN, 0)), a.bf16, A_MN, B_MN);
            const int b = n_acc % ACCS;
            if (!(ok = tc_bar_wait(acc_empty(b), (n_acc / ACCS & 1) ^ 1, &stop))) break;
            tc_fence_after();
            for (int k = c.kb0; k < c.kb1; ++k, ++it) {
                const int s = it % STAGES;
                if (!(ok = tc_bar_wait(full(s), it / STAGES & 1, &stop))) break;
                tc_fence_after();
                const uint32_t at = tiles_at + s * STAGE_BYTES, bt = at + A_BYTES;
#pragma unroll
                for (int q = 0; q < BK / 16; ++q) {
                    const uint64_t da = tc_desc(at + q * (A_MN ? 2048 : 32), A_MN ? 8192 : 16);
#pragma unroll
                    for (int h = 0; h < NB; ++h) {
                        const uint64_t db = tc_desc(bt + h * B_BYTES + q * (B_MN ? 2048 : 32), B_MN ? 8192 : 16);
                        if (h == 0 || c.cols > h * BN) tc_mma<CG>(tmem + (b + h) * ACC_COLS, da, db, idesc[h], k > c.kb0 || q > 0);
                    }
                }
                tc_commit<CG>(empty(s));
            }
            if (!ok) break;
            tc_commit<CG>(acc_full(b));
            ++n_acc;
        }
        if (!ok) {
            stop = 1;
            *a.fault = 1;
            int never = 0;
            tc_commit<CG>(drained);
            tc_bar_wait(drained, 0, &never);
        }
    } else if (warp >= 4 && MODE == DW && count == 0) {
        // no labelled row: zeros
        for (int i = cta * EPI_WARPS + warp - 4; i < a.rows; i += ctas * EPI_WARPS)
            for (int d = lane; d < a.dim; d += 32) a.out[(a.v0 + i) * a.ld_out + d] = 0;
    } else if (warp >= 4) {
        // ---- epilogue: thread = row of the tile, half of the columns per warp
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        Epilogue<MODE, NB> epi(a, &map_out, &map_part, store_at + (warp - 4) * Layout<MODE, NB>::BUFFERS * STORE_BYTES, lane, count);
        int n_acc = 0;
        Work following;
        bool more = todo.next(c);
        if (more) epi.fetch(c, (int)rank, quarter, half);
        for (; more; c = following) {
            const int b = n_acc % ACCS;
            epi.begin(c, (int)rank, quarter, half);
            more = todo.next(following);
            if (more) epi.fetch(following, (int)rank, quarter, half);
            if (!(ok = __all_sync(0xffffffffu, tc_bar_wait(acc_full(b), n_acc / ACCS & 1, &stop)))) break;
            tc_fence_after();
            const uint32_t tacc = tmem + ((uint32_t)(quarter * 32) << 16) + b * ACC_COLS + half * (BN * NB / 2);
            auto hand_back = [&]() {   // the accumulator may be filled again
                tc_fence_before();
                __syncwarp();
                if (lane == 0) tc_bar_arrive_cluster(CG == 1 ? acc_empty(b) : tc_map_rank(acc_empty(b), 0));
            };
            if constexpr (MODE == LOSS) {
                uint32_t r[4][32];
                float x[128];
#pragma unroll
                for (int cc = 0; cc < 4; ++cc) tc_ld_32(tacc + cc * 32, r[cc]);
#pragma unroll
                for (int cc = 0; cc < 4; ++cc) {
                    tc_ld_wait(r[cc]);
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[cc * 32 + j] = __uint_as_float(r[cc][j]);
                }
                hand_back();
                epi.row_statistics(x, half);
            } else if constexpr (MODE == GRAD) {
                uint32_t r[4][32];
                tc_ld_32(tacc, r[0]);
                tc_ld_32(tacc + 32, r[1]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h == 1) tc_ld_32(tacc + 96, r[3]);   // (all four at once would not fit the registers)
                    tc_ld_wait(r[2 * h]);
                    tc_ld_wait(r[2 * h + 1]);
                    if (h == 0) tc_ld_32(tacc + 64, r[2]);   // read under the arithmetic of the first half
                    else hand_back();
                    float x[64];
#pragma unroll
                    for (int j = 0; j < 64; ++j) x[j] = __uint_as_float(r[2 * h + j / 32][j % 32]);
                    epi.gradients(x, h);
                }
            } else {
                const int mine = min(BN * NB / 2, c.cols - half * (BN * NB / 2));   // 0 or less: a narrow tile has nothing for this warp
                if (mine <= 0) hand_back();
                for (int c0 = 0; c0 < mine; c0 += 128) {
                    uint32_t r[2][32];
                    tc_ld_32(tacc + c0, r[0]);
#pragma unroll
                    for (int cc = 0; cc < 4; ++cc) {
                        tc_ld_wait(r[cc & 1]);
                        if (cc < 3) tc_ld_32(tacc + c0 + (cc + 1) * 32, r[(cc + 1) & 1]);   // read under the arithmetic of this chunk
                        else if (c0 + 128 >= mine) hand_back();
                        epi.chunk(r[cc & 1], c0, cc);
                    }
                }
            }
            ++n_acc;
        }
        if (!ok) {
            stop = 1;
            *a.fault = 1;
        }
        if (MODE != LOSS && lane == 0) tc_store_wait();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_group_sync<CG>();
    tc_fence_after();
    if (warp == 2) tc_dealloc<CG>(tmem, TMEM_COLS);
}

template <int MODE, int NB>
__global__ void __launch_bounds__(THREADS, 1) k_softmax_gemm(const GemmArgs a, const __grid_constant__ CUtensorMap map_a,
                                                             const __grid_constant__ CUtensorMap map_b,
                                                             const __grid_constant__ CUtensorMap map_out,
                                                             const __grid_constant__ CUtensorMap map_part) {
    softmax_gemm<MODE, NB>(a, map_a, map_b, map_out, map_part, blockIdx.x, gridDim.x);
}

// DH and DW in one launch, each on a part of the units, where the products are so short that a launch counts.
__global__ void __launch_bounds__(THREADS, 1) k_softmax_both(const GemmArgs dh, const GemmArgs dw, int dh_ctas, const __grid_constant__ CUtensorMap g_k,
                                                             const __grid_constant__ CUtensorMap w_mn, const __grid_constant__ CUtensorMap dh_part,
                                                             const __grid_constant__ CUtensorMap g_mn, const __grid_constant__ CUtensorMap h_mn,
                                                             const __grid_constant__ CUtensorMap dw_out) {
    if ((int)blockIdx.x < dh_ctas) softmax_gemm<DH, 1>(dh, g_k, w_mn, dh_part, dh_part, blockIdx.x, dh_ctas);
    else softmax_gemm<DW, 1>(dw, g_mn, h_mn, dw_out, dw_out, blockIdx.x - dh_ctas, gridDim.x - dh_ctas);
}

// ---- rows with a label, packed -----------------------------------------------------------------------

constexpr int PACK_THREADS = 256, PACK_ROWS = 16;   // rows per block: two per warp
constexpr int PACK_SPAN = 2048;                     // labels per entry of the counts
constexpr int PACK_DIRECT = 8192;                   // up to here every block counts all labels itself

// Copy of a matrix whose rows do not start on 16-byte boundaries, with rows that do.
struct RealignArgs {
    const uint16_t *in;
    long long ld, rows;
    int dim;
    uint16_t *out;
    int ldp;       // a multiple of 8
    int blocks;    // 0: there is nothing to copy
};

__device__ __forceinline__ void realign(const RealignArgs &w, int block) {
    const int chunks = w.ldp / 8;
    for (long long i = block * (long long)PACK_THREADS + threadIdx.x; i < w.rows * chunks; i += (long long)w.blocks * PACK_THREADS) {
        const long long r = i / chunks;
        const int d = (int)(i - r * chunks) * 8;
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = w.in[r * w.ld + min(d + j, w.dim - 1)];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = d + j < w.dim ? x[j] : 0u;
        *reinterpret_cast<uint4 *>(w.out + r * w.ldp + d) = make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
    }
}

struct PackArgs {
    RawLabels labels;
    int n, n_pad;              // rows; rows of the packed copy (a multiple of the tile)
    const uint16_t *hidden;    // 16-bit elements, moved as they are
    long long ld;
    int dim, vec;              // vec: rows can be read 16 bytes at a time
    const float *lse;          // or NULL
    int *span_count;           // [spans], for more than PACK_DIRECT labels
    // results
    int *count, *pos_of, *label;
    float *lse_packed;
    uint16_t *packed;          // [n_pad][ldp]
    int ldp;
    int *status;
};

__device__ __forceinline__ int block_sum_int(int s) {
    __shared__ int w[PACK_THREADS / 32];
    s = __reduce_add_sync(0xffffffffu, s);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) w[threadIdx.x / 32] = s;
    __syncthreads();
    s = 0;
#pragma unroll
    for (int i = 0; i < PACK_THREADS / 32; ++i) s += w[i];
    return s;
}

// Labelled rows among this thread's share of [i0, i1): in front of `mark`, and all.  Eight labels are loaded at a time.
__device__ __forceinline__ void count_labels(const PackArgs &a, int i0, int i1, int mark, int &before, int &all) {
    for (int i = i0 + threadIdx.x; i < i1; i += PACK_THREADS * 8) {
        long long l[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) l[u] = a.labels.raw(min(i + u * PACK_THREADS, i1 - 1));
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int at = i + u * PACK_THREADS, has = at < i1 && l[u] >= 0 && l[u] < a.labels.classes;
            all += has;
            before += at < mark ? has : 0;
        }
    }
}

__global__ void __launch_bounds__(PACK_THREADS) k_pack_count(const PackArgs a) {
    qg_after_prior();
    int s = 0, none = 0;
    count_labels(a, blockIdx.x * PACK_SPAN, min(a.n, (int)(blockIdx.x + 1) * PACK_SPAN), 0, none, s);
    s = block_sum_int(s);
    if (threadIdx.x == 0) a.span_count[blockIdx.x] = s;
}

// The blocks behind those that pack copy the weight.
__global__ void __launch_bounds__(PACK_THREADS) k_pack(const PackArgs a, const RealignArgs w) {
    qg_after_prior();
    if ((int)blockIdx.x >= (int)gridDim.x - w.blocks) {
        realign(w, blockIdx.x - (gridDim.x - w.blocks));
        return;
    }
    __shared__ int place[PACK_ROWS];   // where the block's rows go, -1: no label
    const int r0 = blockIdx.x * PACK_ROWS;
    int before = 0, all = 0;
    if (a.n <= PACK_DIRECT) {
        count_labels(a, 0, a.n, r0, before, all);
    } else {
        const int spans = (a.n + PACK_SPAN - 1) / PACK_SPAN, span = r0 / PACK_SPAN;
        int rest = 0;
        for (int s = threadIdx.x; s < spans; s += PACK_THREADS) {
            const int x = a.span_count[s];
            all += x;
            before += s < span ? x : 0;
        }
        count_labels(a, span * PACK_SPAN, min(a.n, r0), r0, before, rest);
    }
    before = block_sum_int(before);
    all = block_sum_int(all);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = all;
    if (threadIdx.x < 32) {
        const int i = r0 + threadIdx.x;
        const long long l = threadIdx.x < PACK_ROWS && i < a.n ? a.labels.raw(i) : -1;
        const bool labelled = l >= 0 && l < a.labels.classes;
        if (l >= a.labels.classes && a.status) *a.status = 1;
        const unsigned has = __ballot_sync(0xffffffffu, labelled);
        const int p = labelled ? before + __popc(has & ((1u << threadIdx.x) - 1)) : -1;
        if (threadIdx.x < PACK_ROWS) {
            place[threadIdx.x] = p;
            if (i < a.n) a.pos_of[i] = p;
        }
        if (labelled) {
            a.label[p] = (int)l;
            if (a.lse) a.lse_packed[p] = a.lse[i];
        }
    }
    __syncthreads();
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, chunks = a.ldp / 8;   // ldp is a multiple of 8
    for (int h = warp; h < PACK_ROWS; h += PACK_THREADS / 32) {
        if (place[h] >= 0) {
            const uint16_t *in = a.hidden + (r0 + h) * a.ld;
            uint4 *out = reinterpret_cast<uint4 *>(a.packed + (long long)place[h] * a.ldp);
            if (a.vec) {
                const uint4 *q = reinterpret_cast<const uint4 *>(in);
#pragma unroll 4
                for (int k = lane; k < chunks; k += 32) out[k] = q[k];
            } else {
                for (int k = lane; k < chunks; k += 32) {
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = in[min(8 * k + j, a.dim - 1)];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = 8 * k + j < a.dim ? w[j] : 0u;
                    out[k] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
                }
            }
        }
        if (r0 + h >= all && r0 + h < a.n_pad) {   // rows behind the last labelled one: zeros
            uint4 *out = reinterpret_cast<uint4 *>(a.packed + (long long)(r0 + h) * a.ldp);
            for (int k = lane; k < chunks; k += 32) out[k] = make_uint4(0, 0, 0, 0);
        }
    }
}

__global__ void __launch_bounds__(PACK_THREADS) k_realign(const RealignArgs w) {
    qg_after_prior();
    realign(w, blockIdx.x);
}

// ---- few rows -----------------------------------------------------------------------------------------
// Scoring a handful of rows reads the weight once and does next to nothing with it: no packing, no tiles.  A warp
// takes a few classes at a time, 16 bytes of each per lane, multiplies them with one or two rows of H and adds the
// lanes' products in a tree that leaves every lane with one class; its statistics stay in registers until the end.
// Bound by the weight's way out of DRAM (or L2).  From three rows on the tiles are faster: 32000 classes x 512, loss
// from start to end, tiles against this: one row 15.9 and 10.4 us, two 15.9 and 11.7; three 16.0 and, with a four-row variant, 19.2.

constexpr int FEW_ROWS = 2, FEW_CLASSES = 4, FEW_WARPS = 4, FEW_BLOCKS = 5;   // blocks per SM

struct FewArgs {
    const uint16_t *hidden, *weight;
    long long ld_hidden, ld_weight;
    int rows, classes, dim;        // rows of both start on 16 bytes, dim is a multiple of 8
    const float *bias;
    const void *labels;
    int label_type;
    float2 *stat;                  // [rows][gridDim.x]
    float *z_label;
    unsigned *arrived;
    float *loss, *losses, *lse;
    int *status;
};

template <typename T, int R>
__global__ void __launch_bounds__(FEW_WARPS * 32, FEW_BLOCKS) k_loss_few(const FewArgs a) {
    qg_after_prior();
    __shared__ float2 part[FEW_WARPS][R];
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    int label[R], rows = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        long long l = -1;
        if (r < a.rows) l = a.label_type == QGBDT_I64 ? reinterpret_cast<const long long *>(a.labels)[r] : (long long)reinterpret_cast<const int *>(a.labels)[r];
        label[r] = l >= 0 && l < a.classes ? (int)l : -1;
        rows += label[r] >= 0;
        if (blockIdx.x == 0 && threadIdx.x == 0 && l >= a.classes && a.status) *a.status = 1;
    }
    float m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) m[r] = -INFINITY, l[r] = 0.0f;
    const int mine = (lane & 16 ? 2 : 0) + (lane & 8 ? 1 : 0);   // class of the four whose sum this lane gets
    for (int v0 = (blockIdx.x * FEW_WARPS + warp) * FEW_CLASSES; v0 < a.classes; v0 += gridDim.x * FEW_WARPS * FEW_CLASSES) {
        float acc[R][FEW_CLASSES];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < FEW_CLASSES; ++j) acc[r][j] = 0.0f;
#pragma unroll 2
        for (int d = lane * 8; d < a.dim; d += 256) {
            OpsVec<T, 8> w[FEW_CLASSES], h[R];
#pragma unroll
            for (int j = 0; j < FEW_CLASSES; ++j)
                w[j] = *reinterpret_cast<const OpsVec<T, 8> *>(a.weight + (long long)min(v0 + j, a.classes - 1) * a.ld_weight + d);
#pragma unroll
            for (int r = 0; r < R; ++r) h[r] = *reinterpret_cast<const OpsVec<T, 8> *>(a.hidden + (long long)min(r, a.rows - 1) * a.ld_hidden + d);
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int j = 0; j < FEW_CLASSES; ++j) acc[r][j] = __fmaf_rn(OpsType<T>::load(w[j].v[k]), OpsType<T>::load(h[r].v[k]), acc[r][j]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int o = 16, n = 2; o >= 8; o >>= 1, n >>= 1) {
                const bool up = lane & o;
#pragma unroll
                for (int j = 0; j < n; ++j) {
                    const float give = up ? acc[r][j] : acc[r][j + n], keep = up ? acc[r][j + n] : acc[r][j];
                    acc[r][j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                }
            }
            float z = acc[r][0];
#pragma unroll
            for (int o = 4; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
            const int v = v0 + mine;
            if (v < a.classes && (lane & 7) == 0) {
                if (a.bias) z += a.bias[v];
                if (v == label[r]) a.z_label[r] = z;
                const float top = fmaxf(m[r], z), base = top == -INFINITY ? 0.0f : top;
                l[r] = l[r] * tc_ex2((m[r] - base) * LOG2E) + tc_ex2((z - base) * LOG2E);
                m[r] = top;
            }
        }
    }
    auto join = [](float &m, float &l, float m2, float l2) {
        const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
        l = l * tc_ex2((m - base) * LOG2E) + l2 * tc_ex2((m2 - base) * LOG2E);
        m = top;
    };
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int o = 16; o >= 8; o >>= 1) join(m[r], l[r], __shfl_xor_sync(0xffffffffu, m[r], o), __shfl_xor_sync(0xffffffffu, l[r], o));
        if (lane == 0) part[warp][r] = make_float2(m[r], l[r]);
    }
    __syncthreads();
    if (threadIdx.x < R && threadIdx.x < a.rows) {
        float2 s = part[0][threadIdx.x];
        for (int w = 1; w < FEW_WARPS; ++w) join(s.x, s.y, part[w][threadIdx.x].x, part[w][threadIdx.x].y);
        a.stat[threadIdx.x * gridDim.x + blockIdx.x] = s;
    }
    // the block that comes last joins the blocks' statistics, a warp per row
    __shared__ bool last;
    __shared__ float row_loss[R];
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.arrived, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
#pragma unroll
    for (int r = 0; r < R; ++r) {   // all threads for a row after the other; eight statistics in flight each
        if (r >= a.rows) break;
        float m0 = -INFINITY, l0 = 0.0f;
        const float2 *q = a.stat + r * gridDim.x;
        for (int t = threadIdx.x; t < (int)gridDim.x; t += FEW_WARPS * 32 * 8) {
            float2 s[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) s[u] = __ldcg(q + min(t + u * FEW_WARPS * 32, (int)gridDim.x - 1));
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (t + u * FEW_WARPS * 32 < (int)gridDim.x) join(m0, l0, s[u].x, s[u].y);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) join(m0, l0, __shfl_xor_sync(0xffffffffu, m0, o), __shfl_xor_sync(0xffffffffu, l0, o));
        __syncthreads();
        if (lane == 0) part[warp][r] = make_float2(m0, l0);
    }
    __syncthreads();
    if (threadIdx.x < R && threadIdx.x < a.rows) {
        float2 s = part[0][threadIdx.x];
        for (int w = 1; w < FEW_WARPS; ++w) join(s.x, s.y, part[w][threadIdx.x].x, part[w][threadIdx.x].y);
        const bool labelled = (threadIdx.x == 0 ? label[0] : label[R - 1]) >= 0;
        const float lse = labelled ? s.x + logf(s.y) : 0.0f, loss = labelled ? lse - __ldcg(a.z_label + threadIdx.x) : 0.0f;
        a.lse[threadIdx.x] = lse;
        if (a.losses) a.losses[threadIdx.x] = loss;
        row_loss[threadIdx.x] = loss;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double sum = 0.0;
        for (int r = 0; r < a.rows; ++r) sum += (double)row_loss[r];
        *a.loss = (float)(sum / (double)(rows > 0 ? rows : 1));
        *a.arrived = 0;
    }
}

// ---- loss from the tiles' statistics -------------------------------------------------------------------

constexpr int JOIN_THREADS = 256;

struct JoinArgs {
    const float2 *stat;
    int n_tiles;             // statistics per row
    const float *z_label;
    const int *pos_of;       // place of a row among the packed ones, -1: no label; NULL: rows are in their own places,
    RawLabels labels;        // and these are their labels
    int n, lg;               // rows; log2 of the lanes per row
    float *losses, *lse;
    double *block_loss;
    int *block_count;
    unsigned *arrived;
    float *loss;
    int *status;
};

__global__ void __launch_bounds__(JOIN_THREADS) k_loss_join(const JoinArgs a) {
    qg_after_prior();
    __shared__ double w[JOIN_THREADS / 32];
    __shared__ int counts[JOIN_THREADS / 32];
    __shared__ bool last;
    const int lg = a.lg, n = a.n, n_tiles = a.n_tiles;
    const int lanes = 1 << lg, lane = threadIdx.x & (lanes - 1), row = blockIdx.x * (JOIN_THREADS >> lg) + (threadIdx.x >> lg);
    int p = -1;
    if (row < n) {
        if (a.pos_of) {
            p = a.pos_of[row];
        } else {
            const long long y = a.labels.raw(row);
            p = y >= 0 && y < a.labels.classes ? row : -1;
            if (y >= a.labels.classes && lane == 0 && a.status) *a.status = 1;
        }
    }
    float mine = 0.0f, m = -INFINITY, l = 0.0f;
    const float z = p >= 0 ? a.z_label[p] : 0.0f;
    if (p >= 0) {
        const float2 *q = a.stat + (long long)p * n_tiles;
        for (int t = lane; t < n_tiles; t += lanes * 8) {
            float2 s[8];
            float top = m;
#pragma unroll
            for (int u = 0; u < 8; ++u) s[u] = q[min(t + u * lanes, n_tiles - 1)];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (t + u * lanes >= n_tiles) s[u] = make_float2(-INFINITY, 0.0f);
                top = fmaxf(top, s[u].x);
            }
            const float base = top == -INFINITY ? 0.0f : top;
            l *= tc_ex2((m - base) * LOG2E);
#pragma unroll
            for (int u = 0; u < 8; ++u) l += s[u].y * tc_ex2((s[u].x - base) * LOG2E);
            m = top;
        }
    }
    for (int o = lanes / 2; o; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
        const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
        l = l * tc_ex2((m - base) * LOG2E) + l2 * tc_ex2((m2 - base) * LOG2E);
        m = top;
    }
    if (row < n && lane == 0) {
        const float l_out = p >= 0 ? m + logf(l) : 0.0f;
        if (p >= 0) mine = l_out - z;
        a.lse[row] = l_out;
        if (a.losses) a.losses[row] = mine;
    }
    const int labelled = __syncthreads_count(p >= 0 && lane == 0);
    double sum = (double)mine;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) w[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int i = 0; i < JOIN_THREADS / 32; ++i) s += w[i];
        a.block_loss[blockIdx.x] = s;
        a.block_count[blockIdx.x] = labelled;
        __threadfence();
        last = atomicAdd(a.arrived, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    // the block that comes last adds the blocks' sums, in their order
    __threadfence();
    double s = 0.0;
    int count = 0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += JOIN_THREADS) s += *(volatile double *)&a.block_loss[i], count += *(volatile int *)&a.block_count[i];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    count = __reduce_add_sync(0xffffffffu, count);
    if ((threadIdx.x & 31) == 0) w[threadIdx.x / 32] = s, counts[threadIdx.x / 32] = count;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0, count = 0;
        for (int i = 0; i < JOIN_THREADS / 32; ++i) s += w[i], count += counts[i];
        *a.loss = (float)(s / (double)(count > 0 ? count : 1));
        *a.arrived = 0;
    }
}

// ---- gradients out of single-precision fragments ---------------------------------------------------------

// Four columns of a tile's row: the sum over its fragments.
__device__ __forceinline__ void add4(float4 &s, const float *p) {
    const float4 x = *reinterpret_cast<const float4 *>(p);
    s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
}

template <typename T>
__device__ __forceinline__ void write4(T *o, int left, const float4 &s, float scale) {
    OpsVec<T, 4> y;
    y.v[0] = OpsType<T>::store(s.x * scale), y.v[1] = OpsType<T>::store(s.y * scale);
    y.v[2] = OpsType<T>::store(s.z * scale), y.v[3] = OpsType<T>::store(s.w * scale);
    if (left >= 4 && reinterpret_cast<uintptr_t>(o) % sizeof(y) == 0) {
        *reinterpret_cast<OpsVec<T, 4> *>(o) = y;
    } else {
        for (int j = 0; j < 4 && j < left; ++j) o[j] = y.v[j];
    }
}

// The fragments of the pieces of one width.
struct DhParts {
    const float *part;   // NULL: there is no such piece
    int tn, gang, gangs, rounds, kb;
    bool split;
};

// Bias gradient of a piece: sums over groups of 32 rows, in their order; 32 columns per block.
struct BiasArgs {
    const float *part;
    int cols, n;          // cols is a multiple of 256
    float *out;
    int blocks;           // 0: no bias
};

__device__ __forceinline__ void bias_finish(const BiasArgs &b, int block, const float *grad_loss, int count) {
    __shared__ float w[8][32];
    const int v = block * 32 + (threadIdx.x & 31), k = threadIdx.x / 32;
    const int groups = (count + BM - 1) / BM * (BM / 32);
    float s = 0.0f;
#pragma unroll 4
    for (int g = k; g < groups; g += 8) s += b.part[(long long)g * b.cols + v];
    w[k][threadIdx.x & 31] = s;
    __syncthreads();
    if (k == 0 && v < b.n) {
        for (int j = 1; j < 8; ++j) s += w[j][threadIdx.x];
        b.out[v] = count > 0 ? s * out_scale(grad_loss, count) : 0.0f;
    }
}

__global__ void __launch_bounds__(256) k_bias_finish(const BiasArgs b, const float *grad_loss, const int *count) {
    qg_after_prior();
    bias_finish(b, blockIdx.x, grad_loss, *count);
}

// dH: every row of the caller's, zeros where it has no label.  2^lg threads per row, four columns each; where a row has many
// fragments, 2^lg_parts such sets of threads share them (75 fragments a row: all gradients of 300 rows x 30000
// classes x 500 88 us without and 83 with, of 3 x 30000 x 100 47 and 39).  The
// blocks behind these finish the bias of the last piece.
template <typename T>
__global__ void __launch_bounds__(256) k_dh_finish(const DhParts full, const DhParts rest, const int *pos_of, int rows, int dim, const float *grad_loss,
                                                   const int *count, T *out, long long ld_out, int lg, int lg_parts, const BiasArgs bias) {
    qg_after_prior();
    __shared__ float4 part_sum[256];
    if ((int)blockIdx.x >= (int)gridDim.x - bias.blocks) {
        bias_finish(bias, blockIdx.x - (gridDim.x - bias.blocks), grad_loss, *count);
        return;
    }
    const int lane = threadIdx.x & ((1 << lg) - 1), parts = 1 << lg_parts, part = threadIdx.x >> lg & (parts - 1);
    const int r = blockIdx.x * (256 >> lg >> lg_parts) + (threadIdx.x >> lg >> lg_parts);
    const int n = *count, p = r < rows ? pos_of[r] : -1, m_live = (n + BM - 1) / BM;
    const float scale = p >= 0 ? product_scale(grad_loss, n, std::is_same<T, __nv_bfloat16>::value) : 0.0f;   // (an infinite grad_loss times 0 would be NaN)
    // of one set: the gangs g0 to g1 that worked on the row's tile in a round
    struct Span {
        int round = -1, place, g0, g1;
    } span[2];
    auto add = [&](float4 &s, const DhParts &x, Span &w, int d) {
        const int now = d / x.tn / x.gang, member = d / x.tn - now * x.gang;
        if (now != w.round) {
            const Line line(x.rounds * m_live, x.kb, x.gangs, x.split);
            w.round = now, w.place = now * m_live + p / BM;
            w.g0 = line.gang_of((long long)w.place * x.kb), w.g1 = line.gang_of((long long)(w.place + 1) * x.kb - 1);
        }
#pragma unroll 4
        for (int g = w.g0 + part; g <= w.g1; g += parts) add4(s, x.part + (((long long)(w.place + g) * x.gang + member) * BM + p % BM) * x.tn + d % x.tn);
    };
    for (int d0 = 0; d0 < dim; d0 += 4 << lg) {
        const int d = d0 + lane * 4;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (p >= 0 && d < dim) {
            add(s, full, span[0], d);
            if (rest.part) add(s, rest, span[1], d);
        }
        if (lg_parts) {
            part_sum[threadIdx.x] = s;
            __syncthreads();
            if (part == 0)
                for (int k = 1; k < parts; ++k) {
                    const float4 y = part_sum[threadIdx.x + (k << lg)];
                    s.x += y.x, s.y += y.y, s.z += y.z, s.w += y.w;
                }
            __syncthreads();
        }
        if (r < rows && part == 0 && d < dim) write4(out + r * ld_out + d, dim - d, s, scale);
    }
}

// dW: the tiles that a cut falls into; blocks x look at the cut in front of gang x / gang + 1 and the tile of member
// x % gang, blocks y take 8 rows.
template <typename T>
__global__ void __launch_bounds__(256) k_dw_finish(const float *part, int tn, int gang, int gangs, int rounds, int m_tiles, int n_tiles, int rows, int dim,
                                                   const float *grad_loss, const int *count, T *out, long long ld_out) {
    qg_after_prior();
    const int n = *count, kb = (n + BK - 1) / BK;
    if (n == 0) return;
    const Line line(rounds * m_tiles, kb, gangs, true);
    const int g = blockIdx.x / gang + 1, member = blockIdx.x % gang;
    if (g >= line.runs) return;
    const long long cut = line.start(g);
    const int place = (int)(cut / kb);
    if (cut == (long long)place * kb) return;
    const int g0 = line.gang_of((long long)place * kb), g1 = line.gang_of((long long)(place + 1) * kb - 1);
    if (g0 != g - 1) return;   // an earlier cut of the same tile
    const float scale = product_scale(grad_loss, n, std::is_same<T, __nv_bfloat16>::value);
    const int round = place / m_tiles, m = place - round * m_tiles, col = (round * gang + member) * tn;
    const int r = blockIdx.y * 8 + threadIdx.x / 32;
    if (m * BM + r >= rows) return;
    for (int d = (threadIdx.x & 31) * 4; d < tn && col + d < dim; d += 128) {
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int k = g0; k <= g1; ++k) add4(s, part + ((long long)(2 * (k * gang + member) + (k == g0)) * BM + r) * tn + d);
        write4(out + (long long)(m * BM + r) * ld_out + col + d, dim - col - d, s, scale);
    }
}

// ---- launches ----------------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encoder(qgbdt_ctx *c, EncodeTiled *out) {
    static EncodeTiled found = nullptr;   // the same for every context; two threads would store the same value
    if (!found) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        QG_CUDA(c, cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q));
        if (q != cudaDriverEntryPointSuccess || !fn) return qg_fail(c, QGBDT_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
        found = reinterpret_cast<EncodeTiled>(fn);
    }
    *out = found;
    return QGBDT_OK;
}

// Matrix [rows][ld] copied in boxes of 128 bytes by `box` rows, 128-byte swizzle, zeros outside.
int matrix_map(qgbdt_ctx *c, CUtensorMap *m, const void *p, long long cols, long long rows, long long ld, int box, int type) {
    EncodeTiled encode = nullptr;
    int rc = encoder(c, &encode);
    if (rc != QGBDT_OK) return rc;
    const int width = qg_type_size(type);
    const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)ld * width};
    const cuuint32_t b[2] = {128u / width, (cuuint32_t)box}, one[2] = {1, 1};
    const CUtensorMapDataType t = type == QGBDT_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                  : type == QGBDT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                       : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const CUresult r = encode(m, t, 2, const_cast<void *>(p), size, stride, b, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return qg_fail(c, QGBDT_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
    return QGBDT_OK;
}

// Launches a kernel of `units` pairs of CTAs; `bit`: which of the context's kernels it is.
template <typename... P, typename... A>
int pairs(qgbdt_ctx *c, int bit, int smem, void (*kernel)(P...), int units, cudaStream_t st, const A &...args) {
    if (!(c->ops_configured >> bit & 1)) {
        QG_CUDA(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        c->ops_configured |= 1u << bit;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)units * CG);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CG, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    QG_CUDA(c, cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
    c->n_launches++;
    return QGBDT_OK;
}

template <int MODE, int NB>
int gemm(qgbdt_ctx *c, const GemmArgs &a, int units, const CUtensorMap &ma, const CUtensorMap &mb, const CUtensorMap &mo, const CUtensorMap &mp,
         cudaStream_t st) {
    return pairs(c, MODE * 2 + NB - 1, Layout<MODE, NB>::BYTES, k_softmax_gemm<MODE, NB>, units, st, a, ma, mb, mo, mp);
}

int up(int64_t x, int m) { return (int)((x + m - 1) / m * m); }

bool rows_aligned(const void *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }

// The weight with rows that start on 16 bytes: itself, or a copy.
struct Weight {
    const void *p;
    long long ld;
};
size_t weight_bytes(const SoftmaxArgs &a) { return rows_aligned(a.weight, a.ld_weight) ? 0 : qg_ws_size((size_t)a.classes * up(a.dim, 8), 2); }

// Where the weight is read from, and the copy to be made for it.
Weight align_weight(const qgbdt_ctx *c, const SoftmaxArgs &a, QgWorkspace &ws, RealignArgs *copy) {
    *copy = RealignArgs{};
    if (weight_bytes(a) == 0) return Weight{a.weight, a.ld_weight};
    const int ldp = up(a.dim, 8);
    uint16_t *to = ws.take<uint16_t>((size_t)a.classes * ldp);
    const long long blocks = (a.classes * (ldp / 8) + PACK_THREADS - 1) / PACK_THREADS, most = c->sm_count * 16;
    *copy = RealignArgs{reinterpret_cast<const uint16_t *>(a.weight), a.ld_weight, a.classes, a.dim, to, ldp, (int)(blocks < most ? blocks : most)};
    return Weight{to, ldp};
}

// The packed rows.
size_t pack_bytes(const SoftmaxArgs &a) {
    const int n_pad = up(a.rows, 256), ldp = up(a.dim, 8);
    return qg_ws_size((size_t)n_pad * ldp, 2) + 3 * qg_ws_size((size_t)n_pad, 4) + qg_ws_size(1, 4) + qg_ws_size((size_t)a.rows / PACK_SPAN + 1, 4);
}

int pack_rows(qgbdt_ctx *c, const SoftmaxArgs &a, QgWorkspace &ws, const RealignArgs &copy, PackArgs *out, cudaStream_t st) {
    PackArgs p{};
    p.labels = RawLabels{a.labels, a.label_type, (int)a.classes};
    p.n = (int)a.rows, p.n_pad = up(a.rows, 256), p.ldp = up(a.dim, 8);
    p.hidden = reinterpret_cast<const uint16_t *>(a.hidden), p.ld = a.ld_hidden, p.dim = a.dim;
    p.vec = rows_aligned(a.hidden, a.ld_hidden) && a.dim % 8 == 0;
    p.lse = a.lse_in, p.status = a.status;
    p.packed = ws.take<uint16_t>((size_t)p.n_pad * p.ldp);
    p.pos_of = ws.take<int>(p.n_pad), p.label = ws.take<int>(p.n_pad), p.lse_packed = ws.take<float>(p.n_pad);
    p.count = ws.take<int>(1);
    p.span_count = ws.take<int>(a.rows / PACK_SPAN + 1);
    *out = p;
    if (a.rows > PACK_DIRECT) QG_RUN(qg_launch(c, k_pack_count, dim3((unsigned)((a.rows + PACK_SPAN - 1) / PACK_SPAN)), PACK_THREADS, 0, st, p));
    return qg_launch(c, k_pack, dim3((p.n_pad > 0 ? p.n_pad / PACK_ROWS : 1) + copy.blocks), PACK_THREADS, 0, st, p, copy);
}

GemmArgs gemm_args(qgbdt_ctx *c, const SoftmaxArgs &a) {
    GemmArgs g{};
    g.classes = (int)a.classes, g.dim = a.dim, g.bf16 = a.type == QGBDT_BF16, g.fault = c->ops_fault;
    g.bias = a.bias, g.bias_vec = reinterpret_cast<uintptr_t>(a.bias) % 16 == 0, g.grad_loss = a.grad_loss;
    g.m_tiles = up(a.rows, 256) / BM, g.kb = (a.dim + BK - 1) / BK;
    return g;
}

// Units (pairs of CTAs) for a number of tiles; -1: more tiles than a launch can number.
int unit_count(const qgbdt_ctx *c, long long tiles) {
    const int units = c->sm_count / CG;
    if (tiles > 0x3fffffff) return -1;
    return tiles < 1 ? 1 : tiles < units ? (int)tiles : units;
}

// Gangs for products with `lines` row tiles of kb blocks each and n_tiles column tiles: of the sizes up to eight that
// leave at most 6 % of the units without work the largest, or else the size that leaves the fewest.
// Gradients of 8192 rows x 65536 classes x 1024: 2.77 ms with one accumulator throughout, 2.69 ms with this rule; without its
// conditions 1024 x 32000 x 768 went from 140 to 160 us, 512 x 65536 x 512 from 127 to 135, 2048 x 65536 x 1024 from 641 to 672.
constexpr long long WIDE_RUN = 128, WIDE_OPERAND = 48ll << 20;
struct Gangs {
    int size, gangs, rounds;
    bool split;
    int tn, n_tiles;   // columns of a tile, tiles
    int units() const { return size * gangs; }
};
Gangs gang_plan(int units, long long m_tiles, int dim, long long kb, int join_cost) {
    auto plan = [&](int tn) {
        const int n_tiles = (dim + tn - 1) / tn;
        Gangs best{1, units, n_tiles, false, tn, n_tiles};
        double best_use = 0.0;
        for (int g = 1; g <= 8 && g <= n_tiles && g <= units; ++g) {
            const int rounds = (n_tiles + g - 1) / g;
            const double use = (double)(units / g * g) / units * n_tiles / (rounds * g);
            if (use >= 0.94 || use > best_use) best = Gangs{g, units / g, rounds, false, tn, n_tiles}, best_use = use;
        }
        return best;
    };
    // Two accumulators where the epilogue that nothing hides is a small part (long runs), the column tiles come out full,
    // and the second operand stays in L2 (half as many units share a block of the first one).
    Gangs best = plan(2 * BN);
    if ((double)dim / (2 * BN * best.n_tiles) < 0.95 || best.rounds * m_tiles * kb / best.gangs < WIDE_RUN || kb * BK * dim * 2 > WIDE_OPERAND) best = plan(BN);
    // whole tiles where the last round's idle units cost less than joining fragments would
    const long long lines = best.rounds * m_tiles;
    best.split = kb >= SPLIT_KB && (join_cost == 0 || (lines + best.gangs - 1) / best.gangs * kb > lines * kb / best.gangs + join_cost * BN / best.tn);
    const long long most = best.split ? (lines * kb + 3) / 4 : lines;
    if (best.gangs > most) best.gangs = most < 1 ? 1 : (int)most;
    return best;
}

// How the classes are cut into pieces.  All times in what a unit takes for a block of 256 x 256 x 64.
constexpr int64_t PIECE_ELEMENTS = 3ll << 26;   // of g, at most: 384 MiB
constexpr int JOIN_COST = 80;                   // of DW's fragments (DH's are joined in any case)
constexpr int PIECE_COST = 60;                  // of the launches of a piece and of DH's additions

struct Piece {
    int width;       // classes, rounded up to 256
    Gangs dh, dw;
    double cost;
};
Piece piece_plan(const qgbdt_ctx *c, int64_t classes, int n_pad, int dim) {
    Piece p;
    p.width = up(classes, 256);
    const int units = c->sm_count / CG, m_tiles = n_pad / BM, kb = (dim + BK - 1) / BK;
    p.dh = gang_plan(units, m_tiles, dim, p.width / BK, 0);
    p.dw = gang_plan(units, p.width / BM, dim, n_pad / BK, JOIN_COST);
    const long long lines = (long long)p.dw.rounds * (p.width / BM), tiles = (long long)m_tiles * (p.width / BN);
    const double dw = p.dw.split ? (double)lines / p.dw.gangs : (double)((lines + p.dw.gangs - 1) / p.dw.gangs);
    // GRAD's epilogue takes as long as six blocks
    p.cost = (double)((tiles + units - 1) / units) * (kb > 6 ? kb : 6) + (double)m_tiles * ((dim + BN - 1) / BN) * (p.width / BK) / units +
             dw * (n_pad / BK) * p.dw.tn / BN + (p.dw.split ? JOIN_COST : 0) + PIECE_COST;
    return p;
}

// DH and DW of a piece in one launch: the units are divided so that both end together.  It is taken where that ends
// before the two launches would, one of which costs about as long as LAUNCH_COST blocks take; long products, whose tiles have two
// accumulators or are cut (DW), have launches of their own.
// All gradients, two launches and one: 512 rows x 4000 classes x 256 31 and 24 us, 777 x 10007 x 129 42 and 36,
// 3000 x 5000 x 512 69 and 56, 60 x 8000 x 40 25 and 19.
constexpr int LAUNCH_COST = 13;
double longest_run(const Gangs &g, long long m_tiles, long long kb) {
    const long long lines = g.rounds * m_tiles;
    return g.split ? (double)lines * kb / g.gangs : (double)((lines + g.gangs - 1) / g.gangs * kb);
}
bool both_plan(const qgbdt_ctx *c, Piece &p, int n_pad, int dim) {
    const int units = c->sm_count / CG, m_tiles = n_pad / BM, v_tiles = p.width / BM, kb_h = p.width / BK, kb_w = n_pad / BK;
    if (p.dh.tn != BN || p.dw.tn != BN || p.dw.split) return false;
    double best = longest_run(p.dh, m_tiles, kb_h) + longest_run(p.dw, v_tiles, kb_w) + LAUNCH_COST;
    bool found = false;
    const Piece alone = p;
    // DW's whole tiles in one round of its units, in two, ...: the others are DH's, whose products are cut anywhere
    const int tiles = v_tiles * p.dw.n_tiles, first = tiles / units + 1;
    for (int r = first; r < first + 5; ++r) {
        const int u = units - (tiles + r - 1) / r;
        if (u < 1) continue;
        const Gangs h = gang_plan(u, m_tiles, dim, kb_h, 0), w = gang_plan(units - u, v_tiles, dim, kb_w, JOIN_COST);
        if (h.tn != BN || w.tn != BN || w.split) continue;
        const double a = longest_run(h, m_tiles, kb_h), b = longest_run(w, v_tiles, kb_w), cost = a > b ? a : b;
        if (cost < best) best = cost, p.dh = h, p.dw = w, found = true;
    }
    if (!found) p = alone;
    return found;
}

// Pieces of equal width and a narrower last one.  Of some widths that the memory allows (equal shares, and whole rounds of
// DW's gangs) the one with the least cost.
int64_t piece_width(const qgbdt_ctx *c, int64_t classes, int n_pad, int dim) {
    int64_t most = PIECE_ELEMENTS / n_pad / 256 * 256;
    if (most < 256) most = 256;
    if (classes <= most) return classes;
    const int64_t pieces = (classes + most - 1) / most, round = 256ll * piece_plan(c, most, n_pad, dim).dw.gangs;
    int64_t best = most;
    double best_cost = 1e300;
    auto look = [&](int64_t width) {
        if (width < 256 || width > most) return;
        const int64_t rest = classes % width;
        const double cost = (double)(classes / width) * piece_plan(c, width, n_pad, dim).cost + (rest ? piece_plan(c, rest, n_pad, dim).cost : 0.0);
        if (cost < best_cost) best = width, best_cost = cost;
    };
    for (int64_t k = pieces; k < pieces + 4; ++k) look((classes + k - 1) / k + 255 & ~255ll);
    for (int64_t k = most / round; k > 0 && k > most / round - 3; --k) look(k * round);
    return best;
}

template <typename T>
int dh_finish(qgbdt_ctx *c, const SoftmaxArgs &a, const PackArgs &p, const DhParts &full, const DhParts &rest, const BiasArgs &bias, cudaStream_t st) {
    int lg = 0, lg_parts = 0;
    while (lg < (a.rows < 4096 ? 8 : 6) && (4 << lg) < a.dim) ++lg;   // few rows: as many threads per row as there are columns
    const int fragments = full.gangs / (full.rounds * (up(a.rows, 256) / BM)) + 1;   // of a row, or a few more
    while (lg + lg_parts < 8 && (8 << lg_parts) < fragments) ++lg_parts;
    const int rows = 256 >> lg >> lg_parts;
    return qg_launch(c, k_dh_finish<T>, dim3((unsigned)((a.rows + rows - 1) / rows) + bias.blocks), 256, 0, st, full, rest, p.pos_of, (int)a.rows, a.dim,
                     a.grad_loss, p.count, reinterpret_cast<T *>(a.d_hidden), a.ld_d_hidden, lg, lg_parts, bias);
}

template <typename T>
int dw_finish(qgbdt_ctx *c, const SoftmaxArgs &a, const PackArgs &p, const float *part, int tn, const GemmArgs &g, int rows, cudaStream_t st) {
    return qg_launch(c, k_dw_finish<T>, dim3(g.gangs * g.gang, BM / 8), 256, 0, st, part, tn, g.gang, g.gangs, g.rounds, g.m_tiles, g.n_tiles, rows, a.dim, a.grad_loss, p.count,
                                                       reinterpret_cast<T *>(a.d_weight) + g.v0 * a.ld_d_weight, a.ld_d_weight);
}

}  // namespace

// The loss of up to FEW_ROWS rows with aligned operands.
static int loss_few(qgbdt_ctx *c, const SoftmaxArgs &a, cudaStream_t st) {
    const long long most = c->sm_count * FEW_BLOCKS, want = (a.classes + FEW_WARPS * FEW_CLASSES - 1) / (FEW_WARPS * FEW_CLASSES);
    const int blocks = (int)(want < most ? want : most);
    QgWorkspace ws;
    QG_RUN(qg_ws_open(c, qg_ws_size((size_t)FEW_ROWS * blocks, 8) + 256, st, &ws));
    FewArgs f{};
    f.hidden = reinterpret_cast<const uint16_t *>(a.hidden), f.weight = reinterpret_cast<const uint16_t *>(a.weight);
    f.ld_hidden = a.ld_hidden, f.ld_weight = a.ld_weight, f.rows = (int)a.rows, f.classes = (int)a.classes, f.dim = a.dim;
    f.bias = a.bias, f.labels = a.labels, f.label_type = a.label_type, f.status = a.status;
    f.stat = ws.take<float2>((size_t)FEW_ROWS * blocks), f.z_label = ws.take<float>(FEW_ROWS);
    f.arrived = c->d_ops_counters, f.loss = a.loss, f.losses = a.losses, f.lse = a.lse;
    const bool bf16 = a.type == QGBDT_BF16;
    const auto kernel = a.rows == 1 ? (bf16 ? k_loss_few<__nv_bfloat16, 1> : k_loss_few<__half, 1>)
                                    : (bf16 ? k_loss_few<__nv_bfloat16, 2> : k_loss_few<__half, 2>);
    QG_RUN(qg_launch(c, kernel, dim3(blocks), FEW_WARPS * 32, 0, st, f));
    return qg_ws_close(c, st);
}

// Up to here (rows * classes * dim) all rows go through the products, labelled or not: packing takes two launches and a copy
// of H, more than the products it could save.  20000 rows x 1000 classes x 256, all labelled: 36 us packed, 29 us not; none
// labelled, the worst case: 13 and 19 us.  The rule counts products; with dim below about 400 a tile takes as long as its
// epilogue, whatever dim is, so that many classes of small dim with few labelled rows would be better off packed.
constexpr double DIRECT_PRODUCTS = 1e10;

int qg_softmax_ce(qgbdt_ctx *c, const SoftmaxArgs &a, cudaStream_t st) {
    const bool aligned = rows_aligned(a.hidden, a.ld_hidden);
    if (a.rows > 0 && a.rows <= FEW_ROWS && weight_bytes(a) == 0 && aligned && a.dim % 8 == 0) return loss_few(c, a, st);
    const bool direct = aligned && (double)a.rows * (double)a.classes * a.dim <= DIRECT_PRODUCTS;
    const int n_tiles = up(a.classes, BN) / BN, n_pad = up(a.rows, 256);
    JoinArgs j{};
    while (j.lg < 5 && (1 << j.lg) < n_tiles) ++j.lg;   // a lane per two of a row's statistics, at most a warp
    const int join_blocks = a.rows > 0 ? (int)((a.rows + (JOIN_THREADS >> j.lg) - 1) / (JOIN_THREADS >> j.lg)) : 1;
    const int units = unit_count(c, (long long)(n_pad / BM) * n_tiles);
    if (units < 0) return qg_fail(c, QGBDT_ERR_ARG, "rows * classes is too large for one call");
    QgWorkspace ws;
    int rc = qg_ws_open(c, weight_bytes(a) + (direct ? 0 : pack_bytes(a)) + qg_ws_size((size_t)n_pad * n_tiles * 2, 8) + qg_ws_size((size_t)n_pad, 4) +
                               qg_ws_size(join_blocks, 8) + qg_ws_size(join_blocks, 4), st, &ws);
    if (rc != QGBDT_OK) return rc;
    RealignArgs copy;
    const Weight w = align_weight(c, a, ws, &copy);
    GemmArgs g = gemm_args(c, a);
    PackArgs p{};
    if (direct) {
        g.all_rows = (int)a.rows, g.labels = RawLabels{a.labels, a.label_type, (int)a.classes};
        if (copy.blocks) QG_RUN(qg_launch(c, k_realign, dim3(copy.blocks), PACK_THREADS, 0, st, copy));
    } else {
        if ((rc = pack_rows(c, a, ws, copy, &p, st)) != QGBDT_OK) return rc;
        g.count = p.count, g.label = p.label;
    }
    g.n_tiles = n_tiles;
    g.stat = ws.take<float2>((size_t)n_pad * n_tiles * 2);
    g.z_label = ws.take<float>(n_pad);
    if (a.rows > 0) {
        CUtensorMap ma, mb;
        if ((rc = direct ? matrix_map(c, &ma, a.hidden, a.dim, a.rows, a.ld_hidden, 128, a.type)
                         : matrix_map(c, &ma, p.packed, a.dim, n_pad, p.ldp, 128, a.type)) != QGBDT_OK)
            return rc;
        if ((rc = matrix_map(c, &mb, w.p, a.dim, a.classes, w.ld, B_ROWS, a.type)) != QGBDT_OK) return rc;
        if ((rc = gemm<LOSS, 1>(c, g, units, ma, mb, ma, ma, st)) != QGBDT_OK) return rc;
    }
    j.stat = g.stat, j.n_tiles = n_tiles * 2, j.z_label = g.z_label, j.pos_of = p.pos_of, j.labels = g.labels, j.n = (int)a.rows;
    j.losses = a.losses, j.lse = a.lse, j.loss = a.loss, j.status = a.status, j.arrived = c->d_ops_counters;
    j.block_loss = ws.take<double>(join_blocks), j.block_count = ws.take<int>(join_blocks);
    QG_RUN(qg_launch(c, k_loss_join, dim3(join_blocks), JOIN_THREADS, 0, st, j));
    return qg_ws_close(c, st);
}

int qg_softmax_ce_backward(qgbdt_ctx *c, const SoftmaxArgs &a, cudaStream_t st) {
    if (a.rows == 0) {
        if (a.ld_d_weight < 1ll << 30) {
            QG_CUDA(c, cudaMemset2DAsync(a.d_weight, a.ld_d_weight * 2, 0, (size_t)a.dim * 2, a.classes, st));
        } else {   // rows too far apart for one call, and so only a few
            for (int64_t v = 0; v < a.classes; ++v)
                QG_CUDA(c, cudaMemsetAsync(reinterpret_cast<uint16_t *>(a.d_weight) + v * a.ld_d_weight, 0, (size_t)a.dim * 2, st));
        }
        if (a.d_bias) QG_CUDA(c, cudaMemsetAsync(a.d_bias, 0, sizeof(float) * a.classes, st));
        return QGBDT_OK;
    }
    const int n_pad = up(a.rows, 256), m_tiles = n_pad / BM;
    // the pieces: n_full of one width, then (kind 1) what is left
    const int64_t width = piece_width(c, a.classes, n_pad, a.dim), n_full = a.classes / width, left = a.classes - n_full * width;
    Piece kinds[2] = {piece_plan(c, width, n_pad, a.dim), left ? piece_plan(c, left, n_pad, a.dim) : Piece{}};
    const bool both[2] = {both_plan(c, kinds[0], n_pad, a.dim), left && both_plan(c, kinds[1], n_pad, a.dim)};
    const int n_kinds = left ? 2 : 1, ld_g = kinds[0].width;
    if (unit_count(c, (long long)m_tiles * (ld_g / BN)) < 0 || unit_count(c, (long long)m_tiles * ((a.dim + BN - 1) / BN)) < 0)
        return qg_fail(c, QGBDT_ERR_ARG, "rows * classes is too large for one call");
    size_t dh_rows[2] = {0, 0}, dw_floats = 0, bytes = weight_bytes(a) + pack_bytes(a) + qg_ws_size((size_t)n_pad * ld_g, 2) +
                                                       (a.d_bias ? qg_ws_size((size_t)(n_pad / 32) * ld_g, 4) : 0);
    size_t dw_rows[2] = {0, 0};
    for (int i = 0; i < n_kinds; ++i) {
        const Gangs &h = kinds[i].dh, &w = kinds[i].dw;
        dh_rows[i] = ((size_t)m_tiles * h.rounds + h.gangs) * h.size * BM;
        dw_rows[i] = w.split ? 2 * (size_t)w.units() * BM : 0;
        if (dw_rows[i] * w.tn > dw_floats) dw_floats = dw_rows[i] * w.tn;
        bytes += qg_ws_size(dh_rows[i] * h.tn, 4);
    }
    QgWorkspace ws;
    int rc = qg_ws_open(c, bytes + qg_ws_size(dw_floats, 4), st, &ws);
    if (rc != QGBDT_OK) return rc;
    RealignArgs copy;
    PackArgs p;
    const Weight w = align_weight(c, a, ws, &copy);
    if ((rc = pack_rows(c, a, ws, copy, &p, st)) != QGBDT_OK) return rc;
    uint16_t *g_piece = ws.take<uint16_t>((size_t)n_pad * ld_g);
    float *bias_part = a.d_bias ? ws.take<float>((size_t)(n_pad / 32) * ld_g) : nullptr, *dw_part = ws.take<float>(dw_floats);
    GemmArgs base = gemm_args(c, a);
    base.count = p.count, base.label = p.label, base.lse = p.lse_packed;
    const bool bf16 = base.bf16, out_map = rows_aligned(a.d_weight, a.ld_d_weight) && a.dim % 8 == 0;   // tiled copies cut rows off at 16 bytes only
    CUtensorMap h_k, h_mn, w_k, w_mn, g_k, g_mn, g_store, dh_map[2], dw_map[2], out;
    if ((rc = matrix_map(c, &h_k, p.packed, a.dim, n_pad, p.ldp, 128, a.type)) != QGBDT_OK) return rc;
    if ((rc = matrix_map(c, &h_mn, p.packed, a.dim, n_pad, p.ldp, 64, a.type)) != QGBDT_OK) return rc;
    if ((rc = matrix_map(c, &w_k, w.p, a.dim, a.classes, w.ld, B_ROWS, a.type)) != QGBDT_OK) return rc;
    if ((rc = matrix_map(c, &w_mn, w.p, a.dim, a.classes, w.ld, 64, a.type)) != QGBDT_OK) return rc;
    if ((rc = matrix_map(c, &g_k, g_piece, ld_g, n_pad, ld_g, 128, a.type)) != QGBDT_OK) return rc;
    if ((rc = matrix_map(c, &g_mn, g_piece, ld_g, n_pad, ld_g, 64, a.type)) != QGBDT_OK) return rc;
    if ((rc = matrix_map(c, &g_store, g_piece, ld_g, n_pad, ld_g, 32, a.type)) != QGBDT_OK) return rc;
    DhParts parts[2] = {};
    for (int i = 0; i < n_kinds; ++i) {
        const Gangs &h = kinds[i].dh, &d = kinds[i].dw;
        parts[i] = DhParts{ws.take<float>(dh_rows[i] * h.tn), h.tn, h.size, h.gangs, h.rounds, kinds[i].width / BK, h.split};
        if ((rc = matrix_map(c, &dh_map[i], parts[i].part, h.tn, (long long)dh_rows[i], h.tn, 32, QGBDT_F32)) != QGBDT_OK) return rc;
        dw_map[i] = dh_map[i];
        if (d.split && (rc = matrix_map(c, &dw_map[i], dw_part, d.tn, (long long)dw_rows[i], d.tn, 32, QGBDT_F32)) != QGBDT_OK) return rc;
    }
    out = g_store;
    if (out_map && (rc = matrix_map(c, &out, a.d_weight, a.dim, a.classes, a.ld_d_weight, 32, a.type)) != QGBDT_OK) return rc;
    BiasArgs bias{};   // of the last piece, finished with dH
    for (int64_t k = 0; k < n_full + (left ? 1 : 0); ++k) {
        const int kind = k < n_full ? 0 : 1, v0 = (int)(k * width), nv = (int)(kind == 0 ? width : left);
        const Gangs &h = kinds[kind].dh, &d = kinds[kind].dw;
        GemmArgs g = base;
        g.v0 = v0, g.n_tiles = kinds[kind].width / BN, g.bias_part = bias_part;
        if ((rc = gemm<GRAD, 1>(c, g, unit_count(c, (long long)m_tiles * g.n_tiles), h_k, w_k, g_store, g_store, st)) != QGBDT_OK) return rc;
        if (bias_part) {
            bias = BiasArgs{bias_part, kinds[kind].width, nv, a.d_bias + v0, (nv + 31) / 32};
            if (v0 + nv < a.classes) QG_RUN(qg_launch(c, k_bias_finish, dim3(bias.blocks), 256, 0, st, bias, a.grad_loss, base.count));
        }
        GemmArgs gh = base, gw = base;
        gh.v0 = v0, gh.n_tiles = h.n_tiles, gh.kb = kinds[kind].width / BK, gh.add = kind == 0 && k > 0;
        gh.gang = h.size, gh.gangs = h.gangs, gh.rounds = h.rounds, gh.split = h.split;
        gw.v0 = v0, gw.m_tiles = (nv + BM - 1) / BM, gw.n_tiles = d.n_tiles;
        gw.gang = d.size, gw.gangs = d.gangs, gw.rounds = d.rounds, gw.split = d.split;
        gw.rows = nv, gw.out = reinterpret_cast<uint16_t *>(a.d_weight), gw.ld_out = a.ld_d_weight, gw.out_map = out_map;
        if (both[kind]) {
            constexpr int smem = Layout<DH, 1>::BYTES > Layout<DW, 1>::BYTES ? Layout<DH, 1>::BYTES : Layout<DW, 1>::BYTES;
            rc = pairs(c, 8, smem, k_softmax_both, h.units() + d.units(), st, gh, gw, h.units() * CG, g_k, w_mn, dh_map[kind], g_mn, h_mn, out);
            if (rc != QGBDT_OK) return rc;
            continue;
        }
        if ((rc = (h.tn == BN ? gemm<DH, 1> : gemm<DH, 2>)(c, gh, h.units(), g_k, w_mn, g_store, dh_map[kind], st)) != QGBDT_OK) return rc;
        if ((rc = (d.tn == BN ? gemm<DW, 1> : gemm<DW, 2>)(c, gw, d.units(), g_mn, h_mn, out, dw_map[kind], st)) != QGBDT_OK) return rc;
        if (!d.split) continue;
        rc = bf16 ? dw_finish<__nv_bfloat16>(c, a, p, dw_part, d.tn, gw, nv, st) : dw_finish<__half>(c, a, p, dw_part, d.tn, gw, nv, st);
        if (rc != QGBDT_OK) return rc;
    }
    rc = bf16 ? dh_finish<__nv_bfloat16>(c, a, p, parts[0], parts[1], bias, st) : dh_finish<__half>(c, a, p, parts[0], parts[1], bias, st);
    if (rc != QGBDT_OK) return rc;
    return qg_ws_close(c, st);
}
