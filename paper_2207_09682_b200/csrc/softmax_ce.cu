// Softmax cross entropy of a linear classifier over many classes, without stored logits, and its gradients.
//
//   z = H W^T + b,   lse_i = log sum_v exp z_iv,   loss = mean of lse_i - z_i,label
//   g_iv = exp(z_iv - lse_i) - [v == label i],   dH = s g W,   dW = s g^T H,   db = s sum_i g_i
//
// with s = grad_loss / (rows with a label).  Four matrix products on the tensor cores: z once for the loss,
// z again for the gradients (cheaper than 2 bytes per logit out of and into DRAM at these widths, and no
// memory that grows with rows * classes), and the two products with g.  8 * rows * classes * dim operations
// in all; a step that kept the logits would need 6.
//
// One kernel carries all four: a persistent grid whose CTAs (or pairs of CTAs) take tiles of 128 (256) rows by
// 256 columns in turn.  One warp fills a ring of operand tiles with tiled copies, one thread issues the
// matrix instructions, four warps empty the accumulators, of which tensor memory holds two, so that the
// epilogue of a tile runs under the products of the next.  What the epilogues do:
//   LOSS  per row of the tile: maximum and sum of exponentials; the label's logit.  No logit leaves the SM.
//   GRAD  g of a piece of the classes, rounded to the inputs' type (relative error 2^-8 in bf16, 2^-11 in f16,
//         of each g on its own: as much as the outputs' own rounding, averaged down by the sums that follow;
//         the scale s is applied behind those sums, so that small g do not vanish in half precision), and its
//         column sums in single precision for the bias.
//   DH    the piece's contribution to dH, in single precision.
//   DW    rows of dW, complete with every piece, written in the output type.
//
// Rows without a label are taken out first: the labelled rows are packed to the front of a copy of H (which
// also gives the copies their alignment).  Nothing is computed for the others, and what they hold, infinities
// included, never meets a product.
#include <math.h>

#include "ops_internal.cuh"
#include "tensor_core.cuh"

namespace {

constexpr int CG = 2;                       // CTAs per tile
constexpr int BM = 128 * CG, BN = 256, BK = 64;
constexpr int A_BYTES = 128 * BK * 2, B_ROWS = BN / CG, B_BYTES = B_ROWS * BK * 2;
constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int STAGES = 196608 / STAGE_BYTES;
constexpr int EPI_WARPS = 4, THREADS = 128 + EPI_WARPS * 32;
constexpr int STORE_BYTES = 32 * 128;       // 32 rows of 64 columns of g, per warp; two of them
constexpr int SMEM_BYTES = 1024 + STAGES * STAGE_BYTES + EPI_WARPS * 2 * STORE_BYTES;
constexpr int TMEM_COLS = 512, ACC_COLS = 256;
constexpr int GROUP_M = 16;                 // row tiles that go through all column tiles together
constexpr float LOG2E = 1.44269504088896340736f;

enum Mode { LOSS, GRAD, DH, DW };

struct GemmArgs {
    const int *count;           // labelled rows
    int m_tiles, n_tiles;       // tiles (LOSS, GRAD, DH: row tiles for all rows; only those with labelled rows are taken)
    int kb;                     // blocks of 64 along the products' length (DW: taken from the count)
    int splits;                 // parts the length is cut into (DH, DW)
    int classes;                // all classes
    int v0;                     // first class of the piece
    int dim;
    int bf16;
    int *fault;
    // LOSS and GRAD
    const float *bias;
    const int *label;           // [labelled rows]
    float2 *stat;               // [row][n_tiles] maximum, sum of exp(z - maximum)
    float *z_label;             // [row]
    const float *lse;           // [row]
    float *bias_part;           // [m_tiles * 4 * CG][n_tiles * 256] column sums of g over 32 rows
    // DH and DW
    float *part;                // [splits][part_rows][ldp]
    long long part_rows;
    int ldp;
    int add;                    // DH: add to what is there
    void *out;                  // DW without splits: the output
    long long ld_out;
    int out_vec;                // its rows are 16-byte aligned
    const float *grad_loss;
};

struct Tile {
    int m, n, kb0, kb1, split;
};

template <int MODE>
__device__ __forceinline__ Tile tile_at(const GemmArgs &a, int m_live, int kb, int t) {
    Tile r;
    const int per = m_live * a.n_tiles;
    r.split = t / per;
    t -= r.split * per;
    const int group = t / (GROUP_M * a.n_tiles), m0 = group * GROUP_M, gm = min(GROUP_M, m_live - m0);
    t -= group * GROUP_M * a.n_tiles;
    r.n = t / gm;
    r.m = m0 + t - r.n * gm;
    r.kb0 = (int)((long long)kb * r.split / a.splits);
    r.kb1 = (int)((long long)kb * (r.split + 1) / a.splits);
    return r;
}

__device__ __forceinline__ float out_scale(const float *grad_loss, int count) {
    return (grad_loss ? *grad_loss : 1.0f) / (float)(count > 0 ? count : 1);
}

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

template <int MODE>
__global__ void __launch_bounds__(THREADS, 1) k_softmax_gemm(const GemmArgs a, const __grid_constant__ CUtensorMap map_a,
                                                             const __grid_constant__ CUtensorMap map_b,
                                                             const __grid_constant__ CUtensorMap map_g) {
    constexpr bool A_MN = MODE == DW, B_MN = MODE == DH || MODE == DW;   // operand rows run along the products' length
    extern __shared__ char smem_raw[];
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

    const int count = *a.count;
    const int m_live = MODE == DW ? a.m_tiles : (count + BM - 1) / BM;
    const int kb = MODE == DW ? (count + BK - 1) / BK : a.kb;
    const int total = m_live * a.n_tiles * a.splits;
    const int first = blockIdx.x / CG, step = gridDim.x / CG;
    bool ok = true;

    if (warp == 0 && lane == 0) {
        // ---- copies
        int it = 0;
        for (int t = first; t < total && ok; t += step) {
            const Tile c = tile_at<MODE>(a, m_live, kb, t);
            for (int k = c.kb0; k < c.kb1; ++k, ++it) {
                const int s = it % STAGES;
                if (!(ok = tc_bar_wait(empty(s), (it / STAGES & 1) ^ 1, &stop))) break;
                const uint32_t bar = CG == 1 ? full(s) : tc_map_rank(full(s), 0);
                if (rank == 0) tc_bar_expect(full(s), CG * STAGE_BYTES);
                const uint32_t at = tiles_at + s * STAGE_BYTES, bt = at + A_BYTES;
                const int am = c.m * BM + rank * 128, bn = c.n * BN + rank * B_ROWS;
                if (A_MN) {
                    for (int j = 0; j < 2; ++j) tc_load_2d<CG>(at + j * 8192, &map_a, am + 64 * j, k * BK, bar);
                } else {
                    tc_load_2d<CG>(at, &map_a, k * BK, am, bar);
                }
                if (B_MN) {
                    const int y = (MODE == DH ? a.v0 : 0) + k * BK;
                    for (int j = 0; j < B_ROWS / 64; ++j) tc_load_2d<CG>(bt + j * 8192, &map_b, bn + 64 * j, y, bar);
                } else {
                    tc_load_2d<CG>(bt, &map_b, k * BK, a.v0 + bn, bar);
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
        const uint32_t idesc = tc_idesc(BM, BN, a.bf16, A_MN, B_MN);
        int it = 0, n_acc = 0;
        for (int t = first; t < total && ok; t += step) {
            const Tile c = tile_at<MODE>(a, m_live, kb, t);
            if (c.kb0 == c.kb1) continue;
            const int b = n_acc & 1;
            if (!(ok = tc_bar_wait(acc_empty(b), (n_acc / 2 & 1) ^ 1, &stop))) break;
            tc_fence_after();
            for (int k = c.kb0; k < c.kb1; ++k, ++it) {
                const int s = it % STAGES;
                if (!(ok = tc_bar_wait(full(s), it / STAGES & 1, &stop))) break;
                tc_fence_after();
                const uint32_t at = tiles_at + s * STAGE_BYTES, bt = at + A_BYTES;
#pragma unroll
                for (int q = 0; q < BK / 16; ++q) {
                    const uint64_t da = tc_desc(at + q * (A_MN ? 2048 : 32), A_MN ? 8192 : 16);
                    const uint64_t db = tc_desc(bt + q * (B_MN ? 2048 : 32), B_MN ? 8192 : 16);
                    tc_mma<CG>(tmem + b * ACC_COLS, da, db, idesc, k > c.kb0 || q > 0);
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
    } else if (warp >= 4) {
        // ---- epilogue: thread = row of the tile
        const int q = warp & 3;
        const uint32_t tacc = tmem + ((uint32_t)(q * 32) << 16);
        const uint32_t store = store_at + (warp - 4) * 2 * STORE_BYTES;
        int n_acc = 0, n_store = 0;
        for (int t = first; t < total; t += step) {
            const Tile c = tile_at<MODE>(a, m_live, kb, t);
            const bool some = c.kb0 < c.kb1;   // a part of no length: zeros
            const int b = n_acc & 1;
            if (some) {
                if (!(ok = __all_sync(0xffffffffu, tc_bar_wait(acc_full(b), n_acc / 2 & 1, &stop)))) break;
                tc_fence_after();
            }
            const int row_in = c.m * BM + (int)rank * 128 + q * 32;   // the warp's first row
            const int row = row_in + lane;
            const bool live = MODE == DW || row < count;
            float m_run = -INFINITY, l_run = 0.0f, lse = 0.0f, scale = 1.0f;
            int label = -1;
            if (MODE == LOSS || MODE == GRAD) label = live ? a.label[row] : -1;
            if (MODE == GRAD) lse = live ? a.lse[row] : 0.0f;
            if (MODE == DW && a.out) scale = out_scale(a.grad_loss, count);
#pragma unroll 1
            for (int cc = 0; cc < BN / 32; ++cc) {
                const int col = c.n * BN + cc * 32;                  // in the piece (LOSS, GRAD) or in dim (DH, DW)
                uint32_t r[32];
                float x[32];
                if (some) {
                    tc_ld_32(tacc + b * ACC_COLS + cc * 32, r);
                    if (cc == BN / 32 - 1) {   // the accumulator may be filled again
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) tc_bar_arrive_cluster(CG == 1 ? acc_empty(b) : tc_map_rank(acc_empty(b), 0));
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j] = __uint_as_float(r[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j] = 0.0f;
                }
                if (MODE == LOSS || MODE == GRAD) {
                    const int v = a.v0 + col;
                    if (a.bias) {
                        const float bias = v + lane < a.classes ? a.bias[v + lane] : 0.0f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) x[j] += __shfl_sync(0xffffffffu, bias, j);
                    }
                    if (v + 32 > a.classes) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (v + j >= a.classes) x[j] = -INFINITY;
                    }
                    const int lj = label - v;
                    if (MODE == LOSS) {
                        float top = x[0];
#pragma unroll
                        for (int j = 1; j < 32; ++j) top = fmaxf(top, x[j]);
                        top = fmaxf(top, m_run);
                        const float base = top == -INFINITY ? 0.0f : top;
                        float s0 = l_run * tc_ex2((m_run - base) * LOG2E), s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            s0 += tc_ex2((x[j] - base) * LOG2E);
                            s1 += tc_ex2((x[j + 1] - base) * LOG2E);
                            s2 += tc_ex2((x[j + 2] - base) * LOG2E);
                            s3 += tc_ex2((x[j + 3] - base) * LOG2E);
                        }
                        l_run = (s0 + s1) + (s2 + s3);
                        m_run = top;
                        if (lj >= 0 && lj < 32) {
                            float z = x[0];
#pragma unroll
                            for (int j = 1; j < 32; ++j)
                                if (lj == j) z = x[j];
                            a.z_label[row] = z;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) x[j] = tc_ex2((x[j] - lse) * LOG2E);
                        if (lj >= 0 && lj < 32) {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (lj == j) x[j] -= 1.0f;
                        }
                        if (!live) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[j] = 0.0f;
                        }
                        // 32 rows by 64 columns at a time to the buffer of g
                        const uint32_t buf = store + (n_store & 1) * STORE_BYTES;
                        if ((cc & 1) == 0) {   // the copy that used this buffer has read it
                            if (lane == 0) tc_store_wait_read<1>();
                            __syncwarp();
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t w = buf + lane * 128 + (((uint32_t)((cc & 1) * 4 + i) ^ (lane & 7)) << 4);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(w), "r"(pack2(x[8 * i], x[8 * i + 1], a.bf16)),
                                         "r"(pack2(x[8 * i + 2], x[8 * i + 3], a.bf16)), "r"(pack2(x[8 * i + 4], x[8 * i + 5], a.bf16)),
                                         "r"(pack2(x[8 * i + 6], x[8 * i + 7], a.bf16))
                                         : "memory");
                        }
                        if (cc & 1) {
                            tc_fence_async_smem();
                            __syncwarp();
                            if (lane == 0) {
                                tc_store_2d(&map_g, col - 32, row_in, buf);
                                tc_store_commit();
                            }
                            ++n_store;
                        }
                        if (a.bias_part) {
                            const float s = column_sums(x, lane);
                            a.bias_part[(long long)(row_in / 32) * (a.n_tiles * BN) + col + lane] = s;
                        }
                    }
                } else if (MODE == DW && a.out) {
                    const int v = a.v0 + row;
                    if (v < a.classes) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t w[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) w[j] = pack2(x[8 * i + 2 * j] * scale, x[8 * i + 2 * j + 1] * scale, a.bf16);
                            const int d = col + 8 * i;
                            uint16_t *o = reinterpret_cast<uint16_t *>(a.out) + v * a.ld_out + d;
                            if (a.out_vec && d + 8 <= a.dim) {
                                *reinterpret_cast<uint4 *>(o) = make_uint4(w[0], w[1], w[2], w[3]);
                            } else {
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    if (d + j < a.dim) o[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
                            }
                        }
                    }
                } else if (live) {
                    float4 *o = reinterpret_cast<float4 *>(a.part + ((long long)c.split * a.part_rows + row) * a.ldp + col);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (col + 4 * i < a.ldp) {
                            float4 w = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                            if (MODE == DH && a.add) {
                                const float4 y = o[i];
                                w.x += y.x, w.y += y.y, w.z += y.z, w.w += y.w;
                            }
                            o[i] = w;
                        }
                }
            }
            if (MODE == LOSS && live) a.stat[(long long)row * a.n_tiles + c.n] = make_float2(m_run, l_run);
            if (some) ++n_acc;
        }
        if (!ok) {
            stop = 1;
            *a.fault = 1;
        }
        if (MODE == GRAD && lane == 0) tc_store_wait();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_group_sync<CG>();
    tc_fence_after();
    if (warp == 2) tc_dealloc<CG>(tmem, TMEM_COLS);
}

// ---- rows with a label, packed -----------------------------------------------------------------------

constexpr int PACK_THREADS = 256, PACK_ROWS = 64, PACK_SPAN = 8192;   // labels per block, per entry of the counts

struct PackArgs {
    const void *labels;
    int label_type;
    int n, n_pad;              // rows; rows of the packed copy (a multiple of the tile)
    int classes;
    const uint16_t *hidden;    // 16-bit elements, moved as they are
    long long ld;
    int dim, vec;              // vec: rows can be read 16 bytes at a time
    const float *lse;          // or NULL
    int *span_count;           // [spans], with more than one span
    // results
    int *count, *row_of, *pos_of, *label;
    float *lse_packed;
    uint16_t *packed;          // [n_pad][ldp]
    int ldp;
    int *status;
};

__device__ __forceinline__ int label_of(const PackArgs &a, int i) {   // -1: none
    const long long l = a.label_type == QGBDT_I64 ? reinterpret_cast<const long long *>(a.labels)[i] : (long long)reinterpret_cast<const int *>(a.labels)[i];
    if (l >= a.classes && a.status) *a.status = 1;
    return l >= 0 && l < a.classes ? (int)l : -1;
}

__device__ __forceinline__ int block_sum_int(int s) {
    __shared__ int w[PACK_THREADS / 32];
    s = __reduce_add_sync(0xffffffffu, s);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) w[threadIdx.x / 32] = s;
    __syncthreads();
    s = 0;
    for (int i = 0; i < PACK_THREADS / 32; ++i) s += w[i];
    return s;
}

__global__ void __launch_bounds__(PACK_THREADS) k_pack_count(const PackArgs a) {
    const int i0 = blockIdx.x * PACK_SPAN, i1 = min(a.n, i0 + PACK_SPAN);
    int s = 0;
    for (int i = i0 + threadIdx.x; i < i1; i += PACK_THREADS) s += label_of(a, i) >= 0;
    s = block_sum_int(s);
    if (threadIdx.x == 0) a.span_count[blockIdx.x] = s;
}

__global__ void __launch_bounds__(PACK_THREADS) k_pack(const PackArgs a) {
    __shared__ int place[PACK_ROWS];   // where the block's rows go, -1: no label
    const int r0 = blockIdx.x * PACK_ROWS, spans = (a.n + PACK_SPAN - 1) / PACK_SPAN, span = r0 / PACK_SPAN;
    int before = 0, all = 0;
    if (spans > 1)
        for (int s = threadIdx.x; s < spans; s += PACK_THREADS) {
            const int x = a.span_count[s];
            all += x;
            if (s < span) before += x;
        }
    {   // labels of this span in front of this block (and, with a single span, all of them)
        const int i0 = span * PACK_SPAN, i1 = spans > 1 ? min(a.n, r0) : a.n;
        for (int i = i0 + threadIdx.x; i < i1; i += PACK_THREADS) {
            const int has = label_of(a, i) >= 0;
            if (i < r0) before += has;
            if (spans <= 1) all += has;
        }
    }
    before = block_sum_int(before);
    all = block_sum_int(all);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = all;
    if (threadIdx.x < 32) {
        int run = before;
        for (int h = 0; h < PACK_ROWS; h += 32) {
            const int i = r0 + h + threadIdx.x, l = i < a.n ? label_of(a, i) : -1;
            const unsigned has = __ballot_sync(0xffffffffu, l >= 0);
            const int p = l >= 0 ? run + __popc(has & ((1u << threadIdx.x) - 1)) : -1;
            place[h + threadIdx.x] = p;
            if (i < a.n) a.pos_of[i] = p;
            if (p >= 0) {
                a.row_of[p] = i;
                a.label[p] = l;
                if (a.lse) a.lse_packed[p] = a.lse[i];
            }
            run += __popc(has);
        }
    }
    __syncthreads();
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, chunks = a.ldp / 8;   // ldp is a multiple of 8
    for (int h = warp; h < PACK_ROWS; h += PACK_THREADS / 32) {
        if (place[h] >= 0) {
            const uint16_t *in = a.hidden + (r0 + h) * a.ld;
            uint4 *out = reinterpret_cast<uint4 *>(a.packed + (long long)place[h] * a.ldp);
            if (a.vec) {
                for (int k = lane; k < chunks; k += 32) out[k] = reinterpret_cast<const uint4 *>(in)[k];
            } else {
                for (int k = lane; k < chunks; k += 32) {
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int d = 8 * k + 2 * j;
                        w[j] = (d < a.dim ? in[d] : 0u) | (uint32_t)(d + 1 < a.dim ? in[d + 1] : 0u) << 16;
                    }
                    out[k] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
        if (r0 + h >= all && r0 + h < a.n_pad) {   // rows behind the last labelled one: zeros
            uint4 *out = reinterpret_cast<uint4 *>(a.packed + (long long)(r0 + h) * a.ldp);
            for (int k = lane; k < chunks; k += 32) out[k] = make_uint4(0, 0, 0, 0);
        }
    }
}

// Copy of a matrix whose rows do not start on 16-byte boundaries, with rows that do.
__global__ void __launch_bounds__(256) k_realign(const uint16_t *in, long long ld, long long rows, int dim, uint16_t *out, int ldp) {
    const int chunks = ldp / 8;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < rows * chunks; i += (long long)gridDim.x * 256) {
        const long long r = i / chunks;
        const int d = (int)(i - r * chunks) * 8;
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = (d + 2 * j < dim ? in[r * ld + d + 2 * j] : 0u) | (uint32_t)(d + 2 * j + 1 < dim ? in[r * ld + d + 2 * j + 1] : 0u) << 16;
        *reinterpret_cast<uint4 *>(out + r * ldp + d) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// ---- loss from the tiles' statistics -------------------------------------------------------------------

constexpr int JOIN_ROWS = 8;   // one warp per row

__global__ void __launch_bounds__(JOIN_ROWS * 32) k_loss_join(const float2 *stat, int n_tiles, const float *z_label, const int *pos_of, int n,
                                                              const int *count, float *losses, float *lse, double *block_loss,
                                                              unsigned *arrived, float *loss) {
    __shared__ double w[JOIN_ROWS];
    __shared__ bool last;
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, row = blockIdx.x * JOIN_ROWS + warp;
    float mine = 0.0f;
    if (row < n) {
        const int p = pos_of[row];
        float l_out = 0.0f;
        if (p >= 0) {
            float m = -INFINITY, l = 0.0f;
            for (int t = lane; t < n_tiles; t += 32) {
                const float2 s = stat[(long long)p * n_tiles + t];
                const float top = fmaxf(m, s.x), base = top == -INFINITY ? 0.0f : top;
                l = l * tc_ex2((m - base) * LOG2E) + s.y * tc_ex2((s.x - base) * LOG2E);
                m = top;
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
                const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
                l = l * tc_ex2((m - base) * LOG2E) + l2 * tc_ex2((m2 - base) * LOG2E);
                m = top;
            }
            l_out = m + logf(l);
            mine = l_out - z_label[p];
        }
        if (lane == 0) {
            lse[row] = l_out;
            if (losses) losses[row] = mine;
        }
    }
    if (lane == 0) w[warp] = (double)mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int i = 0; i < JOIN_ROWS; ++i) s += w[i];
        block_loss[blockIdx.x] = s;
        __threadfence();
        last = atomicAdd(arrived, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    // the block that comes last adds the blocks' sums, in their order
    __threadfence();
    double s = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += JOIN_ROWS * 32) s += *(volatile double *)&block_loss[i];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) w[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int i = 0; i < JOIN_ROWS; ++i) s += w[i];
        const int c = *count;
        *loss = (float)(s / (double)(c > 0 ? c : 1));
        *arrived = 0;
    }
}

// ---- gradients out of single-precision parts -------------------------------------------------------------

// out[r] = scale * sum over the splits of part[split][pos_of[r]] (pos_of NULL: r itself; negative: zeros).
template <typename T>
__global__ void __launch_bounds__(256) k_grad_finish(const float *part, int splits, long long part_rows, int ldp, const int *pos_of, long long rows,
                                                     int dim, const float *grad_loss, const int *count, T *out, long long ld_out) {
    const float scale = out_scale(grad_loss, *count);
    const int quads = (dim + 3) / 4;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < rows * quads; i += (long long)gridDim.x * 256) {
        const long long r = i / quads;
        const int d = (int)(i - r * quads) * 4;
        const long long p = pos_of ? pos_of[r] : r;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (p >= 0)
            for (int k = 0; k < splits; ++k) {
                const float4 x = *reinterpret_cast<const float4 *>(part + (k * part_rows + p) * ldp + d);
                s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
            }
        OpsVec<T, 4> y;
        y.v[0] = OpsType<T>::store(s.x * scale), y.v[1] = OpsType<T>::store(s.y * scale);
        y.v[2] = OpsType<T>::store(s.z * scale), y.v[3] = OpsType<T>::store(s.w * scale);
        T *o = out + r * ld_out + d;
        if (d + 4 <= dim && reinterpret_cast<uintptr_t>(o) % sizeof(y) == 0) {
            *reinterpret_cast<OpsVec<T, 4> *>(o) = y;
        } else {
            for (int j = 0; j < 4 && d + j < dim; ++j) o[j] = y.v[j];
        }
    }
}

// Bias gradient of a piece: sums over groups of 32 rows, in their order.
__global__ void __launch_bounds__(256) k_bias_finish(const float *part, int cols, int n, const float *grad_loss, const int *count, float *out) {
    __shared__ float w[8][32];
    const int v = blockIdx.x * 32 + (threadIdx.x & 31), k = threadIdx.x / 32;
    const int groups = (*count + BM - 1) / BM * (BM / 32);
    float s = 0.0f;
    for (int g = k; g < groups; g += 8) s += part[(long long)g * cols + v];   // cols is a multiple of 256
    w[k][threadIdx.x & 31] = s;
    __syncthreads();
    if (k == 0 && v < n) {
        for (int j = 1; j < 8; ++j) s += w[j][threadIdx.x];
        out[v] = s * out_scale(grad_loss, *count);
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

// Matrix [rows][ld] of 16-bit elements, copied in boxes of 64 columns by `box` rows, 128-byte swizzle, zeros outside.
int matrix_map(qgbdt_ctx *c, CUtensorMap *m, const void *p, long long cols, long long rows, long long ld, int box, bool bf16) {
    EncodeTiled encode = nullptr;
    int rc = encoder(c, &encode);
    if (rc != QGBDT_OK) return rc;
    const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t b[2] = {64, (cuuint32_t)box}, one[2] = {1, 1};
    const CUresult r = encode(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(p), size, stride, b, one,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return qg_fail(c, QGBDT_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
    return QGBDT_OK;
}

template <int MODE>
int gemm(qgbdt_ctx *c, const GemmArgs &a, const CUtensorMap &ma, const CUtensorMap &mb, const CUtensorMap &mg, cudaStream_t st) {
    QG_CUDA(c, cudaFuncSetAttribute(k_softmax_gemm<MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES));
    const long long tiles = (long long)a.m_tiles * a.n_tiles * a.splits;
    if (tiles > 0x7fffffffll) return qg_fail(c, QGBDT_ERR_ARG, "rows * classes is too large for one call");
    const int units = c->sm_count / CG;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles < units ? (tiles > 0 ? tiles : 1) : units) * CG);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CG, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    QG_CUDA(c, cudaLaunchKernelEx(&cfg, k_softmax_gemm<MODE>, a, ma, mb, mg));
    QG_LAUNCH_CHECK(c);
    return QGBDT_OK;
}

int up(int64_t x, int m) { return (int)((x + m - 1) / m * m); }

// What both directions share: the packed rows and the weight with aligned rows.
struct Common {
    PackArgs pack;
    const void *weight;
    long long ld_weight;
    uint16_t *weight_copy;
    int n_pad, ldp;
};

size_t common_bytes(const SoftmaxArgs &a, bool copy_weight) {
    const int n_pad = up(a.rows, 256), ldp = up(a.dim, 8);
    return qg_ws_size((size_t)n_pad * ldp, 2) + 4 * qg_ws_size((size_t)n_pad, 4) + qg_ws_size(1, 4) + qg_ws_size((size_t)a.rows / PACK_SPAN + 1, 4) +
           (copy_weight ? qg_ws_size((size_t)a.classes * ldp, 2) : 0);
}

bool rows_aligned(const void *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }

int prepare(qgbdt_ctx *c, const SoftmaxArgs &a, QgWorkspace &ws, Common *o, cudaStream_t st) {
    PackArgs &p = o->pack;
    p = PackArgs{};
    o->n_pad = up(a.rows, 256);
    o->ldp = up(a.dim, 8);
    p.labels = a.labels, p.label_type = a.label_type, p.n = (int)a.rows, p.n_pad = o->n_pad, p.classes = (int)a.classes;
    p.hidden = reinterpret_cast<const uint16_t *>(a.hidden), p.ld = a.ld_hidden, p.dim = a.dim;
    p.vec = rows_aligned(a.hidden, a.ld_hidden) && a.dim % 8 == 0;
    p.lse = a.lse_in, p.status = a.status, p.ldp = o->ldp;
    p.packed = ws.take<uint16_t>((size_t)o->n_pad * o->ldp);
    p.row_of = ws.take<int>(o->n_pad), p.pos_of = ws.take<int>(o->n_pad), p.label = ws.take<int>(o->n_pad), p.lse_packed = ws.take<float>(o->n_pad);
    p.count = ws.take<int>(1);
    p.span_count = ws.take<int>(a.rows / PACK_SPAN + 1);
    o->weight = a.weight, o->ld_weight = a.ld_weight;
    if (!rows_aligned(a.weight, a.ld_weight)) {
        uint16_t *copy = ws.take<uint16_t>((size_t)a.classes * o->ldp);
        const long long chunks = a.classes * (o->ldp / 8);
        const long long blocks = (chunks + 255) / 256;
        k_realign<<<(unsigned)(blocks < c->sm_count * 16 ? blocks : c->sm_count * 16), 256, 0, st>>>(
            reinterpret_cast<const uint16_t *>(a.weight), a.ld_weight, a.classes, a.dim, copy, o->ldp);
        QG_LAUNCH_CHECK(c);
        o->weight = copy, o->ld_weight = o->ldp;
    }
    const int spans = (int)((a.rows + PACK_SPAN - 1) / PACK_SPAN);
    if (spans > 1) {
        k_pack_count<<<spans, PACK_THREADS, 0, st>>>(p);
        QG_LAUNCH_CHECK(c);
    }
    k_pack<<<o->n_pad > 0 ? o->n_pad / PACK_ROWS : 1, PACK_THREADS, 0, st>>>(p);
    QG_LAUNCH_CHECK(c);
    return QGBDT_OK;
}

GemmArgs gemm_args(qgbdt_ctx *c, const SoftmaxArgs &a, const Common &o) {
    GemmArgs g{};
    g.count = o.pack.count, g.splits = 1, g.classes = (int)a.classes, g.dim = a.dim, g.bf16 = a.type == QGBDT_BF16, g.fault = c->ops_fault;
    g.bias = a.bias, g.label = o.pack.label, g.lse = o.pack.lse_packed, g.grad_loss = a.grad_loss;
    g.m_tiles = o.n_pad / BM, g.kb = (a.dim + BK - 1) / BK;
    return g;
}

constexpr int64_t PIECE_ELEMENTS = 1ll << 27;   // of g: 256 MiB

// Parts to cut the products' length into so that `tiles` tiles keep all SMs busy; parts hold at least four blocks.
int split_count(int units, long long tiles, int kb) {
    int s = (int)(units / (tiles > 0 ? tiles : 1));
    if (s > kb / 4) s = kb / 4;
    return s < 1 ? 1 : s;
}

template <typename T>
int grad_finish(qgbdt_ctx *c, const float *part, int splits, long long part_rows, int ldp, const int *pos_of, long long rows, int dim,
                const float *grad_loss, const int *count, void *out, long long ld_out, cudaStream_t st) {
    const long long blocks = (rows * ((dim + 3) / 4) + 255) / 256;
    if (blocks <= 0) return QGBDT_OK;
    k_grad_finish<T><<<(unsigned)(blocks < c->sm_count * 16 ? blocks : c->sm_count * 16), 256, 0, st>>>(
        part, splits, part_rows, ldp, pos_of, rows, dim, grad_loss, count, reinterpret_cast<T *>(out), ld_out);
    QG_LAUNCH_CHECK(c);
    return QGBDT_OK;
}

}  // namespace

int qg_softmax_ce(qgbdt_ctx *c, const SoftmaxArgs &a, cudaStream_t st) {
    const bool copy = !rows_aligned(a.weight, a.ld_weight);
    const int n_tiles = up(a.classes, BN) / BN, n_pad = up(a.rows, 256);
    const int join_blocks = a.rows > 0 ? (int)((a.rows + JOIN_ROWS - 1) / JOIN_ROWS) : 1;
    QgWorkspace ws;
    int rc = qg_ws_open(c, common_bytes(a, copy) + qg_ws_size((size_t)n_pad * n_tiles, 8) + qg_ws_size((size_t)n_pad, 4) + qg_ws_size(join_blocks, 8), st, &ws);
    if (rc != QGBDT_OK) return rc;
    Common o;
    if ((rc = prepare(c, a, ws, &o, st)) != QGBDT_OK) return rc;
    GemmArgs g = gemm_args(c, a, o);
    g.n_tiles = n_tiles;
    g.stat = ws.take<float2>((size_t)n_pad * n_tiles);
    g.z_label = ws.take<float>(n_pad);
    double *block_loss = ws.take<double>(join_blocks);
    if (a.rows > 0) {
        CUtensorMap ma, mb;
        if ((rc = matrix_map(c, &ma, o.pack.packed, a.dim, n_pad, o.ldp, 128, g.bf16)) != QGBDT_OK) return rc;
        if ((rc = matrix_map(c, &mb, o.weight, a.dim, a.classes, o.ld_weight, B_ROWS, g.bf16)) != QGBDT_OK) return rc;
        if ((rc = gemm<LOSS>(c, g, ma, mb, ma, st)) != QGBDT_OK) return rc;
    }
    k_loss_join<<<join_blocks, JOIN_ROWS * 32, 0, st>>>(g.stat, n_tiles, g.z_label, o.pack.pos_of, (int)a.rows, o.pack.count, a.losses, a.lse, block_loss,
                                                        c->d_ops_counters, a.loss);
    QG_LAUNCH_CHECK(c);
    return qg_ws_close(c, st);
}

int qg_softmax_ce_backward(qgbdt_ctx *c, const SoftmaxArgs &a, cudaStream_t st) {
    const bool copy = !rows_aligned(a.weight, a.ld_weight);
    const int n_pad = up(a.rows > 0 ? a.rows : 1, 256), units = c->sm_count / CG;
    // pieces of the classes
    int64_t width = PIECE_ELEMENTS / n_pad / 256 * 256;
    if (width < 256) width = 256;
    const int pieces = (int)((a.classes + width - 1) / width);
    width = up((a.classes + pieces - 1) / pieces, 256);
    const int ldf = up(a.dim, 4), d_tiles = (a.dim + BN - 1) / BN;
    const int dh_splits = split_count(units, (long long)(n_pad / BM) * d_tiles, (int)(width / BK));
    const int dw_splits = split_count(units, (width / BM) * d_tiles, n_pad / BK);
    QgWorkspace ws;
    int rc = qg_ws_open(c,
                        common_bytes(a, copy) + qg_ws_size((size_t)n_pad * width, 2) + qg_ws_size((size_t)dh_splits * n_pad * ldf, 4) +
                            (dw_splits > 1 ? qg_ws_size((size_t)dw_splits * width * ldf, 4) : 0) +
                            (a.d_bias ? qg_ws_size((size_t)(n_pad / 32) * width, 4) : 0) + 4096,
                        st, &ws);
    if (rc != QGBDT_OK) return rc;
    Common o;
    if ((rc = prepare(c, a, ws, &o, st)) != QGBDT_OK) return rc;
    uint16_t *g_piece = ws.take<uint16_t>((size_t)n_pad * width);
    float *dh_part = ws.take<float>((size_t)dh_splits * n_pad * ldf);
    float *dw_part = dw_splits > 1 ? ws.take<float>((size_t)dw_splits * width * ldf) : nullptr;
    float *bias_part = a.d_bias ? ws.take<float>((size_t)(n_pad / 32) * width) : nullptr;
    const GemmArgs base = gemm_args(c, a, o);
    const bool bf16 = base.bf16;
    CUtensorMap h_k, h_mn, w_k, w_mn, g_k, g_mn, g_store;
    const int hr = o.n_pad;
    if (hr > 0) {
        if ((rc = matrix_map(c, &h_k, o.pack.packed, a.dim, hr, o.ldp, 128, bf16)) != QGBDT_OK) return rc;
        if ((rc = matrix_map(c, &h_mn, o.pack.packed, a.dim, hr, o.ldp, 64, bf16)) != QGBDT_OK) return rc;
        if ((rc = matrix_map(c, &w_k, o.weight, a.dim, a.classes, o.ld_weight, B_ROWS, bf16)) != QGBDT_OK) return rc;
        if ((rc = matrix_map(c, &w_mn, o.weight, a.dim, a.classes, o.ld_weight, 64, bf16)) != QGBDT_OK) return rc;
        if ((rc = matrix_map(c, &g_k, g_piece, width, hr, width, 128, bf16)) != QGBDT_OK) return rc;
        if ((rc = matrix_map(c, &g_mn, g_piece, width, hr, width, 64, bf16)) != QGBDT_OK) return rc;
        if ((rc = matrix_map(c, &g_store, g_piece, width, hr, width, 32, bf16)) != QGBDT_OK) return rc;
    }
    for (int k = 0; k < pieces; ++k) {
        const int v0 = (int)(k * width);
        const int nv = (int)(a.classes - v0 < width ? a.classes - v0 : width), cols = up(nv, 256);
        if (hr > 0) {
            GemmArgs g = base;
            g.v0 = v0, g.n_tiles = cols / BN, g.bias_part = bias_part;
            if ((rc = gemm<GRAD>(c, g, h_k, w_k, g_store, st)) != QGBDT_OK) return rc;
            if (bias_part) {
                k_bias_finish<<<cols / 32, 256, 0, st>>>(bias_part, cols, nv, a.grad_loss, base.count, a.d_bias + v0);
                QG_LAUNCH_CHECK(c);
            }
            g = base;
            g.v0 = v0, g.n_tiles = d_tiles, g.kb = (nv + BK - 1) / BK, g.splits = dh_splits, g.part = dh_part, g.part_rows = hr, g.ldp = ldf, g.add = k > 0;
            if ((rc = gemm<DH>(c, g, g_k, w_mn, g_k, st)) != QGBDT_OK) return rc;
        } else if (a.d_bias) {
            QG_CUDA(c, cudaMemsetAsync(a.d_bias + v0, 0, sizeof(float) * nv, st));
        }
        GemmArgs g = base;
        g.v0 = v0, g.m_tiles = cols / BM, g.n_tiles = d_tiles, g.splits = dw_splits, g.part = dw_part, g.part_rows = width, g.ldp = ldf;
        if (!dw_part) g.out = a.d_weight, g.ld_out = a.ld_d_weight, g.out_vec = rows_aligned(a.d_weight, a.ld_d_weight);
        if (hr == 0) {   // no rows: no operands, zeros out
            QG_CUDA(c, cudaMemset2DAsync(reinterpret_cast<uint16_t *>(a.d_weight) + v0 * a.ld_d_weight, a.ld_d_weight * 2, 0, (size_t)a.dim * 2, nv, st));
            continue;
        }
        if ((rc = gemm<DW>(c, g, g_mn, h_mn, g_mn, st)) != QGBDT_OK) return rc;
        if (dw_part) {
            char *out = reinterpret_cast<char *>(a.d_weight) + (size_t)v0 * a.ld_d_weight * 2;
            rc = bf16 ? grad_finish<__nv_bfloat16>(c, dw_part, dw_splits, width, ldf, nullptr, nv, a.dim, a.grad_loss, base.count, out, a.ld_d_weight, st)
                      : grad_finish<__half>(c, dw_part, dw_splits, width, ldf, nullptr, nv, a.dim, a.grad_loss, base.count, out, a.ld_d_weight, st);
            if (rc != QGBDT_OK) return rc;
        }
    }
    if (hr > 0) {
        rc = bf16 ? grad_finish<__nv_bfloat16>(c, dh_part, dh_splits, hr, ldf, o.pack.pos_of, a.rows, a.dim, a.grad_loss, base.count, a.d_hidden, a.ld_d_hidden, st)
                  : grad_finish<__half>(c, dh_part, dh_splits, hr, ldf, o.pack.pos_of, a.rows, a.dim, a.grad_loss, base.count, a.d_hidden, a.ld_d_hidden, st);
        if (rc != QGBDT_OK) return rc;
    }
    return qg_ws_close(c, st);
}
