// C ABI of the operators on top of the trees: argument checks and the context's work buffer.
#include <cmath>
#include <new>

#include "ops_internal.cuh"

namespace {

constexpr int OPS_COUNTERS = 64;

int ops_init(qgbdt_ctx *c) {
    if (c->ops_ws_event) return QGBDT_OK;
    if (!c->ops_fault) {
        if (cudaMallocHost(reinterpret_cast<void **>(&c->ops_fault), 64) != cudaSuccess) {
            cudaGetLastError();
            c->ops_fault = nullptr;
            return qg_fail(c, QGBDT_ERR_ALLOC, "cudaMallocHost of 64 bytes failed");
        }
        *c->ops_fault = 0;
    }
    if (!c->d_ops_counters) {
        if (cudaMalloc(reinterpret_cast<void **>(&c->d_ops_counters), OPS_COUNTERS * sizeof(unsigned int)) != cudaSuccess) {
            cudaGetLastError();
            c->d_ops_counters = nullptr;
            return qg_fail(c, QGBDT_ERR_ALLOC, "cudaMalloc of the operators' counters failed");
        }
        QG_CUDA(c, cudaMemset(c->d_ops_counters, 0, OPS_COUNTERS * sizeof(unsigned int)));
        QG_CUDA(c, cudaDeviceSynchronize());
    }
    for (qgbdt_ctx::OpsCapture &e : c->ops_captures)
        if (!e.event) QG_CUDA(c, cudaEventCreateWithFlags(&e.event, cudaEventDisableTiming));
    QG_CUDA(c, cudaEventCreateWithFlags(&c->ops_ws_event, cudaEventDisableTiming));
    return QGBDT_OK;
}

int check_index_type(qgbdt_ctx *c, int32_t t) {
    if (t != QGBDT_I32 && t != QGBDT_I64) return qg_fail(c, QGBDT_ERR_ARG, "index type must be QGBDT_I32 or QGBDT_I64");
    return QGBDT_OK;
}

int check_embed(qgbdt_ctx *c, EmbedArgs &a, bool backward) {
    qg_single_row(backward ? a.rows : a.n_entries, a.dim, 1, &a.ld);
    qg_single_row(backward ? a.n_entries : a.rows, a.dim, 1, &a.ld_out);
    int rc = qg_ops_enter(c);
    if (rc != QGBDT_OK) return rc;
    if (!qg_type_ok(a.type)) return qg_fail(c, QGBDT_ERR_ARG, "element type must be QGBDT_F32, QGBDT_BF16 or QGBDT_F16");
    if ((rc = check_index_type(c, a.token_type)) != QGBDT_OK) return rc;
    if (a.rows < 0 || a.n_entries < 1 || a.n_entries >= (1ll << 31) - 1) return qg_fail(c, QGBDT_ERR_ARG, "rows must be >= 0 and n_entries in [1, 2^31 - 1)");
    if (a.dim < 1 || a.dim > (1 << 20)) return qg_fail(c, QGBDT_ERR_ARG, "dim must be in [1, 2^20]");
    if (a.bag < 1 || a.bag > (1 << 20)) return qg_fail(c, QGBDT_ERR_ARG, "bag must be in [1, 2^20]");
    if (a.rows > ((1ll << 31) - 1) / a.bag) return qg_fail(c, QGBDT_ERR_ARG, "rows * bag must be below 2^31");
    if (a.ld < a.dim || a.ld_out < a.dim || a.ld_tokens < a.bag) return qg_fail(c, QGBDT_ERR_ARG, "a row stride is smaller than the row");
    if (a.ld >= (1ll << 30) || a.ld_out >= (1ll << 30)) return qg_fail(c, QGBDT_ERR_ARG, "row strides must be below 2^30");
    if (!std::isfinite(a.scale)) return qg_fail(c, QGBDT_ERR_ARG, "scale must be finite");
    const bool none = a.rows == 0;
    if ((!none && (!a.table || !a.tokens)) || (!a.out && !(none && !backward))) return qg_fail(c, QGBDT_ERR_ARG, "null pointer");
    const int w = qg_type_size(a.type);
    if (!qg_aligned(a.table, w) || !qg_aligned(a.out, w) || !qg_aligned(a.tokens, a.token_type == QGBDT_I64 ? 8 : 4) || !qg_aligned(a.status, 4))
        return qg_fail(c, QGBDT_ERR_ARG, "a pointer is not aligned to its element");
    return QGBDT_OK;
}

int check_softmax(qgbdt_ctx *c, SoftmaxArgs &a) {
    qg_single_row(a.rows, a.dim, 8, &a.ld_hidden);
    qg_single_row(a.classes, a.dim, 8, &a.ld_weight);
    qg_single_row(a.rows, a.dim, 8, &a.ld_d_hidden);
    qg_single_row(a.classes, a.dim, 8, &a.ld_d_weight);
    int rc = qg_ops_enter(c);
    if (rc != QGBDT_OK) return rc;
    if (a.type != QGBDT_BF16 && a.type != QGBDT_F16) return qg_fail(c, QGBDT_ERR_ARG, "hidden and weight must be QGBDT_BF16 or QGBDT_F16");
    if ((rc = check_index_type(c, a.label_type)) != QGBDT_OK) return rc;
    if (a.rows < 0 || a.rows > (1ll << 24)) return qg_fail(c, QGBDT_ERR_ARG, "rows must be in [0, 2^24]");
    if (a.classes < 1 || a.classes > (1ll << 24)) return qg_fail(c, QGBDT_ERR_ARG, "classes must be in [1, 2^24]");
    if (a.dim < 1 || a.dim > (1 << 16)) return qg_fail(c, QGBDT_ERR_ARG, "dim must be in [1, 2^16]");
    if (a.ld_hidden < a.dim || a.ld_weight < a.dim) return qg_fail(c, QGBDT_ERR_ARG, "a row stride is smaller than the row");
    const int64_t most = 1ll << 39;   // tiled copies take strides below 2^40 bytes
    if (a.ld_hidden >= most || a.ld_weight >= most || a.ld_d_hidden >= most || a.ld_d_weight >= most)
        return qg_fail(c, QGBDT_ERR_ARG, "row strides must be below 2^39");
    if (!a.weight || (a.rows > 0 && (!a.hidden || !a.labels))) return qg_fail(c, QGBDT_ERR_ARG, "null pointer");
    if (!qg_aligned(a.hidden, 2) || !qg_aligned(a.weight, 2) || !qg_aligned(a.bias, 4) || !qg_aligned(a.labels, a.label_type == QGBDT_I64 ? 8 : 4) || !qg_aligned(a.status, 4))
        return qg_fail(c, QGBDT_ERR_ARG, "a pointer is not aligned to its element");
    return QGBDT_OK;
}

// The last call of a capture, or NULL.
qgbdt_ctx::OpsCapture *last_of_capture(qgbdt_ctx *c, unsigned long long id) {
    for (qgbdt_ctx::OpsCapture &e : c->ops_captures)
        if (e.used && e.id == id) return &e;
    return nullptr;
}

}  // namespace

int qg_ops_enter(qgbdt_ctx *c) {
    if (!c) return QGBDT_ERR_ARG;
    if (c->ops_fault && *static_cast<volatile int *>(c->ops_fault)) {
        *static_cast<volatile int *>(c->ops_fault) = 0;
        return qg_fail(c, QGBDT_ERR_CUDA, "a kernel of an earlier operator call gave up waiting for its copies; that call's results are not valid");
    }
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess || device != c->device) {
        cudaGetLastError();
        return qg_fail(c, QGBDT_ERR_STATE, "the context belongs to device %d, the current one is %d", c->device, device);
    }
    return QGBDT_OK;
}

// End of a call: one that failed on its way may have launched kernels, which the next call has to wait for all the same.
int qg_ops_leave(qgbdt_ctx *c, int rc, void *stream) {
    if (c->ops_ws_open) {
        const int closed = qg_ws_close(c, (cudaStream_t)stream);
        if (rc == QGBDT_OK) rc = closed;
    }
    return rc;
}

int qg_ws_open(qgbdt_ctx *c, size_t bytes, cudaStream_t st, QgWorkspace *ws) {
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    unsigned long long capture = 0;
    QG_CUDA(c, cudaStreamGetCaptureInfo(st, &cap, &capture));
    const bool capturing = cap != cudaStreamCaptureStatusNone;
    if (capturing && (!c->ops_ws_event || bytes > c->ops_ws_bytes))
        return qg_fail(c, QGBDT_ERR_STATE, "the work buffer has to grow: make one call of this size before the stream is captured");
    int rc = ops_init(c);
    if (rc != QGBDT_OK) return rc;
    if (bytes > c->ops_ws_bytes) {
        if (c->ops_ws) {
            if (c->ops_ws_captured) {
                // a graph may hold its address; nothing is waited for, and a call that still runs shares the counters with
                // this one, so that the event goes on to order them
                try {
                    c->ops_ws_old.push_back(c->ops_ws);
                } catch (const std::bad_alloc &) {
                    return qg_fail(c, QGBDT_ERR_ALLOC, "no host memory to keep track of the work buffers");
                }
                c->ops_ws_captured = false;   // over the buffer that takes its place
            } else {
                if (c->ops_ws_used) QG_CUDA(c, cudaEventSynchronize(c->ops_ws_event));
                c->ops_ws_used = false;
                cudaFree(c->ops_ws);
            }
            c->ops_ws = nullptr;
            c->ops_ws_bytes = 0;
        }
        const size_t want = (bytes + (bytes >> 3) + 0xfffff) & ~(size_t)0xfffff;   // an eighth more: growing costs a synchronisation
        if (cudaMalloc(&c->ops_ws, want) != cudaSuccess) {
            cudaGetLastError();
            c->ops_ws = nullptr;
            return qg_fail(c, QGBDT_ERR_ALLOC, "cudaMalloc of %zu bytes of work memory failed", want);
        }
        c->ops_ws_bytes = want;
    }
    if (capturing) {
        c->ops_ws_captured = true;
        const qgbdt_ctx::OpsCapture *last = last_of_capture(c, capture);
        if (last && last->stream != st) QG_CUDA(c, cudaStreamWaitEvent(st, last->event, 0));
    } else if (c->ops_ws_used) {
        unsigned long long id = 0;
        QG_CUDA(c, cudaStreamGetId(st, &id));
        if (id != c->ops_ws_stream) QG_CUDA(c, cudaStreamWaitEvent(st, c->ops_ws_event, 0));
    }
    c->ops_ws_open = true;
    ws->at = reinterpret_cast<char *>(c->ops_ws);
    ws->end = ws->at + c->ops_ws_bytes;
    return QGBDT_OK;
}

int qg_ws_close(qgbdt_ctx *c, cudaStream_t st) {
    c->ops_ws_open = false;
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    unsigned long long capture = 0;
    QG_CUDA(c, cudaStreamGetCaptureInfo(st, &cap, &capture));
    if (cap != cudaStreamCaptureStatusNone) {
        qgbdt_ctx::OpsCapture *last = last_of_capture(c, capture);
        if (!last) {
            last = &c->ops_captures[c->ops_capture_next];
            c->ops_capture_next = (c->ops_capture_next + 1) % (int)(sizeof(c->ops_captures) / sizeof(*last));
            last->used = false;
        }
        QG_CUDA(c, cudaEventRecord(last->event, st));
        last->id = capture, last->stream = st, last->used = true;
        return QGBDT_OK;
    }
    QG_CUDA(c, cudaStreamGetId(st, &c->ops_ws_stream));
    QG_CUDA(c, cudaEventRecord(c->ops_ws_event, st));
    c->ops_ws_used = true;
    return QGBDT_OK;
}

void qg_ops_destroy(qgbdt_ctx *c) {
    for (void *p : c->ops_ws_old) cudaFree(p);
    c->ops_ws_old.clear();
    if (c->ops_ws) cudaFree(c->ops_ws);
    if (c->d_ops_counters) cudaFree(c->d_ops_counters);
    if (c->ops_fault) cudaFreeHost(c->ops_fault);
    if (c->ops_ws_event) cudaEventDestroy(c->ops_ws_event);
    for (qgbdt_ctx::OpsCapture &e : c->ops_captures) {
        if (e.event) cudaEventDestroy(e.event);
        e = qgbdt_ctx::OpsCapture{};
    }
    c->ops_ws = nullptr;
    c->d_ops_counters = nullptr;
    c->ops_fault = nullptr;
    c->ops_ws_event = nullptr;
}

extern "C" {

int qgbdt_embed(qgbdt_ctx *c, const void *d_table, int32_t type, int64_t n_entries, int32_t dim, int64_t ld_table,
                const void *d_tokens, int32_t token_type, int64_t n_rows, int32_t bag, int64_t ld_tokens, float scale,
                void *d_out, int64_t ld_out, int32_t *d_status, void *stream) {
    EmbedArgs a{d_table, ld_table, n_entries, dim, type, d_tokens, token_type, n_rows, ld_tokens, bag, scale, d_out, ld_out, d_status};
    int rc = check_embed(c, a, false);
    if (rc != QGBDT_OK || n_rows == 0) return rc;
    return qg_ops_leave(c, qg_embed(c, a, (cudaStream_t)stream), stream);
}

int qgbdt_embed_backward(qgbdt_ctx *c, const void *d_grad, int32_t type, int64_t ld_grad, const void *d_tokens, int32_t token_type,
                         int64_t n_rows, int32_t bag, int64_t ld_tokens, float scale, void *d_grad_table, int64_t n_entries,
                         int32_t dim, int64_t ld_grad_table, int32_t *d_status, void *stream) {
    EmbedArgs a{d_grad, ld_grad, n_entries, dim, type, d_tokens, token_type, n_rows, ld_tokens, bag, scale, d_grad_table, ld_grad_table, d_status};
    int rc = check_embed(c, a, true);
    if (rc != QGBDT_OK) return rc;
    return qg_ops_leave(c, qg_embed_backward(c, a, (cudaStream_t)stream), stream);
}

int qgbdt_softmax_ce(qgbdt_ctx *c, const void *d_hidden, int64_t ld_hidden, const void *d_weight, int64_t ld_weight, int32_t type,
                     const float *d_bias, const void *d_labels, int32_t label_type, int64_t n_rows, int64_t n_classes, int32_t dim,
                     float *d_loss, float *d_losses, float *d_lse, int32_t *d_status, void *stream) {
    SoftmaxArgs a{};
    a.hidden = d_hidden, a.ld_hidden = ld_hidden, a.weight = d_weight, a.ld_weight = ld_weight, a.type = type, a.bias = d_bias;
    a.labels = d_labels, a.label_type = label_type, a.rows = n_rows, a.classes = n_classes, a.dim = dim;
    a.loss = d_loss, a.losses = d_losses, a.lse = d_lse, a.status = d_status;
    int rc = check_softmax(c, a);
    if (rc != QGBDT_OK) return rc;
    if (!d_loss || (n_rows > 0 && !d_lse)) return qg_fail(c, QGBDT_ERR_ARG, "null pointer");
    if (!qg_aligned(d_loss, 4) || !qg_aligned(d_losses, 4) || !qg_aligned(d_lse, 4)) return qg_fail(c, QGBDT_ERR_ARG, "a pointer is not aligned to its element");
    return qg_ops_leave(c, qg_softmax_ce(c, a, (cudaStream_t)stream), stream);
}

int qgbdt_softmax_ce_backward(qgbdt_ctx *c, const void *d_hidden, int64_t ld_hidden, const void *d_weight, int64_t ld_weight,
                              int32_t type, const float *d_bias, const void *d_labels, int32_t label_type, int64_t n_rows,
                              int64_t n_classes, int32_t dim, const float *d_lse, const float *d_grad_loss, void *d_grad_hidden,
                              int64_t ld_grad_hidden, void *d_grad_weight, int64_t ld_grad_weight, float *d_grad_bias,
                              int32_t *d_status, void *stream) {
    SoftmaxArgs a{};
    a.hidden = d_hidden, a.ld_hidden = ld_hidden, a.weight = d_weight, a.ld_weight = ld_weight, a.type = type, a.bias = d_bias;
    a.labels = d_labels, a.label_type = label_type, a.rows = n_rows, a.classes = n_classes, a.dim = dim;
    a.lse_in = d_lse, a.grad_loss = d_grad_loss, a.d_hidden = d_grad_hidden, a.ld_d_hidden = ld_grad_hidden;
    a.d_weight = d_grad_weight, a.ld_d_weight = ld_grad_weight, a.d_bias = d_grad_bias, a.status = d_status;
    int rc = check_softmax(c, a);
    if (rc != QGBDT_OK) return rc;
    if (!d_grad_weight || (n_rows > 0 && (!d_lse || !d_grad_hidden))) return qg_fail(c, QGBDT_ERR_ARG, "null pointer");
    if ((n_rows > 0 && a.ld_d_hidden < dim) || a.ld_d_weight < dim) return qg_fail(c, QGBDT_ERR_ARG, "a row stride is smaller than the row");
    if (!qg_aligned(d_grad_hidden, 2) || !qg_aligned(d_grad_weight, 2) || !qg_aligned(d_lse, 4) || !qg_aligned(d_grad_loss, 4) || !qg_aligned(d_grad_bias, 4))
        return qg_fail(c, QGBDT_ERR_ARG, "a pointer is not aligned to its element");
    return qg_ops_leave(c, qg_softmax_ce_backward(c, a, (cudaStream_t)stream), stream);
}

int qgbdt_clip_grad_norm(qgbdt_ctx *c, const void *const *h_grads, void *const *h_out, const int64_t *h_counts, const int32_t *h_types,
                         int32_t n_tensors, double max_norm, float *d_norm, void *stream) {
    int rc = qg_ops_enter(c);
    if (rc != QGBDT_OK) return rc;
    if (n_tensors < 0 || n_tensors > (1 << 20)) return qg_fail(c, QGBDT_ERR_ARG, "n_tensors must be in [0, 2^20]");
    if (!d_norm || (n_tensors > 0 && (!h_grads || !h_counts || !h_types))) return qg_fail(c, QGBDT_ERR_ARG, "null pointer");
    if (!(max_norm >= 0.0)) return qg_fail(c, QGBDT_ERR_ARG, "max_norm must be >= 0 (infinity: the norm alone)");
    if (!qg_aligned(d_norm, 4)) return qg_fail(c, QGBDT_ERR_ARG, "a pointer is not aligned to its element");
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (h_counts[i] < 0) return qg_fail(c, QGBDT_ERR_ARG, "tensor %d has a negative size", i);
        if (!qg_type_ok(h_types[i])) return qg_fail(c, QGBDT_ERR_ARG, "tensor %d: element type must be QGBDT_F32, QGBDT_BF16 or QGBDT_F16", i);
        if (h_counts[i] == 0) continue;
        if (!h_grads[i] || (h_out && !h_out[i])) return qg_fail(c, QGBDT_ERR_ARG, "tensor %d is NULL", i);
        const int w = qg_type_size(h_types[i]);
        if (!qg_aligned(h_grads[i], w) || (h_out && !qg_aligned(h_out[i], w))) return qg_fail(c, QGBDT_ERR_ARG, "tensor %d is not aligned to its element", i);
    }
    void *const *out = h_out ? h_out : const_cast<void *const *>(reinterpret_cast<const void *const *>(h_grads));
    return qg_ops_leave(c, qg_clip_grad_norm(c, h_grads, out, h_counts, h_types, n_tensors, max_norm, d_norm, (cudaStream_t)stream), stream);
}

}  // extern "C"
