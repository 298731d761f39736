// The operators' work buffer (csrc/api_ops.cu) over a stand-in for the CUDA runtime.  Runs without a GPU; argv[1] names the
// scenario.
#include <cstdio>
#include <cstdlib>

#include "ops_internal.cuh"

#include "fake_cuda.h"

int qg_fail(qgbdt_ctx *, int code, const char *, ...) { return code; }
static int embed_result = QGBDT_OK;
int qg_embed(qgbdt_ctx *c, const EmbedArgs &, cudaStream_t st) {   // opens the buffer, and may fail in the middle
    QgWorkspace ws;
    QG_RUN(qg_ws_open(c, 1000, st, &ws));
    if (embed_result != QGBDT_OK) return embed_result;
    return qg_ws_close(c, st);
}
int qg_embed_backward(qgbdt_ctx *, const EmbedArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_softmax_ce(qgbdt_ctx *, const SoftmaxArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_softmax_ce_backward(qgbdt_ctx *, const SoftmaxArgs &, cudaStream_t) { return QGBDT_OK; }
int qg_clip_grad_norm(qgbdt_ctx *, const void *const *, void *const *, const int64_t *, const int32_t *, int32_t, double, float *, cudaStream_t) { return QGBDT_OK; }

static const cudaStream_t A = (cudaStream_t)1, B = (cudaStream_t)2, C = (cudaStream_t)3;
static const size_t SMALL = 1000, LARGE = 64 << 20, LARGER = 256 << 20;

#define CHECK(x)                                                          \
    do {                                                                  \
        if (!(x)) {                                                       \
            printf("line %d: %s does not hold; calls:\n", __LINE__, #x);  \
            for (const std::string &s : calls) printf("  %s\n", s.c_str()); \
            exit(1);                                                      \
        }                                                                 \
    } while (0)

static qgbdt_ctx c;
static void *use(size_t bytes, cudaStream_t st) {   // one call
    QgWorkspace ws;
    CHECK(qg_ws_open(&c, bytes, st, &ws) == QGBDT_OK);
    CHECK(qg_ws_close(&c, st) == QGBDT_OK);
    return ws.at;
}
static void capture_one(size_t bytes) {
    captures[C] = 77;
    use(bytes, C);
    captures.clear();
}
static int embed(cudaStream_t st) {
    return qgbdt_embed(&c, &c, QGBDT_F32, 4, 4, 4, &c, QGBDT_I32, 1, 1, 1, 1.0f, &c, 4, nullptr, st);
}

int main(int argc, char **argv) {
    const std::string scenario = argc > 1 ? argv[1] : "";
    void *const first = use(SMALL, A);
    if (scenario == "streams") {
        use(SMALL, A);
        CHECK(!noted("wait", A, c.ops_ws_event));
        use(SMALL, B);
        CHECK(noted("wait", B, c.ops_ws_event) && noted("record", c.ops_ws_event, B));
    } else if (scenario == "grow") {   // waits for the last call, then frees its buffer
        use(LARGE, B);
        CHECK(noted("sync", c.ops_ws_event, nullptr) && noted("free", first, nullptr));
    } else if (scenario == "grow after a capture") {   // keeps the buffer, and the order with the last call
        capture_one(SMALL);
        use(LARGE, B);
        CHECK(!noted("free", first, nullptr));
        CHECK(noted("wait", B, c.ops_ws_event) || noted("sync", c.ops_ws_event, nullptr));
    } else if (scenario == "grow twice after a capture") {   // only the buffer under the graph is kept
        capture_one(SMALL);
        void *const second = use(LARGE, A);
        use(LARGER, A);
        CHECK(!noted("free", first, nullptr) && noted("free", second, nullptr));
    } else if (scenario == "one capture") {   // branches of one graph wait for one another's calls
        captures[A] = captures[B] = 5;
        calls.clear();
        use(SMALL, A);
        use(SMALL, B);
        bool joined = false;
        for (cudaEvent_t e = (cudaEvent_t)100; (long)(intptr_t)e < next_handle; e = (cudaEvent_t)((intptr_t)e + 1))
            joined = joined || (noted("record", e, A) && noted("wait", B, e));
        CHECK(joined);
    } else if (scenario == "two captures") {   // nothing joins one capture to another, or to calls outside
        captures[A] = 5, captures[B] = 6;
        calls.clear();
        use(SMALL, A);
        use(SMALL, B);
        use(SMALL, A);
        use(SMALL, C);
        for (const std::string &s : calls) CHECK(s.compare(0, 4, "wait") != 0 || s.compare(0, 6, "wait 3") == 0);
        for (cudaEvent_t e = (cudaEvent_t)100; (long)(intptr_t)e < next_handle; e = (cudaEvent_t)((intptr_t)e + 1))
            CHECK(!(noted("wait", C, e) && (noted("record", e, A) || noted("record", e, B))) || e == c.ops_ws_event);
    } else if (scenario == "failure") {   // what a call that failed on its way has launched is waited for
        embed_result = QGBDT_ERR_CUDA;
        CHECK(embed(B) == QGBDT_ERR_CUDA);
        CHECK(noted("record", c.ops_ws_event, B));
        embed_result = QGBDT_OK;
        CHECK(embed(A) == QGBDT_OK && noted("wait", A, c.ops_ws_event));
    } else if (scenario == "no host memory") {   // an error code, not an exception through the C entry
        capture_one(SMALL);
        no_memory = true;
        QgWorkspace ws;
        const int rc = qg_ws_open(&c, LARGE, A, &ws);
        no_memory = false;
        CHECK(rc == QGBDT_ERR_ALLOC);
        CHECK(use(SMALL, A) == first);
    } else {
        CHECK(!"a scenario of this name");
    }
    printf("ok\n");
    return 0;
}
