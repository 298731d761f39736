#include "fake_cuda.h"

#include <cstdio>
#include <cstdlib>
#include <new>

std::vector<std::string> calls;
std::map<cudaStream_t, unsigned long long> captures;
long next_handle = 100;
bool no_memory = false;

static void note(const char *what, const void *a, const void *b) {
    char text[96];
    snprintf(text, sizeof(text), "%s %ld %ld", what, (long)(intptr_t)a, (long)(intptr_t)b);
    calls.push_back(text);
}
bool noted(const char *what, const void *a, const void *b) {
    char text[96];
    snprintf(text, sizeof(text), "%s %ld %ld", what, (long)(intptr_t)a, (long)(intptr_t)b);
    for (const std::string &s : calls)
        if (s == text) return true;
    return false;
}

void *operator new(size_t n) {
    if (no_memory) throw std::bad_alloc();
    return malloc(n);
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

extern "C" {
cudaError_t cudaMallocHost(void **p, size_t n) { return *p = calloc(1, n), cudaSuccess; }
cudaError_t cudaFreeHost(void *p) { return free(p), cudaSuccess; }
cudaError_t cudaMalloc(void **p, size_t) { return *p = (void *)(next_handle++), cudaSuccess; }
cudaError_t cudaFree(void *p) { return note("free", p, nullptr), cudaSuccess; }
cudaError_t cudaMemset(void *, int, size_t) { return cudaSuccess; }
cudaError_t cudaDeviceSynchronize() { return cudaSuccess; }
cudaError_t cudaGetDevice(int *d) { return *d = 0, cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
const char *cudaGetErrorString(cudaError_t) { return "error"; }
cudaError_t cudaEventCreateWithFlags(cudaEvent_t *e, unsigned) { return *e = (cudaEvent_t)(next_handle++), cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t e, cudaStream_t s) { return note("record", e, s), cudaSuccess; }
cudaError_t cudaEventSynchronize(cudaEvent_t e) { return note("sync", e, nullptr), cudaSuccess; }
cudaError_t cudaStreamWaitEvent(cudaStream_t s, cudaEvent_t e, unsigned) { return note("wait", s, e), cudaSuccess; }
cudaError_t cudaStreamGetId(cudaStream_t s, unsigned long long *id) { return *id = (unsigned long long)(intptr_t)s, cudaSuccess; }
cudaError_t cudaStreamIsCapturing(cudaStream_t s, cudaStreamCaptureStatus *c) {
    return *c = captures.count(s) ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone, cudaSuccess;
}
cudaError_t cudaStreamGetCaptureInfo_v2(cudaStream_t s, cudaStreamCaptureStatus *c, unsigned long long *id, cudaGraph_t *, const cudaGraphNode_t **, size_t *) {
    cudaStreamIsCapturing(s, c);
    if (id && captures.count(s)) *id = captures[s];
    return cudaSuccess;
}
}

// nvcc's start-up code registers kernels through these; there are none
extern "C" {
void **__cudaRegisterFatBinary(void *) { return nullptr; }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
}
