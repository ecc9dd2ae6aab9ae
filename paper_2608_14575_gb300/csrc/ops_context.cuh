// A context of the operators (hwr_ops.h) as their host code sees it: its members,
// errors, memory, and what a call checks before it queues anything.
#pragma once

#include <cudaTypedefs.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <new>
#include <string>

#include <nvtx3/nvToolsExt.h>

#include "ops_internal.cuh"

namespace hwr {

inline PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;
inline thread_local std::string g_create_error;      // of hwr_ops_create

struct ApiRange {
    explicit ApiRange(const char *name) { nvtxRangePushA(name); }
    ~ApiRange() { nvtxRangePop(); }
    ApiRange(const ApiRange &) = delete;
    ApiRange &operator=(const ApiRange &) = delete;
};

// Memory is taken and given back beside captures of other streams: without this, a
// capture that watches the thread (the usual kind) would be spoilt by it.
struct Unwatched {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    Unwatched() { cudaThreadExchangeStreamCaptureMode(&mode); }
    ~Unwatched() { cudaThreadExchangeStreamCaptureMode(&mode); }
    Unwatched(const Unwatched &) = delete;
    Unwatched &operator=(const Unwatched &) = delete;
};

// Device memory that a captured graph may hold, kept until the context goes.
struct Retired {
    void *p;
    Retired *next;
};

}  // namespace hwr

using namespace hwr;

struct hwr_gradients {
    ClipChunk *table = nullptr;
    int chunks = 0, per = 1;
    mutable bool held = false;          // a captured call has the table's address
    hwr_gradients *next = nullptr;      // of the context's lists
};

struct hwr_adamw {
    AdamWTensor *tensors = nullptr;     // device: the tensors, then
    AdamWChunk *table = nullptr;        // their chunks
    int n = 0, bits = 32;
    int *chunk0 = nullptr;              // host, [n + 1]: first chunk of each tensor
    int32_t *step = nullptr;
    mutable bool held = false;
    hwr_adamw *next = nullptr;          // of the context's optimizers
};

// Words that blocks count their arrivals in (zeroed once, self-resetting).
constexpr int ARRIVALS_ROWS = 0, ARRIVALS_STEP = 1024, ARRIVALS = ARRIVALS_STEP + 1;

struct hwr_ops {
    cudaStream_t stream = nullptr;
    bool own_stream = false, broken = false;
    int device = 0;
    int nsm = 1, ctas = 2;       // SMs; CTAs of the grouped products
    int cluster = 8;             // blocks of a dispatch's clusters (test hook HWR_TEST_SMALL_CLUSTERS: 8)
    std::string err;
    char *ws = nullptr;
    size_t ws_cap = 0;
    bool ws_held = false;        // a captured call has its address
    Retired *retired = nullptr;
    hwr_gradients *lists = nullptr;
    hwr_adamw *optimizers = nullptr;
    uint32_t *arrivals = nullptr;
    float *part = nullptr;       // partial tiles of the grouped products
    uint32_t *count = nullptr;   // their arrivals (zeroed once, self-resetting)
    double *sums = nullptr;      // partial sums of squares; then their arrivals and the factor
    int32_t *status_h = nullptr, *status_d = nullptr;   // mapped: bounded waits that ran out
    cudaEvent_t event = nullptr;                         // hwr_ops_after / before
    int test_stall = 0;                                  // HWR_TEST_STALL (see hwr_api.cu)
    int test_device = 0;                                 // HWR_TEST_DEVICE: how far off the current device seems
    long fail_at = 0, allocs = 0;                        // HWR_TEST_FAIL_ALLOC
    long fail_launch = 0, launches = 0;                  // HWR_TEST_FAIL_LAUNCH: of optimizers' kernels, this one fails
};

static inline hwr_status fail(hwr_ops *c, hwr_status s, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    if (c) {
        c->err = buf;
        if (s == HWR_ERR_CUDA || s == HWR_ERR_TIMEOUT) c->broken = true;
    } else {
        g_create_error = buf;
    }
    return s;
}

static inline hwr_status cuda_fail(hwr_ops *c, cudaError_t e, const char *what) {
    return fail(c, e == cudaErrorMemoryAllocation ? HWR_ERR_OOM : HWR_ERR_CUDA, "%s: %s", what,
                cudaGetErrorString(e));
}

#define CK(ctx, call, what)                                     \
    do {                                                        \
        cudaError_t e_ = (call);                                \
        if (e_ != cudaSuccess) return cuda_fail(ctx, e_, what); \
    } while (0)
#define OK(call)                              \
    do {                                      \
        const hwr_status s_ = (call);         \
        if (s_ != HWR_OK) return s_;          \
    } while (0)

static inline hwr_status alive(hwr_ops *c) {
    if (c->broken) return fail(c, HWR_ERR_STATE, "context unusable after an earlier failure");
    if (*(volatile int32_t *)c->status_h != ST_OK)
        return fail(c, HWR_ERR_TIMEOUT, "a device-side wait of an earlier call gave up");
    return HWR_OK;
}

// For calls that launch or allocate.
static inline hwr_status ready(hwr_ops *c) {
    OK(alive(c));
    // (a launch on another device's stream would fail, and break the context)
    int dev = c->device;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(c, e, "cudaGetDevice");
    if (dev + c->test_device != c->device)
        return fail(c, HWR_ERR_INVALID_ARG, "device %d is current, the context is of device %d", dev + c->test_device,
                    c->device);
    return HWR_OK;
}

template <class T>
static inline hwr_status alloc(hwr_ops *c, T **p, size_t n) {
    *p = nullptr;
    if (c->fail_at > 0 && ++c->allocs == c->fail_at)
        return fail(c, HWR_ERR_OOM, "allocation %ld failed (test hook)", c->allocs);
    const Unwatched memory;
    const cudaError_t e = cudaMalloc((void **)p, n * sizeof(T));
    if (e != cudaSuccess) {
        cudaGetLastError();
        *p = nullptr;
        return fail(c, HWR_ERR_OOM, "cudaMalloc(%zu): %s", n * sizeof(T), cudaGetErrorString(e));
    }
    return HWR_OK;
}

// Whether what the context queues now goes into a graph.
static inline hwr_status capturing(hwr_ops *c, bool *yes) {
    *yes = false;
    if (c->stream == cudaStreamLegacy) return HWR_OK;      // (takes no part in captures)
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    CK(c, cudaStreamIsCapturing(c->stream, &st), "capture status");
    *yes = st != cudaStreamCaptureStatusNone;
    return HWR_OK;
}

static inline hwr_status retire(hwr_ops *c, void *p) {
    Retired *r = new (std::nothrow) Retired{p, c->retired};
    if (!r) return fail(c, HWR_ERR_OOM, "host allocation failed");
    c->retired = r;
    return HWR_OK;
}

// A block that a captured call has used stays when a larger one takes its place:
// the graph's replays go on using it.
static inline hwr_status reserve(hwr_ops *c, size_t bytes) {
    bool captured;
    OK(capturing(c, &captured));
    if (bytes <= c->ws_cap) {
        c->ws_held = c->ws_held || (captured && bytes);
        return HWR_OK;
    }
    if (captured)
        return fail(c, HWR_ERR_UNSUPPORTED, "the workspace cannot grow (to %zu bytes) during a stream capture", bytes);
    if (c->ws) {
        if (c->ws_held) {
            OK(retire(c, c->ws));
        } else {
            CK(c, cudaStreamSynchronize(c->stream), "synchronize before regrow");
            const Unwatched memory;
            cudaFree(c->ws);
        }
        c->ws = nullptr;
        c->ws_cap = 0;
        c->ws_held = false;
    }
    const size_t want = bytes <= SIZE_MAX / 2 ? bytes + bytes / 8 : bytes;
    OK(alloc(c, &c->ws, want));
    c->ws_cap = want;
    return HWR_OK;
}

