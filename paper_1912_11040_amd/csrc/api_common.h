// What the files behind the C ABI share: errors, growing the context's buffers, pinned staging, stage marks.
#pragma once

#include <cstdarg>
#include <cstdio>

#include "aug_internal.h"

namespace aug {

inline int fail(aug_ctx* ctx, int code, const char* fmt, ...) {
    if (ctx) {
        char msg[512];
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(msg, sizeof msg, fmt, ap);
        va_end(ap);
        ctx->last_error = msg;
    }
    return code;
}

inline int fail_hip(aug_ctx* ctx, hipError_t e, const char* what) {
    (void)hipGetLastError();
    if (e == hipErrorOutOfMemory) return fail(ctx, AUG_ERR_NOMEM, "%s: out of device memory", what);
    return fail(ctx, AUG_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

#define AUG_HIP(expr, what)                                        \
    do {                                                           \
        hipError_t e__ = (expr);                                   \
        if (e__ != hipSuccess) return fail_hip(ctx, e__, what);    \
    } while (0)

#define AUG_TRY(expr)                                              \
    do {                                                           \
        int rc__ = (expr);                                         \
        if (rc__ != AUG_OK) return rc__;                           \
    } while (0)

// Grow one of the context's device buffers.  Growing frees the old allocation (which waits for the work
// that uses it) and allocates: neither may happen while the stream is being captured into a graph.
inline int grow(aug_ctx* ctx, DeviceBuffer& b, size_t bytes, const char* what) {
    if (bytes <= b.bytes) return AUG_OK;
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(ctx->stream, &st) != hipSuccess) (void)hipGetLastError();
    if (st != hipStreamCaptureStatusNone)
        return fail(ctx, AUG_ERR_UNSUPPORTED, "%s would have to grow while the stream is being captured: "
                    "run the same call once before capturing it", what);
    hipError_t e = b.reserve(bytes);
    if (e != hipSuccess) return fail_hip(ctx, e, what);
    return AUG_OK;
}

// Bytes of a staging slot for n_utt + 1 = n entries: two int64 and two int arrays.
inline size_t ring_bytes(size_t n) { return n * (2 * sizeof(int64_t) + 2 * sizeof(int)); }

// Pinned staging slots of at least `bytes` each, with their events.
inline int ring_reserve(aug_ctx* ctx, size_t bytes) {
    HostRing& r = ctx->ring;
    if (bytes <= r.bytes) return AUG_OK;
    AUG_HIP(hipStreamSynchronize(ctx->stream), "stream synchronize");       // kernels still read the old slots
    if (r.host) {
        AUG_HIP(hipHostFree(r.host), "staging free");
        r.host = nullptr;
    }
    r.bytes = 0;
    const size_t want = (bytes + bytes / 4 + 4095) & ~(size_t)4095;
    AUG_HIP(hipHostMalloc(reinterpret_cast<void**>(&r.host), want * HostRing::kSlots, hipHostMallocDefault),
            "pinned staging buffer");
    AUG_HIP(hipHostGetDevicePointer(reinterpret_cast<void**>(&r.device), r.host, 0), "pinned staging address");
    for (hipEvent_t& e : r.done)
        if (!e) AUG_HIP(hipEventCreateWithFlags(&e, hipEventDisableTiming), "staging event");
    r.bytes = want;
    return AUG_OK;
}

// The kernel that reads the current staging slot has been enqueued.
inline int packing_launched(aug_ctx* ctx) {
    HostRing& r = ctx->ring;
    const int i = r.next, e = i / HostRing::kPerEvent;
    if (i % HostRing::kPerEvent == HostRing::kPerEvent - 1)
        AUG_HIP(hipEventRecord(r.done[e], ctx->stream), "staging event record");
    r.next = (i + 1) % HostRing::kSlots;
    return AUG_OK;
}

// Record an event that closes stage `stage` (or opens a timed span when stage < 0).
inline int mark(aug_ctx* ctx, int stage) {
    if (!ctx->profiling) return AUG_OK;
    hipEvent_t ev;
    AUG_HIP(hipEventCreate(&ev), "event create");
    hipError_t e = hipEventRecord(ev, ctx->stream);
    if (e != hipSuccess) {
        (void)hipEventDestroy(ev);
        return fail_hip(ctx, e, "event record");
    }
    ctx->marks.emplace_back(ev, stage);
    return AUG_OK;
}

inline int enter(aug_ctx* ctx) {
    if (!ctx) return AUG_ERR_INVALID_ARG;
    ctx->last_error.clear();
    AUG_HIP(hipSetDevice(ctx->device), "set device");
    return AUG_OK;
}

}  // namespace aug
