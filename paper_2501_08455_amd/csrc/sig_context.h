// The context behind the C ABI and its device scratch, shared by the translation units that hold entry points.
#ifndef SIG_CONTEXT_H
#define SIG_CONTEXT_H

#include <atomic>
#include <mutex>
#include <new>

#include "sig_internal.h"

// a mapping measured by sig_autotune for one shape
struct TunedPlan {
    int64_t B, L;
    int d, depth, stream_flag;
    sig_plan_t plan;
};

// scratch that a captured graph still uses
struct KeptScratch {
    float *scratch;
    KeptScratch *next;
};

struct sig_ctx {
    int device;
    int num_cu;
    float *fixed_scratch;  // this device's copy of the array in sig_api.hip (sig_compute_noalloc)
    mutable std::mutex lock;       // over everything below
    float *scratch;        // partial signatures of time segments, [B][segments][D], and what other calls keep between launches
    size_t scratch_bytes;
    bool scratch_captured;         // a graph holds its address: it stays until the context goes
    KeptScratch *kept;             // ... outgrown buffers of this kind
    hipStream_t scratch_stream;    // of the last call that used the scratch
    bool scratch_used;             // ... since it was allocated
    bool scratch_shared;           // several streams use it: scratch_event marks the end of the last call (see Scratch)
    int scratch_calls;             // calls in a row on scratch_stream since it began to be shared
    hipEvent_t scratch_event;
    TunedPlan tuned[64];   // filled by sig_autotune, consulted by sig_compute and sig_plan (oldest overwritten)
    std::atomic<int> tuned_count;   // (calls on a context without tuned plans do not lock for them)
    int tuned_next;
};

namespace sig {

// The context's scratch for the launches of one call.  From get() until it goes out of scope, behind the call's last launch,
// no other host thread's call can take the scratch, and a call on another stream than the last one's is ordered behind it
// on the device.  An event behind every call costs 2.6 us (128 paths of 2,000 points, (5,4): 19.8 -> 22.4 us), and a
// stream of the past may be destroyed by now, so that its handle is only compared.  Hence: calls that stay on one stream leave
// no event; the first one on another stream waits for the device, and from there on every call leaves one, until
// kAloneCalls in a row have come on the same stream.
class Scratch {
public:
    Scratch() = default;
    Scratch(const Scratch &) = delete;
    Scratch &operator=(const Scratch &) = delete;
    ~Scratch()
    {
        if (!mark_) return;
        if (hipEventRecord(mark_->scratch_event, mark_->scratch_stream) == hipSuccess) return;
        (void)hipGetLastError();
        (void)hipDeviceSynchronize();
        mark_->scratch_used = false;   // nothing to wait for
    }

    int get(sig_ctx *ctx, size_t bytes, hipStream_t st, float **p)
    {
        hold_ = std::unique_lock<std::mutex>(ctx->lock);
        hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
        int rc = hipStreamIsCapturing(st, &capture) == hipSuccess ? grow(ctx, bytes) : SIG_ERR_HIP;
        // Launches that are being captured run when their graph does, and a capture takes no event from outside it: the
        // order of a graph's replays and other calls is the caller's (sig.h).
        if (rc == SIG_OK) {
            if (capture != hipStreamCaptureStatusNone) ctx->scratch_captured = true;
            else rc = order(ctx, st);
        }
        if (rc == SIG_ERR_HIP) (void)hipGetLastError();
        *p = ctx->scratch;
        if (rc != SIG_OK) hold_.unlock();   // (the call may ask again, for less)
        return rc;
    }

    // whether get() can give `bytes` here: a buffer cannot grow while the stream is being captured
    static bool within_reach(const sig_ctx *ctx, size_t bytes, hipStream_t st)
    {
        std::lock_guard<std::mutex> hold(ctx->lock);
        return bytes <= ctx->scratch_bytes || !captured(st);
    }

    static bool captured(hipStream_t st)
    {
        hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
        return hipStreamIsCapturing(st, &capture) != hipSuccess || capture != hipStreamCaptureStatusNone;
    }

private:
    static constexpr int kAloneCalls = 64;

    static int grow(sig_ctx *ctx, size_t bytes)
    {
        if (bytes <= ctx->scratch_bytes) return SIG_OK;
        if (ctx->scratch && ctx->scratch_captured) {
            KeptScratch *k = new (std::nothrow) KeptScratch{ctx->scratch, ctx->kept};
            if (!k) return SIG_ERR_ALLOC;
            ctx->kept = k;
        } else if (ctx->scratch) {
            // earlier launches may still read the old buffer
            if (hipDeviceSynchronize() != hipSuccess) return SIG_ERR_HIP;
            (void)hipFree(ctx->scratch);
        }
        ctx->scratch = nullptr;
        ctx->scratch_bytes = 0;
        ctx->scratch_captured = false;
        void *p = nullptr;
        if (hipMalloc(&p, bytes) != hipSuccess) {
            (void)hipGetLastError();
            return SIG_ERR_ALLOC;
        }
        ctx->scratch = static_cast<float *>(p);
        ctx->scratch_bytes = bytes;
        ctx->scratch_used = false;
        return SIG_OK;
    }

    int order(sig_ctx *ctx, hipStream_t st)
    {
        // (hipStreamPerThread is another stream in every thread)
        const bool same = ctx->scratch_used && ctx->scratch_stream == st && st != hipStreamPerThread;
        if (same && !ctx->scratch_shared) return SIG_OK;
        if (same) {
            if (++ctx->scratch_calls >= kAloneCalls) ctx->scratch_shared = false;
        } else if (ctx->scratch_used) {
            if (!ctx->scratch_event && hipEventCreateWithFlags(&ctx->scratch_event, hipEventDisableTiming) != hipSuccess)
                return SIG_ERR_HIP;
            const hipError_t e = ctx->scratch_shared ? hipStreamWaitEvent(st, ctx->scratch_event, 0) : hipDeviceSynchronize();
            if (e != hipSuccess) return SIG_ERR_HIP;
            ctx->scratch_shared = true;
            ctx->scratch_calls = 0;
        }
        ctx->scratch_stream = st;
        ctx->scratch_used = true;
        if (ctx->scratch_shared) mark_ = ctx;
        return SIG_OK;
    }

    std::unique_lock<std::mutex> hold_;
    sig_ctx *mark_ = nullptr;
};

}  // namespace sig
#endif
