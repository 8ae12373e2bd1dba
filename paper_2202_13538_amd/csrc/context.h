// The context of libsurel and what every entry point does with it (host side, internal).
#pragma once

#include "../../include/surel.h"

#include <hip/hip_runtime.h>

#include <vector>

struct surel_ctx {
    int device = 0;
    hipStream_t stream = nullptr;
    int max_lds_bytes = 0;
    int n_cu = 0;                 // compute units of the device
    uint32_t spin_limit = 1u << 22;  // bound of every wait inside a kernel
    uint32_t* d_err = nullptr;    // sticky device error word
    hipEvent_t done = nullptr;    // completed by the one launch of a call that reports its total
    void* d_small = nullptr;      // words of the launches that lay small outputs out themselves
    // pinned host memory for small read-backs: a row total; 1 if a bounded wait ran out; a number of
    // distinct vectors or the error word
    int64_t* h_pinned = nullptr;
    void* d_ws = nullptr;         // grow-only workspace: row counts + scan partials
    size_t ws_bytes = 0;
    void* d_rec = nullptr;        // grow-only workspace: per-edge neighbour records of the walk
    size_t rec_bytes = 0;
    void* d_lb = nullptr;         // grow-only workspace: look-back words of the fused kernel
    size_t lb_bytes = 0;
    void* d_prune = nullptr;      // grow-only workspace: hash slots, sort list, counters of prune
    size_t prune_bytes = 0;
    int prune_turn = 0;           // which of two sets of counters the next of these calls takes
    size_t prune_clean = 0;       // bytes of the hash slots in it that are known to be empty
    void* d_batch = nullptr;      // grow-only workspace: sort arrays of the incidence lists, hash
    size_t batch_bytes = 0;       // tables of the mini-batch search
    uint32_t* d_turns = nullptr;  // a word of zero between launches whose last workgroup joins the others' parts
    void* d_model = nullptr;      // grow-only workspace: parts of attention and loss that are joined later
    size_t model_bytes = 0;
    // workspace of plans, attention over a cache and samples.  It grows to twice its size at least, and what it was before
    // stays until the context ends: calls that were captured into a graph go on using it.
    void* d_kept = nullptr;
    size_t kept_bytes = 0;
    void* kept_before[64] = {};
    int n_kept_before = 0;
    void* d_scratch = nullptr;    // this device's copy of the file-scope `scratch` array below
    bool no_spans = false;        // set while a call that must not allocate runs (no new events)
    // optional per-kernel timing (surel_profile_*)
    struct Span {
        int kernel;
        hipEvent_t start, stop;
    };
    bool profiling = false;
    std::vector<Span> spans;          // recorded, not yet read
    std::vector<hipEvent_t> free_events;
    double prof_ms[SUREL_K_COUNT] = {};
    int64_t prof_launches[SUREL_K_COUNT] = {};
};

namespace {

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int device) {
        if (hipGetDevice(&prev) != hipSuccess) return;
        ok = (prev == device) || (hipSetDevice(device) == hipSuccess);
        if (prev == device) prev = -1;
    }
    ~DeviceGuard() {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// The uint16 count arrays are moved as 32-bit words wherever possible.
inline bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

// Brackets the launches made during its lifetime with two events on the context's stream
// when profiling is on; does nothing otherwise.
class KernelSpan {
  public:
    KernelSpan(surel_ctx* ctx, int kernel) : ctx_(ctx) {
        if (!ctx->profiling || ctx->no_spans) return;
        span_.kernel = kernel;
        span_.start = take();
        span_.stop = take();
        if (!span_.start || !span_.stop) {
            give_back();
            return;
        }
        active_ = hipEventRecord(span_.start, ctx->stream) == hipSuccess;
        if (!active_) give_back();
    }
    ~KernelSpan() {
        if (!active_) return;
        if (hipEventRecord(span_.stop, ctx_->stream) == hipSuccess) {
            ctx_->spans.push_back(span_);
        } else {
            give_back();
        }
    }
    KernelSpan(const KernelSpan&) = delete;
    KernelSpan& operator=(const KernelSpan&) = delete;

  private:
    hipEvent_t take() {
        if (!ctx_->free_events.empty()) {
            hipEvent_t e = ctx_->free_events.back();
            ctx_->free_events.pop_back();
            return e;
        }
        hipEvent_t e = nullptr;
        if (hipEventCreate(&e) != hipSuccess) return nullptr;
        return e;
    }
    void give_back() {
        if (span_.start) ctx_->free_events.push_back(span_.start);
        if (span_.stop) ctx_->free_events.push_back(span_.stop);
        span_.start = span_.stop = nullptr;
    }
    surel_ctx* ctx_;
    surel_ctx::Span span_{0, nullptr, nullptr};
    bool active_ = false;
};

// Wait for the stream and fold every recorded span into the per-kernel totals.
inline int drain_spans(surel_ctx* ctx) {
    if (hipStreamSynchronize(ctx->stream) != hipSuccess) return SUREL_E_HIP;
    for (const surel_ctx::Span& sp : ctx->spans) {
        float ms = 0.f;
        if (hipEventElapsedTime(&ms, sp.start, sp.stop) == hipSuccess) {
            ctx->prof_ms[sp.kernel] += (double)ms;
            ctx->prof_launches[sp.kernel] += 1;
        }
        ctx->free_events.push_back(sp.start);
        ctx->free_events.push_back(sp.stop);
    }
    ctx->spans.clear();
    return SUREL_OK;
}

// Grows one of the context's workspaces to `need` bytes (contents are not kept).  The old
// buffer may still be in use by earlier work on the stream, so the stream is drained first.
inline int grow_buffer(surel_ctx* ctx, void** buf, size_t* have, size_t need) {
    if (need <= *have) return SUREL_OK;
    if (hipStreamSynchronize(ctx->stream) != hipSuccess) return SUREL_E_HIP;
    if (*buf) (void)hipFree(*buf);
    *buf = nullptr;
    *have = 0;
    if (hipMalloc(buf, need) != hipSuccess) {
        (void)hipGetLastError();
        return SUREL_E_HIP;
    }
    *have = need;
    return SUREL_OK;
}

// The workspace that captured calls may go on using, with `need` bytes at least (contents are not kept).
inline int grow_kept(surel_ctx* ctx, size_t need) {
    if (need <= ctx->kept_bytes) return SUREL_OK;
    const size_t size = need > 2 * ctx->kept_bytes ? need : 2 * ctx->kept_bytes;
    void* now = nullptr;
    if (ctx->n_kept_before == 64 || hipMalloc(&now, size) != hipSuccess) {
        (void)hipGetLastError();
        return SUREL_E_HIP;
    }
    if (ctx->d_kept) ctx->kept_before[ctx->n_kept_before++] = ctx->d_kept;
    ctx->d_kept = now;
    ctx->kept_bytes = size;
    return SUREL_OK;
}

}  // namespace
