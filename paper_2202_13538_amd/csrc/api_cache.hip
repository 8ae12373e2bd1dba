// The C ABI of libsurel, continued: sequences that run on, over keys and values kept in pages.  See
// include/surel.h for the contract of every entry point.
#include "../../include/surel.h"

#include <hip/hip_runtime.h>

#include <math.h>

#include "cache.h"
#include "context.h"
#include "kernels.h"
#include "sample.h"

namespace {

constexpr int64_t kMostPage = 1ll << 40;                // elements between pages
constexpr double kMostTiles = 281474976710656.0;        // 2^48: tiles of 32 keys of all sequences and heads

bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// A stride between `count` rows or heads, and what the kernels get for it: one that leads nowhere may be any.
bool bad_stride(int64_t elements, int64_t count, int64_t most = SUREL_MAX_STRIDE) {
    return elements < 0 || (count > 1 && (elements > most || elements % 8 != 0));
}
uint32_t stride_bytes(int64_t elements, int64_t count) { return count > 1 ? (uint32_t)(2 * elements) : 0; }

// Whether `pages` pages of `rows` rows are more than may be, or none.
bool bad_pages(int64_t pages, int64_t rows) {
    return pages < 1 || rows < 1 || pages > SUREL_MAX_ROWS || rows > SUREL_MAX_ROWS || pages * rows > SUREL_MAX_ROWS;
}

int cache_args(const surel_cache* c) {
    if (!c) return SUREL_E_NULL;
    if (c->type != SUREL_BF16 && c->type != SUREL_FP16) return SUREL_E_RANGE;
    if (bad_pages(c->n_pages, c->page_rows)) return SUREL_E_RANGE;
    if (c->dim < 8 || c->dim > SUREL_MAX_HEAD_DIM || c->dim % 8 != 0) return SUREL_E_RANGE;
    if (c->kv_heads < 1 || c->kv_heads > 65535) return SUREL_E_RANGE;
    if (bad_stride(c->page, c->n_pages, kMostPage) || bad_stride(c->row, c->page_rows) || bad_stride(c->head, c->kv_heads))
        return SUREL_E_RANGE;
    if (!c->d_k || !c->d_v) return SUREL_E_NULL;
    if (misaligned16(c->d_k) || misaligned16(c->d_v)) return SUREL_E_RANGE;
    return SUREL_OK;
}

}  // namespace

extern "C" {

int surel_cache_plan(surel_ctx* ctx, const int32_t* d_length, const int32_t* d_added, int64_t n_seqs, int64_t n_pages,
                     int32_t page_rows, int32_t max_pages, int64_t n_rows, int32_t* d_pages, int32_t* d_ring,
                     const int64_t* d_turn, int64_t* d_off, int32_t* d_slots, int32_t* d_length_after,
                     int64_t* d_turn_after) {
    if (n_seqs < 0 || n_seqs > SUREL_MAX_SEQS || n_rows < 0 || n_rows > SUREL_MAX_ROWS) return SUREL_E_RANGE;
    if (bad_pages(n_pages, page_rows) || bad_pages(max_pages, page_rows)) return SUREL_E_RANGE;
    if (n_seqs > 0 && (!d_length || !d_added || !d_pages || !d_length_after)) return SUREL_E_NULL;
    if (!d_ring || !d_turn || !d_off || !d_turn_after || (n_rows > 0 && !d_slots)) return SUREL_E_NULL;
    // every workgroup reads what one of them writes: not the same arrays
    if ((n_seqs > 0 && (d_length_after == d_length || d_length_after == d_added)) || d_turn_after == d_turn) return SUREL_E_RANGE;
    if (!ctx) return SUREL_E_CTX;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SUREL_E_HIP;
    if (int rc = grow_kept(ctx, surel::cache_plan_scratch_bytes(n_seqs))) return rc;
    surel::CachePlan p;
    p.length = d_length, p.added = d_added, p.pages = d_pages, p.ring = d_ring, p.turn = d_turn;
    p.off = d_off, p.slots = d_slots, p.length_after = d_length_after, p.turn_after = d_turn_after;
    p.n_seqs = (int32_t)n_seqs, p.n_pages = (int32_t)n_pages, p.width = max_pages, p.n_rows = (int32_t)n_rows;
    p.page_rows = surel::Divisor((uint32_t)page_rows);
    p.err = ctx->d_err;
    KernelSpan span(ctx, SUREL_K_CACHE_PLAN);
    return surel::launch_cache_plan(ctx->stream, ctx->n_cu, p, ctx->d_kept) == hipSuccess ? SUREL_OK : SUREL_E_HIP;
}

int surel_cache_store(surel_ctx* ctx, const surel_cache* cache, const void* d_k, const void* d_v, int64_t k_row,
                      int64_t k_head, int64_t v_row, int64_t v_head, const int32_t* d_slots, int64_t n_rows) {
    if (int rc = cache_args(cache)) return rc;
    if (n_rows < 0 || n_rows > SUREL_MAX_ROWS) return SUREL_E_RANGE;
    if (bad_stride(k_row, n_rows) || bad_stride(k_head, cache->kv_heads) || bad_stride(v_row, n_rows) ||
        bad_stride(v_head, cache->kv_heads))
        return SUREL_E_RANGE;
    if (n_rows > 0 && (!d_k || !d_v || !d_slots)) return SUREL_E_NULL;
    if (misaligned16(d_k) || misaligned16(d_v)) return SUREL_E_RANGE;
    if (!ctx) return SUREL_E_CTX;
    if (n_rows == 0) return SUREL_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SUREL_E_HIP;
    surel::CacheStore a;
    a.k_pages = static_cast<char*>(cache->d_k), a.v_pages = static_cast<char*>(cache->d_v);
    a.page = cache->n_pages > 1 ? 2 * cache->page : 0;
    a.row = stride_bytes(cache->row, cache->page_rows), a.head = stride_bytes(cache->head, cache->kv_heads);
    a.k = static_cast<const char*>(d_k), a.v = static_cast<const char*>(d_v);
    a.k_row = stride_bytes(k_row, n_rows), a.k_head = stride_bytes(k_head, cache->kv_heads);
    a.v_row = stride_bytes(v_row, n_rows), a.v_head = stride_bytes(v_head, cache->kv_heads);
    a.slots = d_slots;
    a.n_rows = (int32_t)n_rows, a.n_slots = (int32_t)(cache->n_pages * cache->page_rows);
    a.kv_heads = cache->kv_heads, a.dim = cache->dim;
    a.page_rows = surel::Divisor((uint32_t)cache->page_rows);
    a.err = ctx->d_err;
    KernelSpan span(ctx, SUREL_K_CACHE_STORE);
    return surel::launch_cache_store(ctx->stream, ctx->n_cu, a) == hipSuccess ? SUREL_OK : SUREL_E_HIP;
}

int surel_cache_attention(surel_ctx* ctx, const surel_cache* cache, const surel_cache_attention_args* x, void* d_out,
                          float* d_lse) {
    if (int rc = cache_args(cache)) return rc;
    if (!x) return SUREL_E_NULL;
    if (x->n_seqs < 0 || x->n_seqs > SUREL_MAX_SEQS || bad_pages(x->max_pages, cache->page_rows)) return SUREL_E_RANGE;
    if (x->heads < 1 || x->heads > 65535 || x->heads % cache->kv_heads != 0) return SUREL_E_RANGE;
    if (bad_stride(x->q_row, x->n_seqs) || bad_stride(x->q_head, x->heads)) return SUREL_E_RANGE;
    if (!(x->scale > 0.f) || !isfinite(x->scale)) return SUREL_E_RANGE;
    if ((x->d_bias == nullptr) != (x->d_bucket == nullptr)) return SUREL_E_NULL;
    if (x->d_bias && (x->n_buckets < 1 || x->n_buckets > 2 * SUREL_MAX_REACH + 1 || x->reach < 0 ||
                      x->reach > SUREL_MAX_REACH))
        return SUREL_E_RANGE;
    if ((double)x->n_seqs * x->max_pages * cache->page_rows / 32.0 * x->heads > kMostTiles) return SUREL_E_RANGE;
    if (x->n_seqs > 0 && (!x->d_q || !x->d_pages || !x->d_length || !d_out || !d_lse)) return SUREL_E_NULL;
    if (misaligned16(x->d_q) || misaligned16(d_out)) return SUREL_E_RANGE;
    if (!ctx) return SUREL_E_CTX;
    if (x->n_seqs == 0) return SUREL_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SUREL_E_HIP;
    surel::CacheAttention a;
    a.k_pages = static_cast<const char*>(cache->d_k), a.v_pages = static_cast<const char*>(cache->d_v);
    a.page = cache->n_pages > 1 ? 2 * cache->page : 0;
    a.row = stride_bytes(cache->row, cache->page_rows), a.head = stride_bytes(cache->head, cache->kv_heads);
    a.q = static_cast<const char*>(x->d_q);
    a.q_row = stride_bytes(x->q_row, x->n_seqs), a.q_head = stride_bytes(x->q_head, x->heads);
    a.pages = x->d_pages, a.length = x->d_length;
    a.n_seqs = (int32_t)x->n_seqs, a.n_pages = (int32_t)cache->n_pages, a.width = x->max_pages;
    a.heads = x->heads, a.kv_heads = cache->kv_heads, a.dim = cache->dim;
    a.scale = x->scale;
    a.bias = x->d_bias, a.bucket = x->d_bucket;
    a.n_buckets = x->d_bias ? x->n_buckets : 0;
    a.reach = x->d_bias ? x->reach : 0;
    a.page_rows = surel::Divisor((uint32_t)cache->page_rows);
    a.out = d_out, a.lse = d_lse;
    a.err = ctx->d_err;
    if (int rc = grow_kept(ctx, surel::cache_attention_scratch_bytes(ctx->n_cu, a))) return rc;
    KernelSpan span(ctx, SUREL_K_CACHE_ATTENTION);
    return surel::launch_cache_attention(ctx->stream, ctx->n_cu, a, cache->type == SUREL_FP16, ctx->d_kept) == hipSuccess
               ? SUREL_OK : SUREL_E_HIP;
}

int surel_sample_classes(surel_ctx* ctx, int32_t type, const void* d_logits, int64_t row, int64_t n_rows,
                         int32_t n_classes, const float* d_u, const float* d_temperature, const int32_t* d_top_k,
                         const float* d_top_p, const float* d_min_p, int32_t* d_class, float* d_logp) {
    if (type != SUREL_BF16 && type != SUREL_FP16 && type != SUREL_FP32) return SUREL_E_RANGE;
    if (n_rows < 0 || n_rows > SUREL_MAX_ROWS || n_classes < 1 || n_classes > SUREL_MAX_NODES) return SUREL_E_RANGE;
    if (row < 0 || (n_rows > 1 && row > kMostPage)) return SUREL_E_RANGE;
    if (n_rows > 0 && (!d_logits || !d_u || !d_class || !d_logp)) return SUREL_E_NULL;
    const int64_t size = type == SUREL_FP32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(d_logits) % (uintptr_t)size != 0) return SUREL_E_RANGE;
    if (!ctx) return SUREL_E_CTX;
    if (n_rows == 0) return SUREL_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SUREL_E_HIP;
    surel::SampleArgs a;
    a.logits = static_cast<const char*>(d_logits);
    a.row = n_rows > 1 ? row * size : 0;
    a.n_rows = (int32_t)n_rows, a.n_classes = n_classes;
    a.u = d_u, a.temperature = d_temperature, a.top_k = d_top_k, a.top_p = d_top_p, a.min_p = d_min_p;
    a.chosen = d_class, a.logp = d_logp;
    a.err = ctx->d_err;
    if (int rc = grow_kept(ctx, surel::sample_scratch_bytes(ctx->n_cu, a, type))) return rc;
    KernelSpan span(ctx, SUREL_K_SAMPLE);
    return surel::launch_sample(ctx->stream, ctx->n_cu, a, type, ctx->d_kept) == hipSuccess ? SUREL_OK : SUREL_E_HIP;
}

}  // extern "C"
