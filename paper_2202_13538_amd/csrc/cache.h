// What the kernels of a paged cache share: how its pages lie, and how rows are found in them.
#pragma once

#include "device_util.h"

namespace surel {

// floor(x / d) for 0 <= x < 2^31 by a multiplication: with 2^l the least power of two >= d and m = ceil(2^(31+l) / d),
// m d exceeds 2^(31+l) by less than 2^l, so x m / 2^(31+l) exceeds x / d by less than 1 / d.
struct Divisor {
    uint32_t m = 0, shift = 0, d = 1;
    Divisor() = default;
    explicit Divisor(uint32_t by) : d(by) {
        uint32_t l = 0;
        while ((uint64_t)1 << l < by) ++l;
        if (l == 0) return;
        m = (uint32_t)((((uint64_t)1 << (31 + l)) + by - 1) / by);
        shift = l - 1;
    }
    __device__ __forceinline__ uint32_t of(uint32_t x) const { return d == 1 ? x : __umulhi(x, m) >> shift; }
};

// The newest step of a cache's bookkeeping, see surel_cache_plan.
struct CachePlan {
    const int32_t *length = nullptr, *added = nullptr;
    int32_t *pages = nullptr, *ring = nullptr;
    const int64_t* turn = nullptr;
    int64_t* off = nullptr;
    int32_t *slots = nullptr, *length_after = nullptr;
    int64_t* turn_after = nullptr;
    int32_t n_seqs = 0, n_pages = 0, width = 0, n_rows = 0;   // width: pages of a sequence, at most
    Divisor page_rows;
    uint32_t* err = nullptr;
};

struct CacheStore {
    char *k_pages = nullptr, *v_pages = nullptr;
    int64_t page = 0;                     // bytes, as all strides here
    uint32_t row = 0, head = 0;
    const char *k = nullptr, *v = nullptr;
    uint32_t k_row = 0, k_head = 0, v_row = 0, v_head = 0;
    const int32_t* slots = nullptr;
    int32_t n_rows = 0, n_slots = 0, kv_heads = 0, dim = 0;
    Divisor page_rows;
    uint32_t* err = nullptr;
};

struct CacheAttention {
    const char *k_pages = nullptr, *v_pages = nullptr, *q = nullptr;
    int64_t page = 0;                     // bytes, as all strides here
    uint32_t row = 0, head = 0, q_row = 0, q_head = 0;
    const int32_t *pages = nullptr, *length = nullptr;
    int32_t n_seqs = 0, n_pages = 0, width = 0, heads = 0, kv_heads = 0, dim = 0;
    float scale = 0.f;
    const void* bias = nullptr;           // [n_buckets][heads] or null
    const int32_t* bucket = nullptr;
    int32_t n_buckets = 0, reach = 0;
    Divisor page_rows;
    void* out = nullptr;
    float* lse = nullptr;
    uint32_t* err = nullptr;
};

}  // namespace surel
