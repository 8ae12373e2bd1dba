// Keys and values of new rows into a paged cache (surel_cache_store).
#include "cache.h"
#include "kernels.h"
#include "matrix_tile.h"

namespace surel {
namespace {

constexpr int kThreads = 256;

// A thread moves 16 bytes of a row's keys and of its values at a time; a workgroup goes over `rows` rows, whose chunks it
// numbers through, so that neighbouring threads move neighbouring chunks.  What bounds it: memory: 200,003 rows of 4
// heads of 80 elements 108 us, 4.7 TB/s (a large copy has 5.1); 256 rows of 8 of 128 3 us, of a call's 10.
__global__ __launch_bounds__(kThreads) void cache_store_kernel(CacheStore a, int rows, Divisor row_chunks, Divisor head_chunks) {
    const int64_t row0 = (int64_t)block_number() * rows;
    if (row0 >= a.n_rows) return;
    const uint32_t n = (uint32_t)min((int64_t)rows, a.n_rows - row0) * row_chunks.d;
    bool bad = false;
    for (uint32_t id = threadIdx.x; id < n; id += kThreads) {
        const uint32_t r = row_chunks.of(id), in_row = id - r * row_chunks.d;
        const uint32_t head = head_chunks.of(in_row), c = in_row - head * head_chunks.d;
        const int64_t row = row0 + r;
        const int32_t slot = a.slots[row];
        if (slot < 0 || slot >= a.n_slots) {
            bad = bad || slot != -1;
            continue;
        }
        const uint32_t page = a.page_rows.of((uint32_t)slot);
        const int64_t to = page * a.page + (int64_t)((uint32_t)slot - page * a.page_rows.d) * a.row + (int64_t)head * a.head + 16 * c;
        const u32x4 k = *reinterpret_cast<const u32x4*>(a.k + row * a.k_row + (int64_t)head * a.k_head + 16 * c);
        const u32x4 v = *reinterpret_cast<const u32x4*>(a.v + row * a.v_row + (int64_t)head * a.v_head + 16 * c);
        *reinterpret_cast<u32x4*>(a.k_pages + to) = k;
        *reinterpret_cast<u32x4*>(a.v_pages + to) = v;
    }
    raise_error(a.err, bad, kDevBadPage);
}

}  // namespace

hipError_t launch_cache_store(hipStream_t stream, int n_cu, const CacheStore& a) {
    const uint32_t row_chunks = (uint32_t)a.kv_heads * (a.dim / 8);
    // two turns of a workgroup's threads
    const int rows = (int)max(1u, 2 * kThreads / row_chunks);
    hipLaunchKernelGGL(cache_store_kernel, grid_of(((int64_t)a.n_rows + rows - 1) / rows), dim3(kThreads), 0, stream, a, rows,
                       Divisor(row_chunks), Divisor(a.dim / 8));
    return hipGetLastError();
}

}  // namespace surel
