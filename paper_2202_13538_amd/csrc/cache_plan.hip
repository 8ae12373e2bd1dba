// One step of a paged cache's bookkeeping (surel_cache_plan).
//
// Three exclusive sums over the sequences: of the rows they add (their offsets), then, with offsets cut at n_rows, of
// the pages they need and of the pages they give back.  Everything else follows from them place by place: the j-th
// new page of a sequence is the ring's entry taken + (its sum) + j, so that neither the page table's new entries nor a
// slot has to wait for another workgroup's writes.
#include "cache.h"
#include "kernels.h"
#include "wave_sums.h"

namespace surel {
namespace {

constexpr int kMostThreads = 1024, kFewThreads = 256, kEach = 4;
constexpr int kChunk = kMostThreads * kEach;   // sequences whose sums one workgroup makes at a time

// Sums of earlier chunks of sequences, where there are several: [chunk][3] of rows, new pages, pages given back.
enum { kRows = 0, kFresh = 1, kBack = 2, kSums = 3 };

// The last i of n with from[i] <= x (from[0] <= x).
__device__ __forceinline__ int last_at_most(const int32_t* from, int n, int32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (from[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The same for all lanes of a wave at once, up to 4,096 numbers: 64 of them are looked at at a time.
__device__ __forceinline__ int wave_last_at_most(const int32_t* from, int n, int32_t x) {
    const int lane = lane_id();
    const int group = max((int)__popcll(__ballot(64 * lane < n && from[min(64 * lane, n - 1)] <= x)) - 1, 0);
    const int at = 64 * group + lane;
    return 64 * group + max((int)__popcll(__ballot(at < n && from[min(at, n - 1)] <= x)) - 1, 0);
}

template <int SEQS>
struct Lists {              // in LDS, of a chunk's sequences
    int32_t off[SEQS];      // of rows
    int32_t fresh[SEQS];    // of new pages
    int32_t back[SEQS];     // of pages given back
    int32_t length[SEQS];
    int32_t after[SEQS];
    double of_wave[16];
};

// STEP 0: a chunk's rows; 1: its pages, new and given back; 2: everything, `parts` workgroups a chunk.  With one chunk
// there is step 2 only.  What bounds it: a launch, three sums of two barriers each and a few trips to memory behind one another
// (256 sequences that add a row each 12 us), and behind these the pages and slots of 256 workgroups (4.2 million slots 24).
// Few threads for few sequences and rows: 256 sequences that add a row each 14 us with 1,024, of which most have nothing to do.
template <int STEP, int kThreads>
__global__ __launch_bounds__(kThreads) void cache_plan_kernel(CachePlan p, int64_t* sums, int chunks, int parts) {
    extern __shared__ __align__(16) char lds[];
    Lists<kEach * kThreads>& l = *reinterpret_cast<Lists<kEach * kThreads>*>(lds);
    const int tid = threadIdx.x, chunk = blockIdx.x / parts, part = blockIdx.x % parts;
    const int s0 = chunk * kChunk, n = min(p.n_seqs - s0, kChunk);   // (n may be 0: of no sequences at all)
    const uint32_t page_rows = p.page_rows.d;
    const int64_t most = (int64_t)p.width * page_rows;

    int32_t length[kEach], added[kEach];
    int64_t rows = 0;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int i = kEach * tid + e;
        length[e] = i < n ? p.length[s0 + i] : 0;
        added[e] = i < n ? p.added[s0 + i] : 0;
        if (length[e] < 0 || length[e] > most) bad = true, length[e] = added[e] = 0;
        rows += max(added[e], 0);
    }
    // (sums as 64-bit floats: 4,096 numbers below 2^31 add up to less than 2^53)
    double all;
    int64_t off = (int64_t)before_in_group((double)rows, l.of_wave, &all);
    const int64_t all_rows = (int64_t)all;
    if (STEP == 0) {
        if (tid == 0) sums[kSums * chunk + kRows] = all_rows;
        return;
    }

    int64_t before[kSums] = {0, 0, 0};   // of the chunks before this one
    if (chunks > 1) {
        for (int k = 0; k < (STEP == 1 ? 1 : (int)kSums); ++k) {
            int64_t x = 0;
            for (int c = tid; c < chunk; c += kThreads) x += sums[kSums * c + k];
            (void)before_in_group((double)x, l.of_wave, &all);
            before[k] = (int64_t)all;
        }
    }
    off += before[kRows];
    const bool cut = before[kRows] + all_rows > p.n_rows;

    int32_t first[kEach + 1], held[kEach], fresh[kEach];
    int64_t want[kEach], new_pages = 0, back_pages = 0;
    bool no_room = false;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        first[e] = (int32_t)min(off, (int64_t)p.n_rows);
        off += max(added[e], 0);
        const int32_t end = (int32_t)min(off, (int64_t)p.n_rows);
        held[e] = (int32_t)p.page_rows.of((uint32_t)length[e] + page_rows - 1);
        want[e] = min((int64_t)length[e] + (end - first[e]), most);
        no_room = no_room || want[e] < (int64_t)length[e] + (end - first[e]);
        fresh[e] = added[e] < 0 ? 0 : max((int32_t)p.page_rows.of((uint32_t)want[e] + page_rows - 1) - held[e], 0);
        new_pages += fresh[e];
        back_pages += added[e] < 0 ? held[e] : 0;
    }
    first[kEach] = (int32_t)min(off, (int64_t)p.n_rows);
    int64_t at_new = (int64_t)before_in_group((double)new_pages, l.of_wave, &all) + before[kFresh];
    const int64_t all_new = (int64_t)all;
    int64_t at_back = (int64_t)before_in_group((double)back_pages, l.of_wave, &all) + before[kBack];
    const int64_t all_back = (int64_t)all;
    if (STEP == 1) {
        if (tid == 0) sums[kSums * chunk + kFresh] = all_new, sums[kSums * chunk + kBack] = all_back;
        return;
    }

    // the ring: pages that can be taken, and places for pages given back
    int64_t taken = p.turn[0], given = p.turn[1];
    const bool bad_ring = taken < 0 || given < taken || given - taken > p.n_pages;
    const int32_t free = bad_ring ? 0 : (int32_t)(given - taken);
    const int32_t room = bad_ring ? 0 : p.n_pages - free;
    const int32_t ring_taken = bad_ring ? 0 : (int32_t)(taken % p.n_pages), ring_given = bad_ring ? 0 : (int32_t)(given % p.n_pages);
    auto ring_at = [&](int32_t from, int32_t i) {   // both below n_pages <= 2^30
        const int32_t at = from + i;
        return at >= p.n_pages ? at - p.n_pages : at;
    };

    bool no_page = false;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int i = kEach * tid + e;
        const int32_t got = (int32_t)min(max((int64_t)free - at_new, (int64_t)0), (int64_t)fresh[e]);
        const int32_t after = added[e] < 0 ? 0 : (int32_t)min(want[e], ((int64_t)held[e] + got) * page_rows);
        no_page = no_page || got < fresh[e];
        if (i < n) {
            l.off[i] = first[e];
            l.fresh[i] = (int32_t)min(at_new, (int64_t)0x7FFFFFFF);
            l.back[i] = (int32_t)min(at_back, (int64_t)0x7FFFFFFF);
            l.length[i] = length[e];
            l.after[i] = after;
            if (part == 0) p.off[s0 + i] = first[e], p.length_after[s0 + i] = after;
        }
        at_new += fresh[e];
        at_back += added[e] < 0 ? held[e] : 0;
    }
    if (part == 0) {
        raise_error(p.err, bad, kDevBadLength);
        raise_error(p.err, no_page, kDevNoPage);
        raise_error(p.err, no_room || cut, kDevCapacity);
        if (tid == 0 && bad_ring) atomicOr(p.err, kDevBadPage);
    }
    const bool last = chunk == chunks - 1;
    const int64_t end_new = before[kFresh] + all_new, end_back = before[kBack] + all_back;
    const int32_t end_rows = (int32_t)min(before[kRows] + all_rows, (int64_t)p.n_rows);
    if (part == 0 && last && tid == 0) {
        p.off[p.n_seqs] = end_rows;
        p.turn_after[0] = taken + min(end_new, (int64_t)free);
        p.turn_after[1] = given + min(end_back, (int64_t)room);
    }
    __syncthreads();

    bool bad_page = false;
    // new entries of the page table
    auto page_of_ring = [&](int32_t i) {   // the ring's i-th free page, or -1
        if (i >= free) return -1;
        const int32_t page = p.ring[ring_at(ring_taken, i)];
        if (page >= 0 && page < p.n_pages) return page;
        bad_page = true;
        return -1;
    };
    const int32_t some_new = (int32_t)min(before[kFresh], (int64_t)0x7FFFFFFF), till_new = (int32_t)min(end_new, (int64_t)0x7FFFFFFF);
    // (the three lists begin with different waves, so that small ones do not wait for each other)
    for (int64_t f = (int64_t)some_new + part * kThreads + (tid ^ kThreads / 2); f < till_new; f += parts * kThreads) {
        const int i = last_at_most(l.fresh, n, (int32_t)f);
        const int32_t at = (int32_t)p.page_rows.of((uint32_t)l.length[i] + page_rows - 1) + (int32_t)f - l.fresh[i];
        p.pages[(int64_t)(s0 + i) * p.width + at] = page_of_ring((int32_t)f);
    }
    // pages given back
    const int64_t till_back = min(end_back, (int64_t)room);
    if (part == 0 && tid == 0 && end_back > room) bad_page = true;
    for (int64_t f = min(before[kBack], (int64_t)0x7FFFFFFF) + part * kThreads + (tid ^ kThreads / 4 * 3); f < till_back; f += parts * kThreads) {
        const int i = last_at_most(l.back, n, (int32_t)f);
        const int32_t page = p.pages[(int64_t)(s0 + i) * p.width + ((int32_t)f - l.back[i])];
        if (page < 0 || page >= p.n_pages) bad_page = true;
        p.ring[ring_at(ring_given, (int32_t)f)] = page;
    }
    // slots, four rows a thread; behind the last sequence's rows there are none
    const int32_t row_begin = (int32_t)min(before[kRows], (int64_t)p.n_rows), row_end = last ? p.n_rows : end_rows;
    const bool wide = (reinterpret_cast<uintptr_t>(p.slots) & 15u) == 0;
    const int lane = tid & 63, first_lane = __builtin_amdgcn_readfirstlane(tid) & ~63;
    for (int64_t wave_row = (row_begin & ~3) + 4 * ((int64_t)part * kThreads + first_lane); wave_row < row_end; wave_row += 4 * (int64_t)parts * kThreads) {
        const int64_t r = wave_row + 4 * lane;
        // a wave's 256 rows are of neighbouring sequences: these first, then a lane's own among them
        int i = 0;
        if (wave_row < end_rows && n > 0) {
            const int lo = wave_last_at_most(l.off, n, max((int32_t)wave_row, row_begin));
            const int hi = wave_last_at_most(l.off, n, (int32_t)min(wave_row + 255, (int64_t)end_rows - 1));
            i = lo + last_at_most(l.off + lo, hi - lo + 1, (int32_t)min(max(r, (int64_t)row_begin), (int64_t)end_rows - 1));
        }
        int32_t slot[4], page = -1, page_seq = -1, page_turn = -1;   // (rows of one page look it up once)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int32_t row = (int32_t)r + e;
            slot[e] = -1;
            if (row < row_begin || row >= end_rows) continue;
            while (i + 1 < n && l.off[i + 1] <= row) ++i;
            const int32_t length = l.length[i], at = length + (row - l.off[i]);
            if (at >= l.after[i]) continue;
            const int32_t turn = (int32_t)p.page_rows.of((uint32_t)at), have = (int32_t)p.page_rows.of((uint32_t)length + page_rows - 1);
            if (i == page_seq && turn == page_turn) {
            } else if (turn < have) {
                page = p.pages[(int64_t)(s0 + i) * p.width + turn];
                if (page < 0 || page >= p.n_pages) bad_page = true, page = -1;
            } else {
                page = page_of_ring(l.fresh[i] + turn - have);
            }
            page_seq = i, page_turn = turn;
            if (page >= 0) slot[e] = (int32_t)((uint32_t)page * page_rows + ((uint32_t)at - (uint32_t)turn * page_rows));
        }
        if (wide && r >= row_begin && r + 4 <= row_end) {
            *reinterpret_cast<int4*>(p.slots + r) = int4{slot[0], slot[1], slot[2], slot[3]};
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (r + e >= row_begin && r + e < row_end) p.slots[r + e] = slot[e];
        }
    }
    raise_error(p.err, bad_page, kDevBadPage);
}

int chunks_of(int64_t n_seqs) { return n_seqs > kChunk ? (int)((n_seqs + kChunk - 1) / kChunk) : 1; }

template <int STEP, int kThreads>
hipError_t launch_step(hipStream_t stream, const CachePlan& p, int64_t* sums, int chunks, int parts) {
    auto kernel = cache_plan_kernel<STEP, kThreads>;
    constexpr size_t bytes = sizeof(Lists<kEach * kThreads>);
    const hipError_t rc = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)bytes);
    if (rc != hipSuccess) return rc;
    hipLaunchKernelGGL(kernel, dim3(chunks * parts), dim3(kThreads), bytes, stream, p, sums, chunks, parts);
    return hipGetLastError();
}

}  // namespace

size_t cache_plan_scratch_bytes(int64_t n_seqs) {
    const int chunks = chunks_of(n_seqs);
    return chunks > 1 ? (size_t)chunks * kSums * sizeof(int64_t) : 0;
}

hipError_t launch_cache_plan(hipStream_t stream, int n_cu, CachePlan p, void* scratch) {
    int64_t* const sums = static_cast<int64_t*>(scratch);
    const int chunks = chunks_of(p.n_seqs);
    // every workgroup makes its chunk's sums first, so it gets two turns of slots to write beside them at least; one fits a compute
    // unit (4.2 million slots by 257 workgroups 29 us)
    const int64_t turns = ((int64_t)p.n_rows / chunks + 8 * kMostThreads - 1) / (8 * kMostThreads);
    const int parts = (int)max((int64_t)1, min(turns, (int64_t)(n_cu / chunks)));
    if (p.n_seqs <= kEach * kFewThreads && parts == 1) return launch_step<2, kFewThreads>(stream, p, sums, 1, 1);
    hipError_t rc = hipSuccess;
    if (chunks > 1) rc = launch_step<0, kMostThreads>(stream, p, sums, chunks, 1);
    if (chunks > 1 && rc == hipSuccess) rc = launch_step<1, kMostThreads>(stream, p, sums, chunks, 1);
    return rc == hipSuccess ? launch_step<2, kMostThreads>(stream, p, sums, chunks, parts) : rc;
}

}  // namespace surel
