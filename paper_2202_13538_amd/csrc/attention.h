// What the attention kernels share: how a call's tensors lie, and which rows meet.
#pragma once

#include "matrix_tile.h"

namespace surel {

struct AttentionArgs {
    const char *q = nullptr, *k = nullptr, *v = nullptr;
    uint32_t q_row = 0, q_head = 0, k_row = 0, k_head = 0, v_row = 0, v_head = 0;  // bytes
    const int64_t *q_off = nullptr, *k_off = nullptr;
    int32_t n_seqs = 0, n_q = 0, n_k = 0;
    int32_t heads = 0, kv_heads = 0, dim = 0;
    int32_t causal = 0;
    float scale = 0.f;            // of q . k
    const void* bias = nullptr;   // [n_buckets][heads] or null
    const int32_t* bucket = nullptr;
    int32_t n_buckets = 0, reach = 0;
    uint32_t* err = nullptr;
};

// The last s with off[s] <= t, of n >= 1 parts.  Looks where equally long ones have it, then around that place in steps
// that double, then halves what is left: one turn of memory where they are equally long.
__device__ __forceinline__ int segment_of(const int64_t* __restrict__ off, int n, int64_t total, int64_t t) {
    int lo = total > 0 ? (int)((double)t * (double)n / (double)total) : 0;
    lo = min(max(lo, 0), n - 1);
    const int64_t here = off[lo], next = off[lo + 1];
    if (here <= t && t < next) return lo;
    int hi, step = 1;
    if (here <= t) {
        hi = lo + 1;
        while (hi < n && off[hi] <= t) {
            lo = hi;
            hi = min(hi + step, n);
            step = min(2 * step, 1 << 29);
        }
        hi = min(hi, n);
    } else {
        hi = lo;
        lo = max(hi - 1, 0);
        while (lo > 0 && off[lo] > t) {
            hi = lo;
            lo = max(lo - step, 0);
            step = min(2 * step, 1 << 29);
        }
    }
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (off[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A sequence's query rows and keys.  Offsets that do not lie in order inside the tensors make it
// empty and raise kDevBadOffsets.
struct Sequence {
    int q0, q1, k0, k1;
};
__device__ __forceinline__ Sequence sequence_at(const AttentionArgs& a, int s) {
    const int64_t q0 = a.q_off[s], q1 = a.q_off[s + 1];
    const bool alike = a.k_off == a.q_off;
    const int64_t k0 = alike ? q0 : a.k_off[s], k1 = alike ? q1 : a.k_off[s + 1];
    if (q0 < 0 || q1 < q0 || q1 > a.n_q || k0 < 0 || k1 < k0 || k1 > a.n_k) {
        atomicOr(a.err, kDevBadOffsets);
        return Sequence{0, 0, 0, 0};
    }
    return Sequence{(int)q0, (int)q1, (int)k0, (int)k1};
}

// Where the last row or key is in no sequence, or the first; one thread of a launch looks.
__device__ __forceinline__ void check_ends(const AttentionArgs& a) {
    if (a.q_off[0] != 0 || a.q_off[a.n_seqs] != a.n_q || a.k_off[0] != 0 || a.k_off[a.n_seqs] != a.n_k)
        atomicOr(a.err, kDevBadOffsets);
}

// Rows of packed sequences in tiles of `rows`: tile by tile through everything (`across`), or each
// sequence in tiles of its own.  Sequence s then has the tiles from off[s] / rows + s on: as many numbers as it
// may need, and at most one too many, without a sum over the sequences before it.
struct TileOfRows {
    int first, last;  // rows
    int seq;          // or -1: of several
};
__device__ __forceinline__ TileOfRows tile_of_rows(const int64_t* __restrict__ off, int n, int total, int rows,
                                                   bool across, int tile) {
    if (across) return TileOfRows{min(tile * rows, total), (int)min((int64_t)(tile + 1) * rows, (int64_t)total), -1};
    // the last s with off[s] / rows + s <= tile: 64 lanes look at as many places at once, so that 4,096
    // sequences take two turns of memory
    const int lane = lane_id();
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64;
        const int64_t at = lo + (int64_t)lane * step;
        const bool below = at < hi && off[at] / rows + at <= tile;
        const int count = __popcll(__ballot(below));   // lane 0's place is below or equal by construction
        lo += (max(count, 1) - 1) * step;
        hi = min(lo + step, hi);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    int64_t r0 = off[lo], r1 = off[lo + 1];
    if (r0 < 0 || r1 < r0 || r1 > total) return TileOfRows{0, 0, lo};
    const int64_t at = r0 + (tile - (r0 / rows + lo)) * rows;
    if (at < r0 || at >= r1) return TileOfRows{0, 0, lo};
    return TileOfRows{(int)at, (int)min(at + rows, r1), lo};
}
inline int64_t tiles_of_rows(int64_t n, int64_t total, int64_t rows, bool across) {
    return across ? (total + rows - 1) / rows : total / rows + n;
}

// One head's bias, in units of log 2, for every distance -reach .. reach, and kBeyond places more at both ends that
// repeat the last ones: a tile of 64 keys (or rows) by 32 rows (or keys) that reaches into -reach .. reach
// anywhere finds all of its distances there, by one address and constant offsets.
constexpr int kBeyond = 96;
// A bias of fp16's lowest value or less is a mask: minus infinity, which no 32-bit sum with a score rounds, so that the
// weights that the gradients make again are zero as well, and a row that it leaves nothing is found by its sum of zero.
template <class T>
__device__ __forceinline__ float bias_of(const AttentionArgs& a, int bucket, int head) {
    const float x = (float)static_cast<const typename T::elem*>(a.bias)[(int64_t)bucket * a.heads + head];
    return x <= -65504.f ? -INFINITY : x * kLog2e;
}
__host__ __device__ constexpr int bias_width(int reach) { return 2 * reach + 1 + 2 * kBeyond; }
template <class T>
__device__ __forceinline__ void fill_bias(float* table, const AttentionArgs& a, int head, int tid, int threads) {
    for (int i = tid; i < bias_width(a.reach); i += threads) {
        int b = a.bucket[min(max(i - kBeyond, 0), 2 * a.reach)];
        if (b < 0 || b >= a.n_buckets) {
            atomicOr(a.err, kDevBadBucket);
            b = 0;
        }
        table[i] = bias_of<T>(a, b, head);
    }
}
// Where a lane's smallest distance of a tile lies (59 places are read from there on), kept inside the table: beyond it all
// places are alike.
__device__ __forceinline__ const float* bias_from(const float* table, int reach, int distance) {
    return table + min(max(distance + reach + kBeyond, 0), 2 * reach + 2 * kBeyond - 59);
}

// (the same in every lane, and the compiler is told so: branches on it are scalar)
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) x = min(x, __shfl_xor(x, m));
    return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) x = max(x, __shfl_xor(x, m));
    return __builtin_amdgcn_readfirstlane(x);
}

}  // namespace surel
