// What the kernels of attention over a cache share: which wave goes over which keys.
#pragma once

#include "attention.h"
#include "cache.h"
#include "cache_share.h"

namespace surel {

// What the waves share, beside the call's arguments.
struct Share {
    const int64_t* entries = nullptr;    // tiles of every `each` sequences, or null: each is 1, a sequence's length says it
    int32_t n_entries = 0, each = 1;
    int32_t waves = 0, units = 1;        // wave w: part w / units of unit w % units
    int32_t head_tiles = 1, columns = 1; // units of a key head, query heads of a unit (the last has fewer)
    bool cuts = false;                   // some sequence may be cut
    int2* cut = nullptr;                 // [waves]: where a wave's is the first part that begins inside a sequence, that one, and
                                         // how many parts have some of it; else -1
    float *part_o = nullptr, *part_ml = nullptr;   // [waves][2][columns][dim], [waves][2][columns][2]: maximum (base 2), sum
};

__device__ __forceinline__ int64_t lane_of(int64_t x, int lane) { return __shfl(x, lane); }
__device__ __forceinline__ int64_t sum_till(int64_t x) {   // of the lanes up to this one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up(x, d);
        if (lane_id() >= d) x += y;
    }
    return x;
}

__device__ __forceinline__ int length_of(const CacheAttention& a, int s) {
    const int n = a.length[s];
    return n < 0 || n > a.width * (int64_t)a.page_rows.d ? 0 : n;
}
__device__ __forceinline__ int tiles_of(int length) { return (length + kCacheTile - 1) / kCacheTile; }

// A list of n <= kLookup counts: its sums by 64 lanes, then the entry that `target` falls into and what is left of it there.
struct Lookup {
    int64_t till, mine;   // lanes' sums
    int per;
    template <class Count>
    __device__ __forceinline__ int64_t sums(int n, Count count) {
        per = (n + 63) / 64;
        const int from = lane_id() * per;
        mine = 0;
#pragma unroll 8
        for (int i = 0; i < per; ++i) mine += from + i < n ? count(min(from + i, n - 1)) : 0;
        till = sum_till(mine);
        return lane_of(till, 63);
    }
    template <class Count>   // target below the list's sum
    __device__ __forceinline__ int find(int n, int64_t target, int64_t* left, Count count) const {
        const int l = min((int)__popcll(__ballot(till <= target)), 63);
        const int64_t rest = target - lane_of(till - mine, l);
        const int at = l * per + lane_id();
        const int64_t x = lane_id() < per && at < n ? count(min(at, n - 1)) : 0;
        const int64_t up_to = sum_till(x);
        const int e = min((int)__popcll(__ballot(lane_id() < per && up_to <= rest)), per - 1);
        *left = rest - lane_of(up_to - x, e);
        return l * per + e;
    }
};

// A tile of a sequence.
struct Place {
    int seq, tile, tiles, length;
};

// Writes zeros for sequences of no keys; every wave takes some, and looks at 64 of them at a time.
__device__ __forceinline__ void write_empty(const CacheAttention& a, const Share& o, int wave) {
    const int lane = lane_id();
    for (int64_t first = (int64_t)wave * 64; first < a.n_seqs; first += (int64_t)o.waves * 64) {
        const int n = first + lane < a.n_seqs ? a.length[first + lane] : 1;
        const bool bad = n < 0 || n > a.width * (int64_t)a.page_rows.d;
        raise_error(a.err, bad, kDevBadLength);
        for (unsigned long long none = __ballot(n == 0 || bad); none != 0; none &= none - 1) {
            const int64_t s = first + (int)__builtin_ctzll(none);
            uint32_t* const out = static_cast<uint32_t*>(a.out) + s * a.heads * (a.dim / 2);
            for (int i = lane; i < a.heads * (a.dim / 2); i += 64) out[i] = 0;
            for (int i = lane; i < a.heads; i += 64) a.lse[s * a.heads + i] = -INFINITY;
        }
    }
}

// A wave's part: where it begins, and how many tiles it has.  Notes where it is the first that begins inside a sequence.
struct Course {
    Place at;
    int64_t first, tiles;   // its first tile's number; 0 tiles: no part
};
__device__ __forceinline__ Course course_of(const CacheAttention& a, const Share& o, int wave) {
    auto tiles_of_seq = [&](int s) { return (int64_t)tiles_of(length_of(a, s)); };
    auto tiles_of_entry = [&](int e) { return o.entries == nullptr ? tiles_of_seq(e) : o.entries[e]; };
    Course c;
    c.first = c.tiles = 0;
    Lookup list;
    const int64_t tiles = list.sums(o.n_entries, tiles_of_entry);
    const int64_t parts = parts_of(tiles, o.waves / o.units), part = wave / o.units;
    if (part < parts) {
        auto place_of = [&](int64_t target) {   // the place of a tile by its number
            int64_t left;
            int s = list.find(o.n_entries, target, &left, tiles_of_entry);
            if (o.entries != nullptr) {
                const int first = s * o.each, n = min(o.each, a.n_seqs - first);
                Lookup inner;
                auto count = [&](int i) { return tiles_of_seq(first + i); };
                (void)inner.sums(n, count);
                s = first + inner.find(n, left, &left, count);
            }
            Place p;
            p.seq = uniform(s);
            p.length = uniform(length_of(a, p.seq));
            p.tiles = tiles_of(p.length);
            p.tile = uniform((int)left);
            return p;
        };
        int64_t begin = part_begin(tiles, parts, part), end = part_begin(tiles, parts, part + 1);
        c.at = place_of(begin);
        const int64_t back = moves_back(c.at.tile, c.at.tiles);
        begin -= back, c.at.tile -= (int)back;
        if (part + 1 < parts) {
            const Place behind = place_of(end);
            end -= moves_back(behind.tile, behind.tiles);
        }
        c.first = begin, c.tiles = end - begin;
    }
    if (o.cuts && lane_id() == 0) {
        const int64_t first = c.tiles > 0 ? c.first - c.at.tile : 0;   // the sequence's first tile
        const bool is_first = c.tiles > 0 && c.at.tile > 0 && part_with(tiles, parts, first) == part - 1;
        o.cut[wave] = is_first ? int2{c.at.seq, (int)(part_with(tiles, parts, first + c.at.tiles - 1) - part + 2)} : int2{-1, 0};
    }
    return c;
}

// The first of the places from .. to - 1 whose count is not zero, else `to`: a wave looks at 256 at a time, so that four trips to
// memory are together.
template <class Count>
__device__ __forceinline__ int first_with_keys(int from, int to, Count count) {
#pragma unroll 1
    for (int at = from; at < to; at += 256) {
        bool some[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) some[i] = count(min(at + 64 * i + lane_id(), to - 1)) != 0;   // (the last may be looked at again)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (const unsigned long long found = __ballot(some[i]); found != 0) return min(at + 64 * i + (int)__builtin_ctzll(found), to - 1);
    }
    return to;
}
// The sequence with keys that comes first behind one, or n_seqs.  Ended sequences have none, and there may be any number of
// them: of more than kLookup sequences, entries of the list are looked through between the places of two of them.
__device__ __forceinline__ int next_with_keys(const CacheAttention& a, const Share& o, int seq) {
    auto keys = [&](int s) { return length_of(a, s); };
    if (o.entries == nullptr) return first_with_keys(seq + 1, a.n_seqs, keys);
    int entry = seq / o.each;
    auto end = [&] { return min((entry + 1) * o.each, a.n_seqs); };
    const int s = first_with_keys(seq + 1, end(), keys);
    if (s < end()) return s;
    entry = first_with_keys(entry + 1, o.n_entries, [&](int e) { return (int)(o.entries[e] != 0); });
    return entry < o.n_entries ? first_with_keys(entry * o.each, end(), keys) : a.n_seqs;
}

// The place behind one, in the same part; of no keys where there is none.  The next sequence is looked at by itself, by a scalar
// load: those of a wave's lanes would wait for the keys that are on their way.  (Two that run, the first and the last of 4,096
// places: a call of 56 us, of a million 94, where none runs 43 and 91; with places looked at one by one 450 us and 108 ms.)
__device__ __forceinline__ Place following(const CacheAttention& a, const Share& o, const Place& p) {
    Place n = p;
    if (++n.tile < p.tiles) return n;
    n.tile = 0;
    int s = p.seq + 1;
    n.length = s < a.n_seqs ? uniform(length_of(a, s)) : 0;
    if (n.length == 0) {
        s = uniform(next_with_keys(a, o, s));
        n.length = s < a.n_seqs ? uniform(length_of(a, s)) : 0;
    }
    n.seq = min(s, a.n_seqs - 1);
    n.tiles = tiles_of(n.length);
    return n;
}

// Biases by distance, in units of log 2, for a call's distances 0 .. farthest: of all heads in LDS where these are few, else
// looked up.  (A bias of fp16's lowest value or less is a mask.)
__host__ __device__ __forceinline__ int farthest(const CacheAttention& a) {   // beyond it biases are alike, or no key is
    const int64_t keys = (int64_t)a.width * a.page_rows.d;
    return a.reach < keys ? a.reach : (int)keys - 1;
}
template <class T>
struct Biases {
    const CacheAttention& a;
    const float* table;   // [heads][far + 1], or null
    int far;
    __device__ __forceinline__ int bucket_of(int distance, bool* bad) const {
        const int b = a.bucket[a.reach - distance];
        const bool none = b < 0 || b >= a.n_buckets;
        *bad = *bad || none;
        return none ? 0 : b;
    }
    __device__ __forceinline__ float in_bucket(int b, int head) const {
        const float x = (float)static_cast<const typename T::elem*>(a.bias)[(int64_t)b * a.heads + head];
        return x <= -65504.f ? -INFINITY : x * kLog2e;
    }
    __device__ __forceinline__ float at(int head, int distance) const {
        if (table != nullptr) return table[head * (far + 1) + distance];
        bool bad = false;
        const float x = in_bucket(bucket_of(distance, &bad), head);
        if (bad) atomicOr(a.err, kDevBadBucket);
        return x;
    }
    // All threads of a workgroup, four entries each at a time, so that their trips to memory are together.
    __device__ __forceinline__ void fill(float* to) const {
        const int n = a.heads * (far + 1), threads = (int)blockDim.x;
        bool bad = false;
#pragma unroll 1
        for (int i0 = threadIdx.x; i0 < n; i0 += 4 * threads) {
            int b[4], head[4];
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = min(i0 + e * threads, n - 1);
                head[e] = i / (far + 1);
                b[e] = bucket_of(i - head[e] * (far + 1), &bad);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = in_bucket(b[e], head[e]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i0 + e * threads < n) to[i0 + e * threads] = x[e];
        }
        raise_error(a.err, bad, kDevBadBucket);
    }
};

// cache_lanes.hip: rows that few query heads share a key head with, by the vector units.
bool lanes_serve(int group);
int lanes_waves(int group, int dim);   // of a compute unit
template <class T>
hipError_t launch_lanes(hipStream_t stream, const CacheAttention& a, const Share& o);

}  // namespace surel
