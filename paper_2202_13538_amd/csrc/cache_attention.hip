// Attention of one row a sequence to its keys in a paged cache (surel_cache_attention).
#include "attention.h"
#include "cache.h"
#include "cache_share.h"
#include "kernels.h"

namespace surel {
namespace {

// fp16: weights are relative to 2^-7 of the largest, so that those down to 2^-21 of it keep all their bits, and stay below 2^15;
// bf16 has the range of 32-bit floats.  What a lane's weights of a tile may add up to before a larger maximum is looked for:
template <class T>
constexpr float kBelow = T::kNarrow ? 7.f : 0.f;
template <class T>
constexpr float kMost = T::kNarrow ? 32768.f : 1024.f;

constexpr int kJoinThreads = 256;
constexpr int kMostDim = 128;

// What the waves share, beside the call's arguments.
struct Share {
    const int64_t* entries = nullptr;    // tiles of every `each` sequences, or null: each is 1, a sequence's length says it
    int32_t n_entries = 0, each = 1;
    int32_t waves = 0;
    int32_t head_tiles = 1, columns = 1; // units of a key head, query heads of a unit (the last has fewer)
    bool cuts = false;                   // some pair may be cut
    int64_t* cut = nullptr;              // [waves]: the pair that a wave's part begins inside of, or -1
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

// A tile of a pair: sequence, unit, tile.
struct Place {
    int seq, unit, tile, tiles, length;
};

template <class T, int DP>
__global__ __launch_bounds__(64) void cache_attention_kernel(CacheAttention a, Share o) {
    constexpr int NB = DP / 32, kRowBytes = Tile<DP>::kRowBytes, kTileBytes = kCacheTile * kRowBytes;
    constexpr int kChunks = Tile<DP>::kChunks, kCopies = kCacheTile * kChunks / 64;
    extern __shared__ __align__(256) char lds[];   // [buffer][keys, values]
    const int lane = threadIdx.x, g = lane >> 5, col = lane & 31;
    const int wave = (int)block_number();
    if (wave >= o.waves) return;
    const int units = a.kv_heads * o.head_tiles, group = a.heads / a.kv_heads;

    // sequences of no keys: zeros
    for (int64_t s = wave; s < a.n_seqs; s += o.waves) {
        const int n = uniform(a.length[s]);
        if (n > 0 && n <= a.width * (int64_t)a.page_rows.d) continue;
        if (n != 0 && lane == 0) atomicOr(a.err, kDevBadLength);
        uint32_t* const out = static_cast<uint32_t*>(a.out) + s * a.heads * (a.dim / 2);
        for (int i = lane; i < a.heads * (a.dim / 2); i += 64) out[i] = 0;
        for (int i = lane; i < a.heads; i += 64) a.lse[s * a.heads + i] = -INFINITY;
    }

    // the wave's part
    auto tiles_of_seq = [&](int s) { return (int64_t)tiles_of(length_of(a, s)) * units; };
    auto tiles_of_entry = [&](int e) { return o.entries == nullptr ? tiles_of_seq(e) : o.entries[e] * units; };
    Lookup list;
    const int64_t tiles = list.sums(o.n_entries, tiles_of_entry);
    const int64_t parts = parts_of(tiles, o.waves);
    if (wave >= parts) {
        if (o.cuts && lane == 0) o.cut[wave] = -1;
        return;
    }
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
        p.unit = uniform((int)(left / p.tiles));
        p.tile = uniform((int)(left - (int64_t)p.unit * p.tiles));
        return p;
    };
    int64_t begin = part_begin(tiles, parts, wave), end = part_begin(tiles, parts, wave + 1);
    Place next = place_of(begin);
    {
        const int64_t back = moves_back(next.tile, next.tiles);
        begin -= back, next.tile -= (int)back;
        if (wave + 1 < parts) {
            const Place behind = place_of(end);
            end -= moves_back(behind.tile, behind.tiles);
        }
    }
    if (o.cuts && lane == 0) o.cut[wave] = begin < end && next.tile > 0 ? (int64_t)next.seq * units + next.unit : -1;
    if (begin >= end) return;

    const float c = a.scale * kLog2e;   // scores in units of log 2
    const bool padded = a.dim != DP;
    auto zero_pads = [&](char* tile) {  // columns at and beyond dim: copies leave them out
        for (int i = lane; i < kCacheTile * kChunks; i += 64) {
            const int r = i / kChunks, ch = i % kChunks;
            if (ch * 8 >= a.dim) *reinterpret_cast<u32x4*>(tile + r * kRowBytes + ((ch ^ Tile<DP>::permuted(r)) * 16)) = u32x4{0, 0, 0, 0};
        }
    };
    if (padded)
        for (int i = 0; i < 4; ++i) zero_pads(lds + i * kTileBytes);

    // Three tiles are on their way at a time: one in LDS, one coming there, and the pages of one looked up.
    auto follow = [&](const Place& p) {   // the place behind this one, in the same part
        Place n = p;
        if (++n.tile < p.tiles) return n;
        n.tile = 0;
        if (++n.unit < units) return n;
        n.unit = 0;
        do {
            if (++n.seq >= a.n_seqs) break;
            n.length = uniform(length_of(a, n.seq));
        } while (n.length == 0);
        n.tiles = tiles_of(n.length);
        return n;
    };
    auto look_up = [&](const Place& p) {   // the page of the tile's key of number `col`
        const int key = min(p.tile * kCacheTile + col, p.length - 1);
        return a.pages[(int64_t)p.seq * a.width + a.page_rows.of((uint32_t)key)];
    };
    typedef __attribute__((address_space(3))) void* lds_ptr;
    typedef const __attribute__((address_space(1))) void* global_ptr;
    auto fetch = [&](const Place& p, int page, int buffer) {   // returns which keys lie in no page, a bit each
        const bool bad = page < 0 || page >= a.n_pages;
        const int key = min(p.tile * kCacheTile + col, p.length - 1);
        const uint32_t in_page = (uint32_t)key - a.page_rows.of((uint32_t)key) * a.page_rows.d;
        const int64_t from = bad ? 0 : page * a.page + (int64_t)in_page * a.row;
        const uint32_t lo = (uint32_t)from, hi = (uint32_t)(from >> 32);
        const int64_t head = (int64_t)(p.unit / o.head_tiles) * a.head;
        char* const k_tile = lds + buffer * 2 * kTileBytes;
#pragma unroll
        for (int n = 0; n < kCopies; ++n) {
            const int id = lane + 64 * n, row = id / kChunks, ch = (id % kChunks) ^ Tile<DP>::permuted(row);
            const uint64_t at = ((uint64_t)__shfl(hi, row) << 32 | __shfl(lo, row)) + head + ch * 16;
            if (ch * 8 < a.dim) {
                __builtin_amdgcn_global_load_lds((global_ptr)(a.k_pages + at), (lds_ptr)(k_tile + n * 1024), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((global_ptr)(a.v_pages + at), (lds_ptr)(k_tile + kTileBytes + n * 1024), 16, 0, 0);
            }
        }
        return (uint32_t)__ballot(bad);
    };
    auto head_of = [&](const Place& p) { return p.unit / o.head_tiles * group + p.unit % o.head_tiles * o.columns + col; };
    auto counts_in = [&](const Place& p) { return col < min(o.columns, group - p.unit % o.head_tiles * o.columns); };

    f32x16 acc[NB];
    float top = -INFINITY, sum = 0.f;
    Stationary<DP> q, q_next;
    int page = look_up(next), first_tile = next.tile;
    Place now = next;
    int64_t left = end - begin;   // tiles of the part, the present one among them
    uint32_t gone = fetch(now, page, 0), gone_next = 0;
    q_next.load(a.q + (int64_t)now.seq * a.q_row + (int64_t)head_of(now) * a.q_head, counts_in(now), a.dim, lane);
    if (left > 1) {
        next = follow(now);
        page = look_up(next);
    }
    bool fresh = true;
    int buffer = 0;
#pragma unroll 1
    for (;; buffer ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0070);   // everything on its way is here, and what was read from LDS
        wave_sync();
        if (gone != 0) {   // keys in no page: zeros, since what is copied in their place need not be finite
            if (lane == 0) atomicOr(a.err, kDevBadPage);
            for (int i = lane; i < 2 * kCacheTile * kChunks; i += 64)
                if (gone >> (i / kChunks % kCacheTile) & 1) *reinterpret_cast<u32x4*>(lds + buffer * 2 * kTileBytes + i * 16) = u32x4{0, 0, 0, 0};
            wave_sync();
        }
        if (fresh) {
            q = q_next;
            top = -INFINITY, sum = 0.f, first_tile = now.tile;
#pragma unroll
            for (int db = 0; db < NB; ++db) acc[db] = f32x16{};
        }
        Place after = next;
        if (left > 1) {
            gone_next = fetch(next, page, buffer ^ 1);
            if (next.tile == 0)
                q_next.load(a.q + (int64_t)next.seq * a.q_row + (int64_t)head_of(next) * a.q_head, counts_in(next), a.dim, lane);
            if (left > 2) {
                after = follow(next);
                page = look_up(after);
            }
        }

        const uint32_t kt = buffer * 2 * kTileBytes, vt = kt + kTileBytes;
        const int key0 = now.tile * kCacheTile, head = head_of(now);
        const bool counts = counts_in(now);
        f32x16 s = scores<T, DP>(lds, kt, q, lane);
        if (a.bias == nullptr) {
            s *= c;
        } else {
            const int ahead = key0 + 4 * g - (now.length - 1) + a.reach;   // place in the list of buckets, of the lane's first key
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                int b = a.bucket[max(min(ahead + row_of(i, 0), a.reach), 0)];
                if (b < 0 || b >= a.n_buckets) {
                    atomicOr(a.err, kDevBadBucket);
                    b = 0;
                }
                const float x = counts ? (float)static_cast<const typename T::elem*>(a.bias)[(int64_t)b * a.heads + head] : 0.f;
                s[i] = __builtin_fmaf(s[i], c, x <= -65504.f ? -INFINITY : x * kLog2e);
            }
        }
        if (key0 + kCacheTile > now.length || gone != 0) {
            const uint32_t none = gone | (key0 + kCacheTile > now.length ? ~0u << (now.length - key0) : 0u);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = none >> row_of(i, g) & 1 ? -INFINITY : s[i];
        }
        auto largest = [&] {
            float most = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) most = fmaxf(most, s[i]);
            return fmaxf(most, from_other_half(most));
        };
        auto raise_top = [&](bool mine) {
            const float most = largest();
            const float to = mine ? fmaxf(top, most - kBelow<T>) : top;
            const float shrink = to == top ? 1.f : exp2_fast(top - to);
            top = to;
            sum *= shrink;
#pragma unroll
            for (int db = 0; db < NB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] *= shrink;
        };
        f32x16 p;
        auto weights = [&] {   // returns their sum
            const float base = top == -INFINITY ? 0.f : top;
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = exp2_fast(s[i] - base);
                part += p[i];
            }
            return part;
        };
        if (__any(top == -INFINITY)) raise_top(top == -INFINITY);
        float part = weights();
        const bool over = !(fmaxf(part, from_other_half(part)) < kMost<T>);
        if (__any(over)) {
            raise_top(over);
            part = weights();
        }
        sum += part;
        accumulate<T, DP>(acc, lds, vt, p, lane);

        const bool ends = now.tile + 1 == now.tiles || left == 1;
        if (ends) {
            const float all = sum + from_other_half(sum);
            if (first_tile > 0 || now.tile + 1 < now.tiles) {   // a part of a pair
                const int64_t at = ((int64_t)wave * 2 + (first_tile > 0 ? 0 : 1)) * o.columns + col;
                if (counts) {
                    if (g == 0) o.part_ml[2 * at] = top, o.part_ml[2 * at + 1] = all;
#pragma unroll
                    for (int db = 0; db < NB; ++db)
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const int d = 32 * db + row_of(i, g);
                            if (d < a.dim)   // dim is a multiple of 8, d of 4
                                *reinterpret_cast<f32x4*>(o.part_o + at * a.dim + d) =
                                    f32x4{acc[db][i], acc[db][i + 1], acc[db][i + 2], acc[db][i + 3]};
                        }
                }
            } else {
                const int64_t row = (int64_t)now.seq * a.heads;
                if (counts && g == 0) a.lse[row + head] = (top + log2_fast(all)) * kLn2;
                const bool none = all == 0.f;   // all that it sees is masked by a bias, or in no page
                const int columns = min(o.columns, group - now.unit % o.head_tiles * o.columns);
                store_rows<T, DP>(acc, none ? 0.f : 1.f / all, none, lds + kt, a.dim, lane, [&](int r) -> char* {
                    if (r >= columns) return nullptr;
                    return static_cast<char*>(a.out) + (row + head - col + r) * a.dim * 2;
                });
                if (padded) zero_pads(lds + kt);
            }
        }
        if (--left == 0) break;
        fresh = ends;
        now = next, next = after, gone = gone_next;
    }
}

// The sums of a pair that several waves share: a workgroup for every wave whose part begins inside a pair, and column;
// the pair's first of these joins.  Its waves take parts in turn, in a fixed order.
template <class T>
__global__ __launch_bounds__(kJoinThreads) void cache_attention_join_kernel(CacheAttention a, Share o) {
    constexpr int kWaves = kJoinThreads / 64;
    __shared__ float tops[kWaves], totals[kWaves], sums[kWaves][kMostDim];
    const int64_t block = block_number();
    const int w = (int)(block / o.columns), column = (int)(block % o.columns);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (w < 1 || w >= o.waves) return;
    const int64_t pair = o.cut[w];
    if (pair < 0 || o.cut[w - 1] == pair) return;
    const int units = a.kv_heads * o.head_tiles, group = a.heads / a.kv_heads;
    const int unit = (int)(pair % units), seq = (int)(pair / units), column0 = unit % o.head_tiles * o.columns;
    if (column >= min(o.columns, group - column0)) return;
    int last = w;   // the last wave with a part of the pair
    for (int from = w + 1;; from += 64) {
        const unsigned long long in = __ballot(from + lane < o.waves && o.cut[min(from + lane, o.waves - 1)] == pair);
        const int n = in == ~0ull ? 64 : (int)__builtin_ctzll(~in);
        last += n;
        if (n < 64) break;
    }
    const int parts = last - w + 2;   // of waves w - 1 (its second), w, .. last (their first)
    auto part_of = [&](int i) { return ((int64_t)(w - 1 + i) * 2 + (i == 0 ? 1 : 0)) * o.columns + column; };
    float top = -INFINITY;
    for (int i = threadIdx.x; i < parts; i += kJoinThreads) {
        const float2 ml = *reinterpret_cast<const float2*>(o.part_ml + 2 * part_of(i));
        if (ml.y != 0.f) top = fmaxf(top, ml.x);   // (a part that saw nothing has no say)
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
    if (lane == 0) tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWaves; ++k) top = fmaxf(top, tops[k]);
    const float base = top == -INFINITY ? 0.f : top;
    f32x2 x = {0.f, 0.f};
    float total = 0.f;
    const bool mine = 2 * lane < a.dim;
#pragma unroll 8
    for (int i = wave; i < parts; i += kWaves) {
        const int64_t at = part_of(i);
        const float2 ml = *reinterpret_cast<const float2*>(o.part_ml + 2 * at);
        const float weight = ml.y == 0.f ? 0.f : ml.x == top ? 1.f : exp2_fast(ml.x - base);
        const f32x2 y = mine ? *reinterpret_cast<const f32x2*>(o.part_o + at * a.dim + 2 * lane) : f32x2{0.f, 0.f};
        total = __builtin_fmaf(weight, ml.y, total);
        if (weight != 0.f) x[0] = __builtin_fmaf(weight, y[0], x[0]), x[1] = __builtin_fmaf(weight, y[1], x[1]);
    }
    if (lane == 0) totals[wave] = total;
    if (mine) sums[wave][2 * lane] = x[0], sums[wave][2 * lane + 1] = x[1];
    __syncthreads();
    if (wave != 0) return;
    total = 0.f;
    x = f32x2{0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        total += totals[k];
        if (mine) x[0] += sums[k][2 * lane], x[1] += sums[k][2 * lane + 1];
    }
    const int64_t row = (int64_t)seq * a.heads + unit / o.head_tiles * group + column0 + column;
    if (lane == 0) a.lse[row] = total == 0.f ? -INFINITY : (top + log2_fast(total)) * kLn2;
    const float scale = total == 0.f ? 0.f : 1.f / total;
    if (mine) static_cast<uint32_t*>(a.out)[row * (a.dim / 2) + lane] = pack2<T>(x[0] * scale, x[1] * scale);
}

// Tiles of every `each` sequences: a wave an entry.
__global__ __launch_bounds__(256) void cache_entries_kernel(CacheAttention a, int64_t* entries, int n_entries, int each) {
    const int64_t e = (int64_t)block_number() * 4 + (threadIdx.x >> 6);
    if (e >= n_entries) return;
    int64_t n = 0;
    for (int64_t s = e * each + (threadIdx.x & 63); s < min((e + 1) * each, (int64_t)a.n_seqs); s += 64) n += tiles_of(length_of(a, (int)s));
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) n += __shfl_xor(n, m);
    if ((threadIdx.x & 63) == 0) entries[e] = n;
}

// Waves of a compute unit: as many as its 160 KB of LDS have room for, two buffers of keys and values each.
int padded_dim(int dim) { return (dim + 31) / 32 * 32; }
int tile_bytes(int dim) { return 4 * kCacheTile * 2 * padded_dim(dim); }
int waves_of_a_unit(int dim) { return 163840 / tile_bytes(dim) < 16 ? 163840 / tile_bytes(dim) : 16; }

struct Plan {
    Share o;
    size_t entry_bytes = 0, cut_bytes = 0, o_bytes = 0, ml_bytes = 0;
    size_t bytes() const { return entry_bytes + cut_bytes + o_bytes + ml_bytes; }
};
Plan plan_of(int n_cu, const CacheAttention& a) {
    Plan p;
    const int group = a.heads / a.kv_heads;
    p.o.head_tiles = (group + 31) / 32;
    p.o.columns = group < 32 ? group : 32;
    p.o.each = (int32_t)seqs_of_an_entry(a.n_seqs);
    p.o.n_entries = (int32_t)((a.n_seqs + p.o.each - 1) / p.o.each);
    const int64_t most_tiles = ((int64_t)a.width * a.page_rows.d + kCacheTile - 1) / kCacheTile;
    p.o.cuts = may_be_cut(most_tiles);
    const int64_t waves = parts_of(most_tiles * a.kv_heads * p.o.head_tiles * a.n_seqs, (int64_t)n_cu * waves_of_a_unit(a.dim));
    p.o.waves = (int32_t)waves;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    if (p.o.each > 1) p.entry_bytes = up((size_t)p.o.n_entries * 8);
    if (p.o.cuts) {
        p.cut_bytes = up((size_t)waves * 8);
        p.o_bytes = up((size_t)waves * 2 * p.o.columns * a.dim * 4);
        p.ml_bytes = up((size_t)waves * 2 * p.o.columns * 8);
    }
    return p;
}

template <class T, int DP>
hipError_t launch(hipStream_t stream, const CacheAttention& a, const Share& o) {
    hipLaunchKernelGGL((cache_attention_kernel<T, DP>), grid_of(o.waves), dim3(64), tile_bytes(DP), stream, a, o);
    return hipGetLastError();
}

template <class T>
hipError_t launch_type(hipStream_t stream, const CacheAttention& a, const Share& o) {
    hipError_t rc = a.dim <= 32   ? launch<T, 32>(stream, a, o)
                    : a.dim <= 64 ? launch<T, 64>(stream, a, o)
                    : a.dim <= 96 ? launch<T, 96>(stream, a, o)
                                  : launch<T, 128>(stream, a, o);
    if (rc != hipSuccess || !o.cuts) return rc;
    hipLaunchKernelGGL(cache_attention_join_kernel<T>, grid_of((int64_t)o.waves * o.columns), dim3(kJoinThreads), 0, stream, a, o);
    return hipGetLastError();
}

}  // namespace

size_t cache_attention_scratch_bytes(int n_cu, const CacheAttention& a) { return plan_of(n_cu, a).bytes(); }

hipError_t launch_cache_attention(hipStream_t stream, int n_cu, CacheAttention a, bool half, void* scratch) {
    Plan p = plan_of(n_cu, a);
    char* at = static_cast<char*>(scratch);
    if (p.o.each > 1) {
        int64_t* const entries = reinterpret_cast<int64_t*>(at);
        hipLaunchKernelGGL(cache_entries_kernel, grid_of((p.o.n_entries + 3) / 4), dim3(256), 0, stream, a, entries, p.o.n_entries, p.o.each);
        if (const hipError_t rc = hipGetLastError(); rc != hipSuccess) return rc;
        p.o.entries = entries;
        at += p.entry_bytes;
    }
    if (p.o.cuts) {
        p.o.cut = reinterpret_cast<int64_t*>(at);
        p.o.part_o = reinterpret_cast<float*>(at + p.cut_bytes);
        p.o.part_ml = reinterpret_cast<float*>(at + p.cut_bytes + p.o_bytes);
    }
    return half ? launch_type<Fp16>(stream, a, p.o) : launch_type<Bf16>(stream, a, p.o);
}

}  // namespace surel
