// Attention of one row a sequence to its keys in a paged cache (surel_cache_attention).
#include "cache_attention.h"
#include "kernels.h"

namespace surel {
namespace {

constexpr int kJoinThreads = 512;

constexpr int kThreads = 256;
constexpr int kMostTable = 4096;   // biases of all heads by distance that are kept in LDS

// fp16: weights are relative to 2^-7 of the largest, so that those down to 2^-21 of it keep all their bits, and stay below 2^15;
// bf16 has the range of 32-bit floats.  What a lane's weights of a tile may add up to before a larger maximum is looked for:
template <class T>
constexpr float kBelow = T::kNarrow ? 7.f : 0.f;
template <class T>
constexpr float kMost = T::kNarrow ? 32768.f : 1024.f;

// C[16 x 16] += A[16 x 32] B[32 x 16] of one wave: lane l holds the row (of A) or column (of B) l % 16 and the inner values
// 8 (l / 16) .. + 7; of C it holds column l % 16 and rows 4 (l / 16) .. + 3.
__device__ __forceinline__ f32x4 mma16(Bf16, u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16::x8, a), __builtin_bit_cast(Bf16::x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(Fp16, u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Fp16::x8, a), __builtin_bit_cast(Fp16::x8, b), c, 0, 0, 0);
}
// The values of the lanes 16, 32 and 48 further on, with op.
template <class Op>
__device__ __forceinline__ float over_quarters(float x, Op op) {
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t w = __float_as_uint(x);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Waves of a SIMD: what registers have room for, and a compute unit's 160 KB of LDS, with two buffers of a tile's values each.
constexpr int waves_of_a_simd(int padded, int blocks) {
    return blocks == 2 ? (padded > 64 ? 1 : 2) : padded > 64 ? 2 : padded > 32 ? 3 : 4;
}

// One wave: up to 16 BLOCKS query heads that share a key head, over its part of all keys (cache_share.h), 32 at a time.
// Scores are K q^T, so that a head's lie in the four lanes of a column, its softmax runs inside lanes, and the weights are the
// operand of out^T += V^T p^T as they come.  Keys go from memory to registers, as the first product's operand lies; values, which
// the second needs transposed, through LDS, without passing through registers.
// What bounds it: memory, and for caches of a gigabyte and less the starts and ends of parts.  256 caches of 1 to 8,192 keys, 16
// heads to 2 of 128 elements, with a bias: 229 us, 4.5 TB/s; 1,024 of them 788 with the join, 5.4 TB/s.  (With 32-column
// products and keys through LDS as well, 302: four times the softmax for 8 heads, and half the waves.)  Weights are rounded to
// 16 bits for their product, as surel_attention's are (results of that call: 0.0020 of their size off, where their own rounding alone
// is 0.0017); sums and statistics are 32-bit.
template <class T, int DP, int BLOCKS>
__global__ __launch_bounds__(kThreads, waves_of_a_simd(DP, BLOCKS)) void cache_attention_kernel(CacheAttention a, Share o, int in_table) {
    constexpr int NB = DP / 16, NK = DP / 32, kRowBytes = Tile<DP>::kRowBytes, kTileBytes = kCacheTile * kRowBytes;
    constexpr int kChunks = Tile<DP>::kChunks, kCopies = kCacheTile * kChunks / 64;
    extern __shared__ __align__(256) char lds[];   // [wave][buffer], then biases, see Biases
    const int lane = threadIdx.x & 63, in_group = uniform((int)(threadIdx.x >> 6));
    const int g = lane >> 4, col = lane & 15, of_tile = lane & 31;
    const int wave = (int)block_number() * (kThreads / 64) + in_group;
    float* const table = reinterpret_cast<float*>(lds + kThreads / 64 * 2 * kTileBytes);
    const Biases<T> biases = {a, in_table ? table : nullptr, farthest(a)};
    if (in_table) {
        biases.fill(table);
        __syncthreads();
    }
    const int far = biases.far;
    if (wave >= o.waves) return;
    write_empty(a, o, wave);
    const int group = a.heads / a.kv_heads, unit = wave % o.units, column0 = unit % o.head_tiles * o.columns;
    const int columns = min(o.columns, group - column0), head = unit / o.head_tiles * group + column0;   // the unit's
    const Course course = course_of(a, o, wave);
    if (course.tiles <= 0) return;

    const float c = a.scale * kLog2e;   // scores in units of log 2
    char* const tiles = lds + in_group * 2 * kTileBytes;
    if (a.dim != DP) {                  // columns at and beyond dim: copies leave them out
        for (int i = lane; i < 2 * kCacheTile * kChunks; i += 64) {
            const int r = i / kChunks, ch = i % kChunks ^ Tile<DP>::permuted(r % kCacheTile);
            if (ch * 8 >= a.dim) *reinterpret_cast<u32x4*>(tiles + i * 16) = u32x4{0, 0, 0, 0};
        }
    }
    // where a lane's transposed values begin: 4 rows of its quarter, 4 elements of 16 columns each
    const int tr_row = 4 * g + (col >> 2), tr_chunk = (col & 3) >> 1;

    auto look_up = [&](const Place& p) {   // the page of the tile's key of number `of_tile`
        const int key = p.tile * kCacheTile + of_tile;
        return key < p.length ? a.pages[(int64_t)p.seq * a.width + a.page_rows.of((uint32_t)key)] : 0;
    };
    typedef __attribute__((address_space(3))) void* lds_ptr;
    typedef const __attribute__((address_space(1))) void* global_ptr;
    const char* const k_src = a.k_pages + (int64_t)(unit / o.head_tiles) * a.head;
    const char* const v_src = a.v_pages + (int64_t)(unit / o.head_tiles) * a.head;
    // Sends a tile's keys to registers and its values to LDS; returns which keys there are, a bit each.
    auto fetch = [&](const Place& p, int page, u32x4 (&k)[2][NK], int buffer) {
        const int key = p.tile * kCacheTile + of_tile;
        const bool bad = page < 0 || page >= a.n_pages;
        raise_error(a.err, bad, kDevBadPage);
        const uint32_t in_page = (uint32_t)key - a.page_rows.of((uint32_t)key) * a.page_rows.d;
        const bool there = !bad && key < p.length;
        const int64_t from = there ? page * a.page + (int64_t)in_page * a.row : 0;
        const uint32_t seen = (uint32_t)__ballot(there);
        const uint32_t lo = (uint32_t)from, hi = (uint32_t)(from >> 32);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char* const row = k_src + (int64_t)((uint64_t)(uint32_t)__shfl((int)hi, 16 * h + col) << 32 | (uint32_t)__shfl((int)lo, 16 * h + col));
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) {
                k[h][ks] = u32x4{0, 0, 0, 0};
                if ((seen >> (16 * h + col) & 1) && (4 * ks + g) * 8 < a.dim) k[h][ks] = *reinterpret_cast<const u32x4*>(row + (4 * ks + g) * 16);
            }
        }
        char* const tile = tiles + buffer * kTileBytes;
#pragma unroll
        for (int n = 0; n < kCopies; ++n) {
            const int id = lane + 64 * n, row = id / kChunks, ch = (id % kChunks) ^ Tile<DP>::permuted(row);
            const uint64_t at = (uint64_t)(uint32_t)__shfl((int)hi, row) << 32 | (uint32_t)__shfl((int)lo, row);
            if (ch * 8 < a.dim && (seen >> row & 1))
                __builtin_amdgcn_global_load_lds((global_ptr)(v_src + at + ch * 16), (lds_ptr)(tile + n * 1024), 16, 0, 0);
        }
        return seen;
    };
    auto load_q = [&](const Place& p, u32x4 (&q)[BLOCKS][NK]) {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) {
                q[b][ks] = u32x4{0, 0, 0, 0};
                if (16 * b + col < columns && (4 * ks + g) * 8 < a.dim)
                    q[b][ks] = *reinterpret_cast<const u32x4*>(a.q + (int64_t)p.seq * a.q_row + (int64_t)(head + 16 * b + col) * a.q_head +
                                                               (4 * ks + g) * 16);
            }
    };

    f32x4 acc[BLOCKS][NB];
    float top[BLOCKS], sum[BLOCKS];
    u32x4 k[2][2][NK], q[BLOCKS][NK], q_next[BLOCKS][NK];
    Place now = course.at, next = now, after;
    int64_t left = course.tiles;   // tiles of the part, the present one among them
    uint32_t there[2] = {0, 0};
    int page = look_up(now), page_next = 0, first_tile = 0;
    if (left > 1) next = following(a, o, now), page_next = look_up(next);
    load_q(now, q_next);
    there[0] = fetch(now, page, k[0], 0);
    page = page_next;
    after = next;
    bool fresh = true;

    // Three tiles are on their way at a time: one here, one coming, and the pages of one looked up.
    auto turn = [&](auto of) __attribute__((always_inline)) {
        constexpr int buffer = decltype(of)::value;
        __builtin_amdgcn_s_waitcnt(0x0070);   // everything on its way is here, and what was read from LDS
        wave_sync();
        if (fresh) {
            first_tile = now.tile;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                top[b] = -INFINITY, sum[b] = 0.f;
#pragma unroll
                for (int ks = 0; ks < NK; ++ks) q[b][ks] = q_next[b][ks];
#pragma unroll
                for (int db = 0; db < NB; ++db) acc[b][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        if (left > 1) {
            if (left > 2) after = following(a, o, next), page_next = look_up(after);
            if (next.tile == 0) load_q(next, q_next);
            there[buffer ^ 1] = fetch(next, page, k[buffer ^ 1], buffer ^ 1);
        }

        const uint32_t seen = there[buffer];
        char* const tile = tiles + buffer * kTileBytes;
        if (seen != ~0u) {   // values in places of no key: what is there need not be finite
            for (int i = lane; i < kCacheTile * kChunks; i += 64)
                if (!(seen >> (i / kChunks) & 1)) *reinterpret_cast<u32x4*>(tile + i * 16) = u32x4{0, 0, 0, 0};
            wave_sync();
        }
        const int nearest = now.length - 1 - now.tile * kCacheTile;   // distance of the tile's first key
        u32x4 weights[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            f32x4 s[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < NK; ++ks) s[h] = mma16(T(), k[buffer][h][ks], q[b][ks], s[h]);
            }
            const int my_head = head + min(16 * b + col, columns - 1);
            if (a.bias == nullptr) {
#pragma unroll
                for (int h = 0; h < 2; ++h) s[h] *= c;
            } else if (nearest - (kCacheTile - 1) >= far) {   // all of its keys are as far as the farthest bucket
                const float x = biases.at(my_head, far);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[h][i] = __builtin_fmaf(s[h][i], c, x);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int d = min(max(nearest - (16 * h + 4 * g + i), 0), far);
                        s[h][i] = __builtin_fmaf(s[h][i], c, biases.at(my_head, d));
                    }
            }
            if (seen != ~0u) {
                const uint32_t mine = seen >> (4 * g);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[h][i] = mine >> (16 * h + i) & 1 ? s[h][i] : -INFINITY;
            }
            // Weights are relative to a maximum of earlier keys, and as exact for being up to some hundreds: the maximum of
            // these keys is looked for only where their weights add up to kMost or a head meets its first key.
            auto raise_top = [&](bool mine) {
                float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
                most = over_quarters(most, [](float x, float y) { return fmaxf(x, y); });
                const float to = mine ? fmaxf(top[b], most - kBelow<T>) : top[b];
                const float shrink = to == top[b] ? 1.f : exp2_fast(top[b] - to);
                top[b] = to;
                sum[b] *= shrink;
#pragma unroll
                for (int db = 0; db < NB; ++db) acc[b][db] *= shrink;
            };
            float p[8];
            auto weigh = [&] {   // returns their sum
                const float base = top[b] == -INFINITY ? 0.f : top[b];
                float part = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = exp2_fast(s[i >> 2][i & 3] - base);
                    part += p[i];
                }
                return part;
            };
            if (__any(top[b] == -INFINITY)) raise_top(top[b] == -INFINITY);
            float part = weigh();
            const bool over = !(over_quarters(part, [](float x, float y) { return fmaxf(x, y); }) < kMost<T>);
            if (__any(over)) {
                raise_top(over);
                part = weigh();
            }
            sum[b] += part;
#pragma unroll
            for (int e = 0; e < 4; ++e) weights[b][e] = pack2<T>(p[2 * e], p[2 * e + 1]);
        }
#pragma unroll
        for (int db = 0; db < NB; ++db) {
            typedef short v4i16 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) v4i16* tr_ptr;
            u32x4 x;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 16 * h + tr_row;
                const char* const place = tile + r * kRowBytes + (((2 * db + tr_chunk) ^ Tile<DP>::permuted(r)) * 16) + (col & 1) * 8;
                const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)place));
                x[2 * h] = y[0], x[2 * h + 1] = y[1];
            }
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) acc[b][db] = mma16(T(), x, weights[b], acc[b][db]);
        }

        const bool ends = now.tile + 1 == now.tiles || left == 1;
        if (ends) {
            const bool part = first_tile > 0 || now.tile + 1 < now.tiles;   // of a pair
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const float all = over_quarters(sum[b], [](float x, float y) { return x + y; });
                const int column = 16 * b + col;
                if (column >= columns) continue;
                if (part) {
                    const int64_t at = ((int64_t)wave * 2 + (first_tile > 0 ? 0 : 1)) * o.columns + column;
                    if (g == 0) o.part_ml[2 * at] = top[b], o.part_ml[2 * at + 1] = all;
#pragma unroll
                    for (int db = 0; db < NB; ++db)
                        if (16 * db + 4 * g < a.dim) *reinterpret_cast<f32x4*>(o.part_o + at * a.dim + 16 * db + 4 * g) = acc[b][db];
                } else {
                    const int64_t row = (int64_t)now.seq * a.heads + head + column;
                    if (g == 0) a.lse[row] = (top[b] + log2_fast(all)) * kLn2;
                    const bool none = all == 0.f;   // all that it sees is masked by a bias, or in no page
                    const float scale = none ? 0.f : 1.f / all;
#pragma unroll
                    for (int db = 0; db < NB; ++db)
                        if (16 * db + 4 * g < a.dim)
                            *reinterpret_cast<u32x2*>(static_cast<char*>(a.out) + (row * a.dim + 16 * db + 4 * g) * 2) =
                                none ? u32x2{0, 0}
                                     : u32x2{pack2<T>(acc[b][db][0] * scale, acc[b][db][1] * scale), pack2<T>(acc[b][db][2] * scale, acc[b][db][3] * scale)};
                }
            }
        }
        --left;
        fresh = ends;
        now = next, next = after, page = page_next;
    };
#pragma unroll 1
    while (true) {
        turn(Constant<0>());
        if (left == 0) break;
        turn(Constant<1>());
        if (left == 0) break;
    }
}

// The sums of sequences that several waves share: a workgroup for every wave but the first parts', which works where that
// one's is the first part that begins inside a sequence.  Waves take the maximum and the sum of columns, then threads
// take pairs of elements, and where these are few a share of the parts, always the same ones.
// What bounds it: a launch of mostly idle workgroups (4 us) and a few trips to memory: 15 us for 24 sums of 85 parts, 12 for 512 of
// five.  (A branch around a part's weight keeps loads of several parts from being under way together: 26 and 34 us.)
template <class T>
__global__ __launch_bounds__(kJoinThreads) void cache_attention_join_kernel(CacheAttention a, Share o) {
    constexpr int kWaves = kJoinThreads / 64;
    __shared__ float tops[32], totals[32];
    __shared__ f32x2 sums[kJoinThreads];
    const int w = (int)block_number() + o.units, tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
    if (w >= o.waves) return;
    const int2 note = o.cut[w];
    if (note.x < 0) return;
    const int seq = note.x, parts = note.y, group = a.heads / a.kv_heads;
    const int unit = w % o.units, column0 = unit % o.head_tiles * o.columns, columns = min(o.columns, group - column0);
    // A part's sums: of the wave of the part before w's the second, of w and those behind it the first.
    const int64_t first = ((int64_t)(w - o.units) * 2 + 1) * o.columns, step = 2 * (int64_t)o.units * o.columns;
    auto part_of = [&](int i) { return first + i * step - (i > 0 ? o.columns : 0); };
    for (int column = wave; column < columns; column += kWaves) {
        float top = -INFINITY, total = 0.f;
#pragma unroll 1
        for (int i = lane; i < parts; i += 64) {
            const f32x2 ml = *reinterpret_cast<const f32x2*>(o.part_ml + 2 * (part_of(i) + column));
            if (ml[1] == 0.f) continue;   // (a part that saw nothing has no say)
            const float most = fmaxf(top, ml[0]);
            total = total * (top == most ? 1.f : exp2_fast(top - most)) + ml[1] * (ml[0] == most ? 1.f : exp2_fast(ml[0] - most));
            top = most;
        }
#pragma unroll 1
        for (int m = 1; m < 64; m <<= 1) {
            const float other = __shfl_xor(top, m), other_total = __shfl_xor(total, m), most = fmaxf(top, other);
            total = (total == 0.f ? 0.f : total * (top == most ? 1.f : exp2_fast(top - most))) +
                    (other_total == 0.f ? 0.f : other_total * (other == most ? 1.f : exp2_fast(other - most)));
            top = most;
        }
        if (lane == 0) {
            tops[column] = top, totals[column] = total;
            a.lse[(int64_t)seq * a.heads + unit / o.head_tiles * group + column0 + column] =
                total == 0.f ? -INFINITY : (top + log2_fast(total)) * kLn2;
        }
    }
    __syncthreads();
    const int pairs = columns * (a.dim / 2), shares = max(kJoinThreads / pairs, 1);
    const int share = shares > 1 ? tid / pairs : 0;
#pragma unroll 1
    for (int p = shares > 1 ? tid % pairs : tid; p < pairs && share < shares; p += kJoinThreads) {
        const int column = p / (a.dim / 2), d = 2 * (p - column * (a.dim / 2));
        const float total = totals[column], base = tops[column] == -INFINITY ? 0.f : tops[column];
        f32x2 x = {0.f, 0.f};
#pragma unroll 8   // (no branches: loads of eight parts are under way at a time)
        for (int i = share; i < parts; i += shares) {
            const int64_t at = part_of(i) + column;
            const f32x2 ml = *reinterpret_cast<const f32x2*>(o.part_ml + 2 * at), y = *reinterpret_cast<const f32x2*>(o.part_o + at * a.dim + d);
            const float weight = exp2_fast(ml[0] - base);   // (a part that saw nothing has a maximum of minus infinity)
            x[0] = __builtin_fmaf(weight, y[0], x[0]), x[1] = __builtin_fmaf(weight, y[1], x[1]);
        }
        if (shares > 1) sums[tid] = x;
        else {
            const float scale = total == 0.f ? 0.f : 1.f / total;
            static_cast<uint32_t*>(a.out)[(((int64_t)seq * a.heads + unit / o.head_tiles * group + column0 + column) * a.dim + d) / 2] =
                total == 0.f ? 0u : pack2<T>(x[0] * scale, x[1] * scale);
        }
    }
    if (shares == 1) return;
    __syncthreads();
    if (tid >= pairs) return;
    f32x2 x = sums[tid];
    for (int k = 1; k < shares; ++k) x += sums[tid + k * pairs];
    const int column = tid / (a.dim / 2), d = 2 * (tid - column * (a.dim / 2));
    const float total = totals[column], scale = total == 0.f ? 0.f : 1.f / total;
    static_cast<uint32_t*>(a.out)[(((int64_t)seq * a.heads + unit / o.head_tiles * group + column0 + column) * a.dim + d) / 2] =
        total == 0.f ? 0u : pack2<T>(x[0] * scale, x[1] * scale);
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

int padded_dim(int dim) { return (dim + 31) / 32 * 32; }

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
    const int of_a_unit = lanes_serve(group) ? lanes_waves(group, a.dim) : 4 * waves_of_a_simd(padded_dim(a.dim), group > 16 ? 2 : 1);
    p.o.units = a.kv_heads * p.o.head_tiles;
    const int64_t of_each = (int64_t)n_cu * of_a_unit / p.o.units;
    p.o.waves = (int32_t)(p.o.units * parts_of(most_tiles * a.n_seqs, of_each > 1 ? of_each : 1));
    const size_t waves = (size_t)p.o.waves;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    if (p.o.each > 1) p.entry_bytes = up((size_t)p.o.n_entries * 8);
    if (p.o.cuts) {
        p.cut_bytes = up(waves * sizeof(int2));
        p.o_bytes = up(waves * 2 * p.o.columns * a.dim * 4);
        p.ml_bytes = up(waves * 2 * p.o.columns * 8);
    }
    return p;
}

template <class T, int DP, int BLOCKS>
hipError_t launch(hipStream_t stream, const CacheAttention& a, const Share& o) {
    const int64_t entries = a.bias == nullptr ? 0 : (int64_t)a.heads * (farthest(a) + 1);
    const bool in_table = entries > 0 && entries <= kMostTable;
    const size_t bytes = kThreads / 64 * 2 * kCacheTile * Tile<DP>::kRowBytes + (in_table ? entries * sizeof(float) : 0);
    auto kernel = cache_attention_kernel<T, DP, BLOCKS>;
    if (bytes > 65536) {
        const hipError_t rc = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (rc != hipSuccess) return rc;
    }
    hipLaunchKernelGGL(kernel, grid_of((o.waves + kThreads / 64 - 1) / (kThreads / 64)), dim3(kThreads), bytes, stream, a, o, in_table ? 1 : 0);
    return hipGetLastError();
}
template <class T, int DP>
hipError_t launch_blocks(hipStream_t stream, const CacheAttention& a, const Share& o) {
    return a.heads / a.kv_heads > 16 ? launch<T, DP, 2>(stream, a, o) : launch<T, DP, 1>(stream, a, o);
}

template <class T>
hipError_t launch_type(hipStream_t stream, const CacheAttention& a, const Share& o) {
    hipError_t rc = lanes_serve(a.heads / a.kv_heads) ? launch_lanes<T>(stream, a, o)
                    : a.dim <= 32 ? launch_blocks<T, 32>(stream, a, o)
                    : a.dim <= 64 ? launch_blocks<T, 64>(stream, a, o)
                    : a.dim <= 96 ? launch_blocks<T, 96>(stream, a, o)
                                  : launch_blocks<T, 128>(stream, a, o);
    if (rc != hipSuccess || !o.cuts) return rc;
    hipLaunchKernelGGL(cache_attention_join_kernel<T>, grid_of(max(o.waves - o.units, 1)), dim3(kJoinThreads), 0, stream, a, o);
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
        p.o.cut = reinterpret_cast<int2*>(at);
        p.o.part_o = reinterpret_cast<float*>(at + p.cut_bytes);
        p.o.part_ml = reinterpret_cast<float*>(at + p.cut_bytes + p.o_bytes);
    }
    return half ? launch_type<Fp16>(stream, a, p.o) : launch_type<Bf16>(stream, a, p.o);
}

}  // namespace surel
