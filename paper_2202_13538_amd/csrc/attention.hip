// Attention of packed query rows to packed keys (surel_attention).
#include "attention.h"
#include "kernels.h"

namespace surel {
namespace {

constexpr int kThreads = 256;
constexpr float kSlack = 8.f;    // how far (base 2) scores may rise before weights are made relative to another one, see the kernel
// fp16: weights are relative to 2^-7 of the largest, so that those down to 2^-21 of it keep all their bits, and stay below 2^15;
// bf16 has the range of 32-bit floats.
template <class T>
constexpr float kBelow = T::kNarrow ? 7.f : 0.f;
template <class T>
constexpr float kMost = T::kNarrow ? 32768.f : 1024.f;  // what a lane's weights of a tile may add up to

struct AttentionOut {
    void* out = nullptr;        // [n_q][heads][dim]
    float* lse = nullptr;       // [n_q][heads]
    float* part_o = nullptr;    // splits > 1: [split][n_q][heads][dim], not divided by the sum
    float* part_ml = nullptr;   //             [split][n_q][heads][2]: maximum (base 2), sum
    int splits = 1;
    int pack = 1;               // heads of a group that share a tile
    int across = 0;
    int tiles = 0;              // of rows
};

template <int DP, int WR, int WAVES>
struct ForwardShape {
    static constexpr int WK = WAVES / WR;
    static constexpr int kThreads = 64 * WAVES;
    static constexpr int kKeys = WR > 1 ? 64 : 32;   // keys that a wave takes at a time
    static constexpr int kTileKeys = kKeys * WK;
    static constexpr int kBuffers = 2;
    static constexpr int kTileBytes = kTileKeys * Tile<DP>::kRowBytes;
    static constexpr int kLds = 2 * kBuffers * kTileBytes;
};

// One workgroup: 32 WR rows of queries, a row being a token and one of `pack` heads of a group, against
// the keys that any of them sees.  The keys stream through LDS, 64 at a time; a wave holds its 32 query
// rows in registers and computes scores^T = K q^T, so that a row's scores lie in one lane and its partner, the
// softmax runs inside lanes, and the weights are the operand of out^T += V^T p^T as they come.
//   WR = 4: four waves, 128 rows, all waves take every key tile.
//   WR = 1: 32 rows (single tokens, a pooling row a set); four waves take different keys of a tile of 128
//           and join their sums at the end, or one wave takes all (WAVES = 1): a quarter of the LDS and no barrier
//           between waves, so that more tiles of a compute unit have loads in flight (see forward_plan).
// What bounds it: with 128 rows the matrix units, and beside them the seven vector instructions a score (16,384 causal rows of
// 16 heads of 128 elements 1.07 ms, 1.03 PFLOP/s of the 1.12 of a large product; 5 causal sequences of 333 to 4,096 rows
// with a bias 0.21 ms); over walks of 16 steps, memory (16,384 of them with 8 heads of 64 elements 0.25 ms, 4.3 TB/s).
// With 32 rows, memory: 8,192 pooling rows over up to 1,602 keys 0.60 ms, 5.6 TB/s, nearly all of it read.
// (A pooling row fills one of a wave's 32 columns a head; the other columns' products cost nothing that shows.)
template <class T, int DP, int WR, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP > 64 ? 2 : DP > 32 ? 3 : 4) void attention_kernel(AttentionArgs a, AttentionOut o) {
    using Shape = ForwardShape<DP, WR, WAVES>;
    constexpr int WK = Shape::WK, kThreads = Shape::kThreads, kBlocks = Shape::kKeys / 32, NB = DP / 32;
    extern __shared__ __align__(16) char lds[];
    __shared__ int range[2][4];
    char* const k_tile = lds;
    char* const v_tile = lds + Shape::kBuffers * Shape::kTileBytes;
    float* const bias = reinterpret_cast<float*>(lds + Shape::kLds);

    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, g = lane >> 5, col = lane & 31;
    const int wr = WR == 1 ? 0 : wave, wk = WR == 1 ? wave : 0;
    const int n_head_tiles = a.heads / o.pack;
    uint32_t block = block_number();
    if (block == 0 && tid == 0) check_ends(a);
    const int head0 = block % n_head_tiles * o.pack;
    block /= n_head_tiles;
    const int split = block % o.splits;
    block /= o.splits;
    if (block >= (uint32_t)o.tiles) return;
    // a causal sequence's last rows see the most keys: they come first
    const int tile_no = a.causal ? o.tiles - 1 - (int)block : (int)block;
    const int tokens = 32 * WR / o.pack;
    const TileOfRows tile = tile_of_rows(a.q_off, a.n_seqs, a.n_q, tokens, o.across, tile_no);
    if (tile.first >= tile.last) return;

    // the lane's row, and the keys that it sees: lo <= key < hi; `diag` is the key that it stands at
    const int row = 32 * wr + col;
    const int token = tile.first + row / o.pack, head = head0 + row % o.pack;
    const bool counts = token < tile.last && row < tokens * o.pack;
    Stationary<DP> q;
    q.load(a.q + (int64_t)token * a.q_row + (int64_t)head * a.q_head, counts, a.dim, lane);
    int lo = 0, hi = 0x7FFFFFFF, diag = 0;
    if (counts) {
        const int s = tile.seq >= 0 ? tile.seq : segment_of(a.q_off, a.n_seqs, a.n_q, token);
        const Sequence seq = sequence_at(a, s);
        diag = seq.k1 - (seq.q1 - token);
        lo = seq.k0;
        hi = a.causal ? min(seq.k1, diag + 1) : seq.k1;
        if (hi <= lo || token < seq.q0 || token >= seq.q1) lo = hi = 0;
    }
    const bool sees = counts && hi > lo;
    const int wave_lo = wave_min(sees ? lo : 0x7FFFFFFF), wave_hi = wave_max(sees ? hi : 0);
    const int all_lo = wave_max(lo), all_hi = wave_min(hi);   // every row sees what lies between
    const int diag_min = wave_min(counts ? diag : 0x7FFFFFFF), diag_max = wave_max(counts ? diag : -0x3FFFFFFF);
    if (!counts) diag = diag_min;
    int tile_lo = wave_lo, tile_hi = wave_hi;
    if (WR > 1) {
        if (lane == 0) range[0][wave] = wave_lo, range[1][wave] = wave_hi;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) tile_lo = min(tile_lo, range[0][w]), tile_hi = max(tile_hi, range[1][w]);
    }
    int key_begin = tile_lo, key_end = tile_hi;
    if (o.splits > 1 && tile_hi > tile_lo) {
        const int n = (tile_hi - tile_lo + Shape::kTileKeys - 1) / Shape::kTileKeys;
        const int each = (n + o.splits - 1) / o.splits * Shape::kTileKeys;
        key_begin = (int)min((int64_t)tile_lo + (int64_t)split * each, (int64_t)tile_hi);
        key_end = (int)min((int64_t)key_begin + each, (int64_t)tile_hi);
    }

    const float c = a.scale * kLog2e;   // scores in units of log 2
    const int width = bias_width(a.reach);
    if (a.bias != nullptr)
        for (int p = 0; p < o.pack; ++p) fill_bias<T>(bias + p * width, a, head0 + p, tid, kThreads);
    const float* const my_bias = bias + (row % o.pack) * width;
    __syncthreads();
    float bias_behind = 0.f, bias_ahead = 0.f;
    if (a.bias != nullptr) bias_behind = my_bias[0], bias_ahead = my_bias[width - 1];

    const int kv_head = head0 / (a.heads / a.kv_heads);
    const char* const k_src = a.k + (int64_t)kv_head * a.k_head;
    const char* const v_src = a.v + (int64_t)kv_head * a.v_head;
    f32x16 acc[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db) acc[db] = f32x16{};
    float top = sees ? -INFINITY : 0.f, sum = 0.f;   // what weights are taken relative to (base 2), and their sum

    auto fetch = [&](int key, int buffer) {
        const int rows = key_end - key;
        copy_tile<DP, Shape::kTileKeys, kThreads>(k_tile + buffer * Shape::kTileBytes, k_src + (int64_t)key * a.k_row,
                                                  a.k_row, rows, a.dim, tid);
        copy_tile<DP, Shape::kTileKeys, kThreads>(v_tile + buffer * Shape::kTileBytes, v_src + (int64_t)key * a.v_row,
                                                  a.v_row, rows, a.dim, tid);
    };
    auto raise_top = [&](float most, bool mine) {
        const float now = mine ? fmaxf(top, most - kBelow<T>) : top;
        const float shrink = now == top ? 1.f : exp2_fast(top - now);
        top = now;
        sum *= shrink;
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] *= shrink;
    };
    auto bias_at = [&](int key) {
        return a.bias == nullptr ? 0.f : my_bias[min(max(key - diag, -a.reach), a.reach) + a.reach + kBeyond];
    };

    if (key_begin < key_end) fetch(key_begin, 0);
    tile_arrived();
    __syncthreads();
    const int last = min(hi, key_end);
    alternate(key_begin, key_end, Shape::kTileKeys, [&](int key, auto of) __attribute__((always_inline)) {
        constexpr int buffer = decltype(of)::value;
        if (key + Shape::kTileKeys < key_end) fetch(key + Shape::kTileKeys, buffer ^ 1);
        const int key0 = key + wk * Shape::kKeys;
        if (key0 < min(wave_hi, key_end) && key0 + Shape::kKeys > wave_lo) {
            const uint32_t kt = buffer * Shape::kTileBytes + wk * Shape::kKeys * Tile<DP>::kRowBytes;
            const uint32_t vt = kt + Shape::kBuffers * Shape::kTileBytes;
            f32x16 s[kBlocks];
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) s[b] = scores<T, DP>(lds, kt + 32 * b * Tile<DP>::kRowBytes, q, lane);
            const bool whole = key0 >= all_lo && key0 + Shape::kKeys <= min(all_hi, key_end);
            const bool behind = key0 + Shape::kKeys - 1 - diag_min <= -a.reach, ahead = key0 - diag_max >= a.reach;
            const bool plain = whole && (a.bias == nullptr || behind || ahead);
            const float far = behind ? bias_behind : bias_ahead;
            if (!plain) {   // scores, in units of log 2, of what the row sees
                if (a.bias != nullptr) {
                    const float* const from = bias_from(my_bias, a.reach, key0 + 4 * g - diag);
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[b][i] = __builtin_fmaf(s[b][i], c, from[32 * b + row_of(i, 0)]);
                } else {
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b) s[b] *= c;
                }
                if (!whole) {
                    const uint32_t first = key0 + 4 * g - lo, span = max(last - lo, 0);
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            s[b][i] = first + (32 * b + row_of(i, 0)) < span ? s[b][i] : -INFINITY;
                }
            }
            // Weights relative to a maximum of earlier keys: 32-bit sums and 16-bit floats are as exact
            // for weights of some hundreds as for those below one, so that most tiles need no rescaling.  With few
            // scores in registers the maximum of these keys is looked for only where their weights add up to kMost or
            // a row meets its first key (two of seven instructions a score less, 8,192 pooling rows 0.84 -> 0.76 ms);
            // with 32 of them there is no room to keep scores beside weights, and it is always looked for (1.15 against
            // 1.18 ms for 16,384 causal rows).  Either is a row's own affair: no other row's result depends on it.
            const float times = plain ? c : 1.f, plus = plain ? far : 0.f;
            auto largest = [&] {
                float most = s[0][0];
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most = fmaxf(most, s[b][i]);
                most = __builtin_fmaf(most, times, plus);
                return fmaxf(most, from_other_half(most));
            };
            auto weights = [&](f32x16 (&p)[kBlocks]) {   // returns their sum
                const float less = plus - (top == -INFINITY ? 0.f : top);
                float part = 0.f;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        p[b][i] = exp2_fast(__builtin_fmaf(s[b][i], times, less));
                        part += p[b][i];
                    }
                return part;
            };
            if constexpr (kBlocks > 1) {
                const float most = largest();
                const bool over = most > top + (kSlack + kBelow<T>);
                if (__any(over)) raise_top(most, over);
                sum += weights(s);
            } else {
                if (__any(top == -INFINITY)) raise_top(largest(), top == -INFINITY);
                f32x16 p[kBlocks];
                float part = weights(p);
                const bool over = !(fmaxf(part, from_other_half(part)) < kMost<T>);
                if (__any(over)) {
                    raise_top(largest(), over);
                    part = weights(p);
                }
                sum += part;
                s[0] = p[0];
            }
            // (weights are rounded to the inputs' 16 bits for the second product, the sum is of the
            // unrounded ones)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) accumulate<T, DP>(acc, lds, vt + 32 * b * Tile<DP>::kRowBytes, s[b], lane);
        }
        tile_arrived();
        __syncthreads();
    });
    sum += from_other_half(sum);
    // The wave's keys once more, without what a row does not see: for rows whose own scores are numbers.  (Where those are not, no
    // result is; but of heads that do not fill a tile's rows, what lies beyond them repeats their start, and 0 times infinity is none.)
    if (__any(sees && has_nan(acc) && (sum == sum || a.dim != DP))) {
        const float first_top = top, first_sum = sum;   // right whatever values are, if they are numbers
#pragma unroll
        for (int db = 0; db < NB; ++db) acc[db] = f32x16{};
        top = sees ? -INFINITY : 0.f;
        sum = 0.f;
#pragma unroll 1
        for (int j = max(key_begin, wave_lo); j < min(key_end, wave_hi); ++j) {
            if (WK > 1 && (j - key_begin) / Shape::kKeys % WK != wk) continue;   // (another wave's, which may keep its sums)
            const float dot = dot_row<T, DP>(q, k_src + (int64_t)j * a.k_row, a.dim, lane);
            const bool seen = j >= lo && j < last;
            const float x = seen ? __builtin_fmaf(dot, c, bias_at(j)) : -INFINITY;
            raise_top(x, true);
            if (seen) {
                const float w = exp2_fast(x - (top == -INFINITY ? 0.f : top));
                sum += w;
                accumulate_row<T, DP>(acc, v_src + (int64_t)j * a.v_row, w, a.dim, g);
            }
            if ((j & 15) == 15 && __all(!sees || sum != sum || (first_sum == first_sum && all_nan(acc)))) {
                top = first_top, sum = first_sum;
                break;
            }
        }
    }

    if (WK > 1) {   // the waves' sums: 2 and 3 to 0 and 1, then 1 to 0
        float* const ml = reinterpret_cast<float*>(lds);            // [2][64]
        float* const sums = ml + 2 * 64;                            // [2][NB * 16][64]
#pragma unroll 1
        for (int half = 2; half >= 1; half >>= 1) {
            if (wave >= half && wave < 2 * half) {
                const int at = wave - half;
                if (g == 0) ml[at * 64 + col] = top, ml[at * 64 + 32 + col] = sum;
#pragma unroll
                for (int db = 0; db < NB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sums[(at * NB * 16 + db * 16 + i) * 64 + lane] = acc[db][i];
            }
            __syncthreads();
            if (wave < half) {
                const float other = ml[wave * 64 + col], other_sum = ml[wave * 64 + 32 + col];
                const float now = fmaxf(top, other), base = now == -INFINITY ? 0.f : now;
                const float mine = now == top ? 1.f : exp2_fast(top - base);
                const float theirs = now == other ? 1.f : exp2_fast(other - base);
                top = now;
                sum = sum * mine + other_sum * theirs;
#pragma unroll
                for (int db = 0; db < NB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        acc[db][i] = acc[db][i] * mine + sums[(wave * NB * 16 + db * 16 + i) * 64 + lane] * theirs;
            }
            __syncthreads();
        }
        if (wave != 0) return;
    }

    const int64_t at = (int64_t)token * a.heads + head;
    if (o.splits > 1) {
        if (!counts) return;
        const int64_t part = (int64_t)split * a.n_q * a.heads + at;
        if (g == 0) o.part_ml[2 * part] = top, o.part_ml[2 * part + 1] = sum;
        float* const dst = o.part_o + part * a.dim;
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * db + row_of(i, g);
                if (d < a.dim)   // dim is a multiple of 8, d of 4
                    *reinterpret_cast<f32x4*>(dst + d) = f32x4{acc[db][i], acc[db][i + 1], acc[db][i + 2], acc[db][i + 3]};
            }
        return;
    }
    if (counts && g == 0) o.lse[at] = sees ? (top + log2_fast(sum)) * kLn2 : -INFINITY;
    const bool none = !sees || sum == 0.f;   // (or all that it sees is masked by a bias)
    const float scale = none ? 0.f : 1.f / sum;
    store_rows<T, DP>(acc, scale, none, lds + wr * 32 * Tile<DP>::kRowBytes, a.dim, lane, [&](int r) -> char* {
        const int row_there = 32 * wr + r, token_there = tile.first + row_there / o.pack;
        if (token_there >= tile.last || row_there >= tokens * o.pack) return nullptr;
        return static_cast<char*>(o.out) + ((int64_t)token_there * a.heads + head0 + row_there % o.pack) * a.dim * 2;
    });
}

// One wave a row: the parts of a row whose keys went to several workgroups (128 at most, two a lane).  A launch
// and a few trips to memory: 192 rows of 22 parts of 128 elements 8 us.
template <class T>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(AttentionOut o, int64_t n_rows, int dim) {
    const int64_t row = (int64_t)block_number() * (kThreads / 64) + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= n_rows) return;
    float m[2], l[2], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int s = lane + 64 * e;
        const float2 x = s < o.splits ? reinterpret_cast<const float2*>(o.part_ml)[s * n_rows + row] : float2{-INFINITY, 0.f};
        m[e] = x.x, l[e] = x.y;
        if (l[e] != 0.f) top = fmaxf(top, m[e]);   // (a part that saw nothing has no say)
    }
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        m[e] = l[e] == 0.f ? 0.f : m[e] == top ? 1.f : exp2_fast(m[e] - base);   // the part's weight
        sum += m[e] * l[e];
    }
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
    f32x2 x = {0.f, 0.f};
    const bool mine = 2 * lane < dim;
#pragma unroll 8
    for (int s = 0; s < o.splits; ++s) {
        const float w = __shfl(s < 64 ? m[0] : m[1], s & 63);
        const f32x2 y = mine ? *reinterpret_cast<const f32x2*>(&o.part_o[(s * n_rows + row) * dim + 2 * lane]) : f32x2{0.f, 0.f};
        if (w != 0.f) x[0] = __builtin_fmaf(w, y[0], x[0]), x[1] = __builtin_fmaf(w, y[1], x[1]);
    }
    // (a sum of zero: the row sees no key at all)
    if (lane == 0) o.lse[row] = sum == 0.f ? -INFINITY : (top + log2_fast(sum)) * kLn2;
    const float scale = sum == 0.f ? 0.f : 1.f / sum;
    if (mine) static_cast<uint32_t*>(o.out)[row * (dim / 2) + lane] = pack2<T>(x[0] * scale, x[1] * scale);
}

struct ForwardPlan {
    int rows = 128, pack = 1, splits = 1, waves = 4;
    bool across = false;
    int64_t tiles = 0;
};

// How rows are put into tiles, and whether keys are split over workgroups, from the means of the lengths
// (which are all that the host knows).
ForwardPlan forward_plan(const AttentionArgs& a, int n_cu) {
    ForwardPlan p;
    const int group = a.heads / a.kv_heads;
    const double mean_q = (double)a.n_q / a.n_seqs, mean_k = (double)a.n_k / a.n_seqs;
    // the bias of every head of a tile lies in LDS: 24 KB of it at most
    auto fits = [&](int pack) { return a.bias == nullptr || pack == 1 || (int64_t)pack * bias_width(a.reach) * 4 <= 24576; };
    // Tiles across sequences where these are short and alike (8,192 walks of 17
    // nodes 157 us against 269, 2,048 sequences of up to 80 rows 110 against 207, of 120 rows 147 against 152).  With a
    // bias the rows of a tile have to stand at neighbouring keys, which those of several sequences do only where
    // queries and keys lie alike.
    p.across = mean_q < 128 && mean_k <= 256 && mean_k <= 2 * mean_q && (a.bias == nullptr || a.q_off == a.k_off);
    if (!p.across) {
        for (int d = 1; d <= group && d <= 32; ++d)
            if (group % d == 0 && fits(d) && mean_q * d <= 32) p.rows = 32, p.pack = d;
        if (p.rows == 128)
            for (int d = group; d >= 1; --d)
                if (group % d == 0 && d <= 128 && fits(d) && (mean_q * d >= 128 || p.pack == 1 || d > p.pack)) p.pack = d;
    }
    const int64_t heads = a.heads / p.pack;
    p.tiles = tiles_of_rows(a.n_seqs, a.n_q, p.rows / p.pack, p.across);
    const double full = p.across ? (double)p.tiles : a.n_seqs * ceil(mean_q * p.pack / p.rows);
    const double blocks = full * heads;
    // 32 rows: one wave a tile where there are enough of these, or of their keys, to keep loads in flight; four, which take
    // four times the LDS, where a tile's own keys have to be shared for that.  Four against one, in us: 32,768 tiles
    // of 64 elements over 16 keys each 449 / 97, over 200 680 / 330, over 800 1,472 / 1,309, 2,048 of them over 2,000 239 / 262;
    // 128 of 128 elements over 2,000 40 / 31, over 200 14.7 / 19.1; 32 over 500 14.5 / 21.9, over 32,768 119 / 105.  Of up to
    // 64 elements in few tiles (8 over 100,000 keys 58 / 62) two workgroups of four waves fit a compute unit.
    if (p.rows == 32 && ((blocks >= 2 * n_cu && mean_k <= 1024) || (a.dim > 64 && blocks * mean_k >= 256.0 * n_cu))) p.waves = 1;
    // Keys are split where tiles do not fill the device, into parts of 256 at least, since a row's parts are
    // written and joined: 32 tiles over 32,768 keys 542 us in one part, 119 in 16; four times the parts 129.
    if (blocks < 2 * n_cu) {
        const double most = mean_k / 256;
        p.splits = (int)fmax(1.0, fmin(fmin(ceil(2.0 * n_cu / blocks), most), 128.0));
    }
    return p;
}

int64_t blocks_of(const AttentionArgs& a, const ForwardPlan& p) { return p.tiles * (a.heads / p.pack) * p.splits; }

template <class T, int DP, int WR, int WAVES>
hipError_t launch(hipStream_t stream, const AttentionArgs& a, const AttentionOut& o, int64_t blocks) {
    const size_t bytes = ForwardShape<DP, WR, WAVES>::kLds +
                         (a.bias != nullptr ? (size_t)o.pack * bias_width(a.reach) * sizeof(float) : 0);
    auto kernel = attention_kernel<T, DP, WR, WAVES>;
    if (bytes > 65536) {
        const hipError_t rc = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                  hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (rc != hipSuccess) return rc;
    }
    hipLaunchKernelGGL(kernel, grid_of(blocks), dim3(64 * WAVES), bytes, stream, a, o);
    return hipGetLastError();
}

template <class T, int DP>
hipError_t launch_rows(hipStream_t stream, const AttentionArgs& a, const AttentionOut& o, const ForwardPlan& p, int64_t blocks) {
    return p.rows == 128 ? launch<T, DP, 4, 4>(stream, a, o, blocks)
           : p.waves == 4 ? launch<T, DP, 1, 4>(stream, a, o, blocks)
                          : launch<T, DP, 1, 1>(stream, a, o, blocks);
}

template <class T>
hipError_t launch_type(hipStream_t stream, const AttentionArgs& a, const AttentionOut& o, const ForwardPlan& p) {
    const int64_t blocks = blocks_of(a, p);
    if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
    hipError_t rc = a.dim <= 32   ? launch_rows<T, 32>(stream, a, o, p, blocks)
                    : a.dim <= 64 ? launch_rows<T, 64>(stream, a, o, p, blocks)
                    : a.dim <= 96 ? launch_rows<T, 96>(stream, a, o, p, blocks)
                                  : launch_rows<T, 128>(stream, a, o, p, blocks);
    if (rc != hipSuccess || p.splits == 1) return rc;
    const int64_t n_rows = (int64_t)a.n_q * a.heads;
    hipLaunchKernelGGL(attention_join_kernel<T>, grid_of((n_rows + 3) / 4), dim3(kThreads), 0, stream, o, n_rows, a.dim);
    return hipGetLastError();
}

}  // namespace

size_t attention_scratch_bytes(int n_cu, const AttentionArgs& a) {
    const ForwardPlan p = forward_plan(a, n_cu);
    return p.splits == 1 ? 0 : (size_t)p.splits * a.n_q * a.heads * (a.dim + 2) * sizeof(float);
}

int64_t attention_blocks(int n_cu, const AttentionArgs& a) { return blocks_of(a, forward_plan(a, n_cu)); }

hipError_t launch_attention(hipStream_t stream, int n_cu, const AttentionArgs& a, bool half, void* out, float* lse,
                            void* scratch) {
    const ForwardPlan p = forward_plan(a, n_cu);
    AttentionOut o;
    o.out = out;
    o.lse = lse;
    o.splits = p.splits;
    o.pack = p.pack;
    o.across = p.across;
    o.tiles = (int)p.tiles;
    if (p.splits > 1) {
        o.part_o = static_cast<float*>(scratch);
        o.part_ml = o.part_o + (int64_t)p.splits * a.n_q * a.heads * a.dim;
    }
    return half ? launch_type<Fp16>(stream, a, o, p) : launch_type<Bf16>(stream, a, o, p);
}

}  // namespace surel
