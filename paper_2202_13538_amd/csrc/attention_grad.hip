// The gradients of attention (surel_attention_grad).
//
// With the weights p_ij = exp(s_ij - lse_i) of the forward pass, dp_ij = do_i . v_j and delta_i = do_i . o_i:
//   dv_j = sum_i p_ij do_i        ds_ij = p_ij (dp_ij - delta_i)
//   dq_i = scale sum_j ds_ij k_j  dk_j = scale sum_i ds_ij q_i   dbias_b = sum of ds_ij with distance in bucket b
// Scores are made again from q and k.  Two kernels: one goes over the keys of a tile of query rows (dq), one
// over the query rows of a tile of keys (dk, dv, dbias).  Each sum then lives in one workgroup's registers and is
// the same every time; that costs the scores and dp a second time (7 products instead of 5), where one
// kernel would add dq up in memory with atomics in whatever order its workgroups run.
#include "attention.h"
#include "kernels.h"

namespace surel {
namespace {

constexpr int kThreads = 256;
constexpr int kTileRows = 64;      // streamed rows of a tile
constexpr int kRowBlocks = 1024;   // workgroups of attention_grad_rows_kernel, at most
constexpr int kDiagonals = 48;     // distances between 16 query rows and 32 keys (47), a row of LDS
constexpr int kMaxReach = 1024;    // SUREL_MAX_REACH

struct GradArgs {
    const char *dout = nullptr, *out = nullptr;  // [n_q][heads][dim]
    const float* lse = nullptr;                  // [n_q][heads]
    char *dq = nullptr, *dk = nullptr, *dv = nullptr;
    void* dbias = nullptr;
    float *lse2 = nullptr, *delta = nullptr;  // [heads][n_q]: lse in units of log 2
    float* dout_size = nullptr;               // [heads][n_q]: lengths of dout's rows (fp16 only)
    float* v_size = nullptr;                  // [kv_heads][n_k]: of values (fp16 only, unless `twice`)
    float* by_distance = nullptr;             // [heads][tiles][2 reach + 1]: ds of a tile of keys
    int q_tiles = 0, k_tiles = 0;
    int across_q = 0, across_k = 0;
    int twice = 0;                            // delta from the weights themselves, see attention_dq_kernel
};

__global__ __launch_bounds__(kThreads) void zero_kernel(uint16_t* dst, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) dst[i] = 0;
}

// The sum of eight fp16's squares.  (By dot products of packed pairs: unpacked ones would stay in registers until the
// second look of the kernels below, which unpacks them too.  They may take subnormal numbers for zeros: lengths get
// what 128 of those have at most, 2^-10.5, and a little more.)
constexpr float kUnder = 0x1p-10f;
__device__ __forceinline__ float square_of(const u32x4& x) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const Fp16::x2 p = __builtin_bit_cast(Fp16::x2, x[e]);
        sum = __builtin_amdgcn_fdot2(p, p, sum, false);
    }
    return sum;
}

// (a row that sees nothing, or nothing that its bias does not mask: all of its weights become zero)
__device__ __forceinline__ float in_log2(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// delta and lse by head, so that a tile's 64 rows lie behind one another, and for fp16 the lengths of values.  16 lanes a
// row and head, four of these at a time.
template <class T>
__global__ __launch_bounds__(kThreads) void attention_grad_rows_kernel(AttentionArgs a, GradArgs w) {
    constexpr int kEach = 4, kRows = kThreads / 16;
    const int64_t n_rows = (int64_t)a.n_q * a.heads;
    const int c = threadIdx.x & 15;
    for (int64_t first = (int64_t)blockIdx.x * kRows * kEach; first < n_rows; first += (int64_t)gridDim.x * kRows * kEach) {
        u32x4 x[kEach], y[kEach];
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            const int64_t row = first + n * kRows + (threadIdx.x >> 4);
            x[n] = y[n] = u32x4{0, 0, 0, 0};
            if (row < n_rows && c * 8 < a.dim) {
                x[n] = *reinterpret_cast<const u32x4*>(w.dout + (row * a.dim + c * 8) * 2);
                y[n] = *reinterpret_cast<const u32x4*>(w.out + (row * a.dim + c * 8) * 2);
            }
        }
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            const int64_t row = first + n * kRows + (threadIdx.x >> 4);
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x2 p = unpack2<T>(x[n][e]), q = unpack2<T>(y[n][e]);
                sum = __builtin_fmaf(p[0], q[0], __builtin_fmaf(p[1], q[1], sum));
            }
#pragma unroll
            for (int m = 1; m < 16; m <<= 1) sum += __shfl_xor(sum, m);
            if (row < n_rows && c == 0) {
                const int64_t at = (row % a.heads) * a.n_q + row / a.heads;
                w.delta[at] = sum;
                w.lse2[at] = in_log2(w.lse[row]);
            }
        }
    }
    if (!T::kNarrow) return;
    const int64_t n_values = (int64_t)a.n_k * a.kv_heads;
    for (int64_t row = (int64_t)blockIdx.x * kRows + (threadIdx.x >> 4); row < n_values; row += (int64_t)gridDim.x * kRows) {
        const int64_t key = row / a.kv_heads, head = row % a.kv_heads;
        u32x4 x = {0, 0, 0, 0};
        if (c * 8 < a.dim) x = *reinterpret_cast<const u32x4*>(a.v + key * a.v_row + head * a.v_head + c * 16);
        float sum = square_of(x);
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) sum += __shfl_xor(sum, m);
        if (c == 0) w.v_size[head * a.n_k + key] = sqrtf(sum) + kUnder;
    }
}

// fp16 only.  What ds is multiplied by before it is rounded is a power of two of each query row (for dq) or key (for dk): it
// brings a bound of the largest |ds| that the row or key can meet to 2^14 .. 2^15.  So nothing overflows, whatever values and
// gradients are; rounded away is 2^-39 of the bound.  |ds_ij| = p |dp_ij - delta_i| is at most |dp_ij| + |delta_i|, and
// |dp_ij| at most the length of do_i times that of v_j.  What is not finite has no say: who sees it is not finite anyway.
// bf16 has the range of 32-bit floats.
__device__ __forceinline__ int lift_for(float bound) {
    return bound > 0.f && bound < INFINITY ? min(max(14 - ilogbf(bound), -60), 60) : 0;
}
__device__ __forceinline__ float finite_or_zero(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }
// The largest of all threads of a workgroup; `scratch` holds 4 words of LDS of this call's own.
__device__ __forceinline__ float largest_of_all(float x, float* scratch, int tid) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x = fmaxf(x, __shfl_xor(x, m));
    if ((tid & 63) == 0) scratch[tid >> 6] = x;
    __syncthreads();
    return fmaxf(fmaxf(scratch[0], scratch[1]), fmaxf(scratch[2], scratch[3]));
}
// The length of a lane's row (of fp16).
template <int DP>
__device__ __forceinline__ float size_of(const Stationary<DP>& row) {
    float sum = 0.f;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) sum += square_of(row.k[ks]);
    return sqrtf(sum + from_other_half(sum)) + kUnder;
}

// The product of two rows in memory, by a lane and its partner.
template <class T>
__device__ __forceinline__ float dot_of_rows(const char* x, const char* y, int dim, int g) {
    float sum = 0.f;
#pragma unroll 1
    for (int c = g; c * 8 < dim; c += 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f32x2 p = unpack2<T>(reinterpret_cast<const uint32_t*>(x + c * 16)[e]);
            const f32x2 q = unpack2<T>(reinterpret_cast<const uint32_t*>(y + c * 16)[e]);
            sum = __builtin_fmaf(p[0], q[0], __builtin_fmaf(p[1], q[1], sum));
        }
    return sum + from_other_half(sum);
}

// dq of 128 query rows of one head, 32 a wave.
//
// delta_i = do_i . o_i comes from an o whose weights and results were rounded to 16 bits.  The sum of ds_ij over j
// is what it is off by, since it should be zero; the row's delta in memory is corrected by that for dk and dbias.  dq
// itself would need the keys' weighted sum as a fourth product.  With few keys a row the error is as
// large as that of rounding ds, and the keys are there again at once: their ds are summed up in a round of
// its own first (`twice`; walks of 16 steps, 262,144 rows of 8 heads of 64 elements: dq 0.0029 -> 0.0024 off).
//
// What bounds it: over walks, memory, keys and values once a round (16,384 walks of 16 steps with 8 heads of 64 elements
// 0.36 ms); else vector instructions between three products a tile, at two waves a SIMD (5 causal sequences of 333 to
// 4,096 rows with 16 heads of 128 elements 0.29 ms, 24 of up to 2,048 with 12 heads of 80 elements 0.27).  Turns
// unrolled over buffers, which gains elsewhere, lose here (378 -> 422 us with two rounds).
template <class T, int DP>
__global__ __launch_bounds__(kThreads, DP > 64 ? 2 : DP > 32 ? 3 : 4) void attention_dq_kernel(AttentionArgs a, GradArgs w) {
    constexpr int NB = DP / 32, kTileBytes = kTileRows * Tile<DP>::kRowBytes;
    extern __shared__ __align__(16) char lds[];
    __shared__ int range[2][4];
    __shared__ float maxima[4];
    char* const k_tile = lds;
    char* const v_tile = lds + 2 * kTileBytes;
    float* const bias = reinterpret_cast<float*>(lds + 4 * kTileBytes);
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, g = lane >> 5, col = lane & 31;

    const uint32_t number = block_number();
    const int head = number % a.heads, block = number / a.heads, tile_no = a.causal ? w.q_tiles - 1 - block : block;
    if (number == 0 && tid == 0) check_ends(a);
    if (block >= w.q_tiles) return;
    const TileOfRows tile = tile_of_rows(a.q_off, a.n_seqs, a.n_q, 128, w.across_q, tile_no);
    if (tile.first >= tile.last) return;
    const int token = tile.first + 32 * wave + col;
    const bool counts = token < tile.last;
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
    const int all_lo = wave_max(lo), all_hi = wave_min(hi);
    const int diag_min = wave_min(counts ? diag : 0x7FFFFFFF), diag_max = wave_max(counts ? diag : -0x3FFFFFFF);
    if (!counts) diag = diag_min;
    if (lane == 0) range[0][wave] = wave_lo, range[1][wave] = wave_hi;
    if (a.bias != nullptr) fill_bias<T>(bias, a, head, tid, kThreads);
    __syncthreads();
    int key_begin = 0x7FFFFFFF, key_end = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) key_begin = min(key_begin, range[0][i]), key_end = max(key_end, range[1][i]);

    Stationary<DP> q, dout;
    q.load(a.q + (int64_t)token * a.q_row + (int64_t)head * a.q_head, counts, a.dim, lane);
    const int64_t row_bytes = ((int64_t)token * a.heads + head) * a.dim * 2;
    dout.load(w.dout + row_bytes, counts, a.dim, lane);
    const int64_t by_head = (int64_t)head * a.n_q + token;
    float lse2 = 0.f, delta = 0.f;
    if (counts) {
        if (w.twice) lse2 = in_log2(w.lse[(int64_t)token * a.heads + head]);
        else lse2 = w.lse2[by_head], delta = w.delta[by_head];
    }
    const float c = a.scale * kLog2e;
    int lift = 0;
    float base = lse2, most = 0.f;   // base: less the lift, with which ds then comes out; most: |ds| and delta's share of it
    if (T::kNarrow) {
        const float size = size_of(dout);
        if (counts && g == 0) w.dout_size[by_head] = size;
        if (!w.twice) {
            const float* const sizes = w.v_size + (int64_t)(head / (a.heads / a.kv_heads)) * a.n_k;
            for (int i = tid; i < key_end - key_begin; i += kThreads) most = fmaxf(most, finite_or_zero(sizes[key_begin + i]));
            most = size * largest_of_all(most, maxima, tid);
        }
    }
    float bias_behind = 0.f, bias_ahead = 0.f;
    if (a.bias != nullptr) bias_behind = bias[0], bias_ahead = bias[bias_width(a.reach) - 1];

    const int kv_head = head / (a.heads / a.kv_heads);
    const char* const k_src = a.k + (int64_t)kv_head * a.k_head;
    const char* const v_src = a.v + (int64_t)kv_head * a.v_head;
    auto fetch = [&](int key, int buffer) {
        const int rows = key_end - key;
        copy_tile<DP, kTileRows, kThreads>(k_tile + buffer * kTileBytes, k_src + (int64_t)key * a.k_row, a.k_row, rows, a.dim, tid);
        copy_tile<DP, kTileRows, kThreads>(v_tile + buffer * kTileBytes, v_src + (int64_t)key * a.v_row, a.v_row, rows, a.dim, tid);
    };
    auto bias_at = [&](int key) { return a.bias == nullptr ? 0.f : bias[min(max(key - diag, -a.reach), a.reach) + a.reach + kBeyond]; };

    f32x16 acc[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db) acc[db] = f32x16{};
    float sum = 0.f;   // of ds
#pragma unroll 1
    for (int round = w.twice ? 0 : 1; round < 2; ++round) {
        if (T::kNarrow && round == 1) {
            lift = lift_for(fmaxf(most, from_other_half(most)) + fabsf(delta));
            base = lse2 - (float)lift;
        }
        if (key_begin < key_end) fetch(key_begin, 0);
        tile_arrived();
        __syncthreads();
        int buffer = 0;
#pragma unroll 1
        for (int key = key_begin; key < key_end; key += kTileRows, buffer ^= 1) {
            if (key + kTileRows < key_end) fetch(key + kTileRows, buffer ^ 1);
#pragma unroll
            for (int b = 0; b < kTileRows; b += 32) {
                const int key0 = key + b;
                if (key0 >= wave_hi || key0 + 32 <= wave_lo) continue;
                const uint32_t kt = buffer * kTileBytes + b * Tile<DP>::kRowBytes, vt = kt + 2 * kTileBytes;
                f32x16 s = scores<T, DP>(lds, kt, q, lane);
                const f32x16 dp = scores<T, DP>(lds, vt, dout, lane);
                const bool whole = key0 >= all_lo && key0 + 32 <= all_hi;
                const bool behind = key0 + 31 - diag_min <= -a.reach, ahead = key0 - diag_max >= a.reach;
                if (whole && (a.bias == nullptr || behind || ahead)) {
                    const float add = (behind ? bias_behind : bias_ahead) - base;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = exp2_fast(__builtin_fmaf(s[i], c, add)) * (dp[i] - delta);
                } else {
                    if (a.bias != nullptr) {
                        const float* const from = bias_from(bias, a.reach, key0 + 4 * g - diag);
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], c, from[row_of(i, 0)]);
                    } else {
                        s *= c;
                    }
                    const uint32_t first = key0 + 4 * g - lo, span = hi - lo;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float ds = exp2_fast(s[i] - base) * (dp[i] - delta);
                        s[i] = whole || first + row_of(i, 0) < span ? ds : 0.f;
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += s[i];
                if (T::kNarrow && round == 0) {   // (delta is zero still)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(s[i]));
                }
                if (round == 1) accumulate<T, DP>(acc, lds, kt, s, lane);   // (ds rounded to the inputs' 16 bits)
            }
            tile_arrived();
            __syncthreads();
        }
        const float off = ldexpf(sum + from_other_half(sum), -lift);
        sum = 0.f;
        if (off == off) delta += off;
        else if (round == 0 && counts) delta = dot_of_rows<T>(w.dout + row_bytes, w.out + row_bytes, a.dim, g);
    }
    if (counts && g == 0) {
        w.delta[by_head] = delta;
        if (w.twice) w.lse2[by_head] = lse2;
    }
    // Once more, without what a row does not see: for rows whose score gradients are numbers, as delta shows, which is do . out
    // where their sum is none.  (It need not be theirs: beyond a head's width a tile repeats its start, and 0 times infinity is none.)
    if (__any(sees && has_nan(acc) && delta == delta)) {
#pragma unroll
        for (int db = 0; db < NB; ++db) acc[db] = f32x16{};
#pragma unroll 1
        for (int j = wave_lo; j < wave_hi; ++j) {
            const float dot = dot_row<T, DP>(q, k_src + (int64_t)j * a.k_row, a.dim, lane);
            const float dp = dot_row<T, DP>(dout, v_src + (int64_t)j * a.v_row, a.dim, lane);
            if (j >= lo && j < hi)
                accumulate_row<T, DP>(acc, k_src + (int64_t)j * a.k_row,
                                      exp2_fast(__builtin_fmaf(dot, c, bias_at(j) - base)) * (dp - delta), a.dim, g);
        }
    }
    store_rows<T, DP>(acc, ldexpf(a.scale, -lift), !sees, lds + wave * 32 * Tile<DP>::kRowBytes, a.dim, lane,
                      [&](int r) -> char* {
                          const int there = tile.first + 32 * wave + r;
                          return there < tile.last ? w.dq + ((int64_t)there * a.heads + head) * a.dim * 2 : nullptr;
                      });
}

// dk and dv of 32 WR keys of one key head, 32 a wave, over the query rows of all heads of its group, and the sums of
// ds by distance.
//   WR = 4: 128 keys, every wave takes all rows of a tile;
//   WR = 2: 64 keys for twice as many workgroups: two waves share keys, take every other 32 rows, and add their
//           sums up at the end.
// What bounds it: over walks, memory and the sums by distance (16,384 walks of 16 steps with 8 heads of 64 elements
// 0.46 ms); else the wait of one product for another, since keys, values and both sums leave registers for one
// wave a SIMD of rows of 128 elements, two of shorter ones (5 causal sequences of 333 to 4,096 rows with 16 heads of
// 128 elements to 4 of keys 0.73 ms, 24 of up to 2,048 with 12 heads of 80 elements 0.45).  Tried at those sizes and slower:
// dk and dv in launches of their own (448 + 720 us), p and ds by two waves that exchange them (805 and 718 us),
// two blocks of rows at a time (over 900 us).
template <class T, int DP, int WR>
__global__ __launch_bounds__(kThreads, DP > 96 ? 1 : 2) void attention_dkv_kernel(AttentionArgs a, GradArgs w) {
    constexpr int NB = DP / 32, kTileBytes = kTileRows * Tile<DP>::kRowBytes, WK = 4 / WR;
    // fp16: weights, at most 1, are multiplied by 2^14 before they are rounded for dv, and ds with them: one of 2^-28, of a
    // row that sees 2^28 keys alike, still has all its bits.  (As they are, weights of rows of 16,000 keys would be subnormal.)
    constexpr int kWeightLift = T::kNarrow ? 14 : 0;
    constexpr float kWeightDown = 1.f / (1 << kWeightLift);
    extern __shared__ __align__(16) char lds[];
    __shared__ int range[2][4];
    __shared__ float maxima[2][4];
    __shared__ __align__(16) float stats[2][2][kTileRows];   // [buffer][(lift of weights - lse) / scale, -delta][row]
    char* const q_tile = lds;
    char* const o_tile = lds + 2 * kTileBytes;
    const int width = 2 * a.reach + 1;
    float* const sums_of_waves = reinterpret_cast<float*>(lds + 4 * kTileBytes);   // [4][width]
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, g = lane >> 5, col = lane & 31;
    const int wr = wave % WR, wk = wave / WR;
    float* const sums = sums_of_waves + wave * width;
    float* const all_diagonals = sums_of_waves + 4 * width;                        // [4][16][kDiagonals]
    float* const diagonals = all_diagonals + wave * 16 * kDiagonals;
    float* const bias = all_diagonals + 4 * 16 * kDiagonals;

    const uint32_t number = block_number();
    const int kv_head = number % a.kv_heads, tile_no = number / a.kv_heads;
    if (tile_no >= w.k_tiles) return;
    const TileOfRows tile = tile_of_rows(a.k_off, a.n_seqs, a.n_k, 32 * WR, w.across_k, tile_no);
    auto by_distance = [&](int head) { return w.by_distance + ((int64_t)head * w.k_tiles + tile_no) * width; };
    const int group = a.heads / a.kv_heads;
    if (tile.first >= tile.last) {
        if (a.bias != nullptr)
            for (int h = kv_head * group; h < (kv_head + 1) * group; ++h)
                for (int d = tid; d < width; d += kThreads) by_distance(h)[d] = 0.f;
        return;
    }
    // the lane's key, the query rows that see it (lo <= t < hi), and `place`: a row t is place - t away
    const int key0 = tile.first + 32 * wr, key = key0 + col;
    const bool counts = key < tile.last;
    int lo = 0, hi = 0, place = 0;
    if (counts) {
        const int s = tile.seq >= 0 ? tile.seq : segment_of(a.k_off, a.n_seqs, a.n_k, key);
        const Sequence seq = sequence_at(a, s);
        place = key - seq.k1 + seq.q1;
        hi = seq.q1;
        lo = a.causal ? max(seq.q0, place) : seq.q0;
        if (hi <= lo || key < seq.k0 || key >= seq.k1) lo = hi = 0;
    }
    const bool sees = counts && hi > lo, full = __all(counts);
    const int wave_lo = wave_min(sees ? lo : 0x7FFFFFFF), wave_hi = wave_max(sees ? hi : 0);
    const int all_lo = wave_max(counts ? lo : 0), all_hi = wave_min(counts ? hi : 0x7FFFFFFF);
    const int place_min = wave_min(counts ? place : 0x7FFFFFFF), place_max = wave_max(counts ? place : -0x3FFFFFFF);
    const int place0 = place_min;   // of the wave's first key: the others' lie behind it one by one
    if (lane == 0) range[0][wave] = wave_lo, range[1][wave] = wave_hi;
    if (a.bias != nullptr)
        for (int i = tid; i < 4 * 16 * kDiagonals; i += kThreads) all_diagonals[i] = 0.f;
    __syncthreads();
    int row_begin = 0x7FFFFFFF, row_end = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) row_begin = min(row_begin, range[0][i]), row_end = max(row_end, range[1][i]);

    Stationary<DP> k, v;
    k.load(a.k + (int64_t)key * a.k_row + (int64_t)kv_head * a.k_head, counts, a.dim, lane);
    v.load(a.v + (int64_t)key * a.v_row + (int64_t)kv_head * a.v_head, counts, a.dim, lane);
    const float c = a.scale * kLog2e;
    int lift = 0;
    if (T::kNarrow) {
        float size = 0.f, delta = 0.f;
        for (int h = kv_head * group; h < (kv_head + 1) * group; ++h)
            for (int i = tid; i < row_end - row_begin; i += kThreads) {   // (begin is beyond end where no row sees a key)
                const int64_t at = (int64_t)h * a.n_q + row_begin + i;
                size = fmaxf(size, finite_or_zero(w.dout_size[at]));
                delta = fmaxf(delta, finite_or_zero(w.delta[at]));
            }
        size = largest_of_all(size, maxima[0], tid);
        lift = lift_for(size * size_of(v) + largest_of_all(delta, maxima[1], tid));
    }
    const float up = ldexpf(1.f, lift - kWeightLift);

    f32x16 dk[NB], dv[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db) dk[db] = dv[db] = f32x16{};
#pragma unroll 1
    for (int h = kv_head * group; h < (kv_head + 1) * group; ++h) {
        const char* const q_src = a.q + (int64_t)h * a.q_head;
        const char* const o_src = w.dout + (int64_t)h * a.dim * 2;
        const uint32_t o_row = (uint32_t)a.heads * a.dim * 2;
        float stat = 0.f;
        auto fetch = [&](int row, int buffer) {
            const int rows = row_end - row, t = tid;
            copy_tile<DP, kTileRows, kThreads>(q_tile + buffer * kTileBytes, q_src + (int64_t)row * a.q_row, a.q_row, rows, a.dim, t);
            copy_tile<DP, kTileRows, kThreads>(o_tile + buffer * kTileBytes, o_src + (int64_t)row * o_row, o_row, rows, a.dim, t);
            if (t < 2 * kTileRows)
                stat = (t < kTileRows ? w.lse2 : w.delta)[(int64_t)h * a.n_q + min(row + (t & (kTileRows - 1)), row_end - 1)];
        };
        auto keep = [&](int buffer) {
            const int t = tid;
            if (t < 2 * kTileRows) stats[buffer][t / kTileRows][t & (kTileRows - 1)] = t < kTileRows ? (stat - kWeightLift) * (-1.f / c) : -stat;
        };
        if (row_begin < row_end) {
            fetch(row_begin, 0);
            keep(0);
        }
        if (a.bias != nullptr) {
            fill_bias<T>(bias, a, h, tid, kThreads);
            for (int d = tid; d < 4 * width; d += kThreads) sums_of_waves[d] = 0.f;
        }
        float sum_behind = 0.f, sum_ahead = 0.f;   // of ds, distances of reach and more
        tile_arrived();
        __syncthreads();
        float bias_behind = 0.f, bias_ahead = 0.f;
        if (a.bias != nullptr) bias_behind = bias[0], bias_ahead = bias[bias_width(a.reach) - 1];
        int buffer = 0;
#pragma unroll 1
        for (int row = row_begin; row < row_end; row += kTileRows, buffer ^= 1) {
            const bool more = row + kTileRows < row_end;
            if (more) fetch(row + kTileRows, buffer ^ 1);
#pragma unroll 1
            for (int b = 32 * wk; b < kTileRows; b += 32 * WK) {
                const int row0 = row + b;
                if (row0 >= wave_hi || row0 + 32 <= wave_lo) continue;
                const uint32_t qt = buffer * kTileBytes + b * Tile<DP>::kRowBytes, ot = qt + 2 * kTileBytes;
                // (products start from these, so that these need neither registers nor additions)
                f32x16 p = scores<T, DP>(lds, qt, k, lane, by_row(&stats[buffer][0][b], g));
                f32x16 ds = scores<T, DP>(lds, ot, v, lane, by_row(&stats[buffer][1][b], g));
                const bool whole = row0 >= all_lo && row0 + 32 <= all_hi;
                const bool behind = place_max - row0 <= -a.reach, ahead = place_min - (row0 + 31) >= a.reach;
                const bool plain = whole && (a.bias == nullptr || behind || ahead);
                if (plain) {
                    const float add = behind ? bias_behind : bias_ahead;
#pragma unroll
                    for (int i = 0; i < 16; ++i) p[i] = __builtin_fmaf(p[i], c, add);
                } else {
                    if (a.bias != nullptr) {
                        // (rows ahead lie at smaller distances: counted from the last of them)
                        const float* const from = bias_from(bias, a.reach, place - (row0 + 4 * g) - 27);
#pragma unroll
                        for (int i = 0; i < 16; ++i) p[i] = __builtin_fmaf(p[i], c, from[27 - row_of(i, 0)]);
                    } else {
                        p *= c;
                    }
                    if (!whole || !full) {
                        const uint32_t first = row0 + 4 * g - lo, span = hi - lo;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const bool seen = first + row_of(i, 0) < span;
                            p[i] = seen ? p[i] : -INFINITY;
                            ds[i] = seen ? ds[i] : 0.f;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    p[i] = exp2_fast(p[i]);
                    ds[i] *= p[i];
                }
                if (a.bias != nullptr) {
                    if (plain) {
                        float sum = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum += ds[i];
                        sum = counts ? sum : 0.f;
                        if (behind) sum_behind += sum;
                        else sum_ahead += sum;
                    } else {
                        // Neighbouring keys lie at neighbouring places, so 16 rows' ds, each row moved one place
                        // against the one before, have a distance a column: every lane adds one up.  (Adding every
                        // element to its distance's sum with LDS atomics takes 30 cycles for 32 lanes.)  The
                        // corners that no ds falls on stay zero.
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int t = row_of(e, g);
                                diagonals[t * kDiagonals + col - t + 15] = ds[8 * half + e];
                            }
                            wave_sync();
                            if (lane < kDiagonals - 1) {
                                float sum = 0.f;
#pragma unroll
                                for (int t = 0; t < 16; ++t) sum += diagonals[t * kDiagonals + lane];
                                const int d = place0 + lane - 15 - (row0 + 16 * half);
                                if (d <= -a.reach) sum_behind += sum;
                                else if (d >= a.reach) sum_ahead += sum;
                                else sums[d + a.reach] += sum;
                            }
                            wave_sync();
                        }
                    }
                }
                if (T::kNarrow) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) ds[i] *= up;
                }
                accumulate<T, DP>(dv, lds, ot, p, lane);    // (p and ds rounded to the inputs' 16 bits)
                accumulate<T, DP>(dk, lds, qt, ds, lane);
            }
            if (more) keep(buffer ^ 1);
            tile_arrived();
            __syncthreads();
        }
        if (a.bias != nullptr) {
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) sum_behind += __shfl_xor(sum_behind, m), sum_ahead += __shfl_xor(sum_ahead, m);
            if (lane == 0) {
                if (a.reach == 0) sums[0] = sum_behind + sum_ahead;
                else sums[0] = sum_behind, sums[2 * a.reach] = sum_ahead;
            }
            __syncthreads();
            for (int d = tid; d < width; d += kThreads)
                by_distance(h)[d] = ((sums_of_waves[d] + sums_of_waves[width + d]) +
                                     (sums_of_waves[2 * width + d] + sums_of_waves[3 * width + d])) * kWeightDown;
            __syncthreads();
        }
    }
    // Once more, without rows that do not see the key: for sums that are not numbers though all that the key is seen by is.  (lse is
    // none where a row's weights are, delta where its score gradients are.)
    const bool dk_bad = sees && has_nan(dk), dv_bad = sees && has_nan(dv);
    bool dk_none = false, dv_none = false;
    auto unexplained = [&] { return __any((dk_bad && !dk_none) || (dv_bad && !dv_none)); };
#pragma unroll 1
    for (int h = kv_head * group; h < (kv_head + 1) * group && unexplained(); ++h)
#pragma unroll 1
        for (int t0 = wave_lo; t0 < wave_hi && unexplained(); t0 += 64) {
            const int64_t at = (int64_t)h * a.n_q + min(t0 + lane, wave_hi - 1);
            const bool weights = w.lse2[at] == w.lse2[at], scores = w.delta[at] == w.delta[at];
#pragma unroll 1
            for (uint64_t rows = __ballot(!weights || !scores), of_weights = __ballot(!weights); rows != 0; rows &= rows - 1) {
                const int n = __builtin_ctzll(rows);
                const bool seen = t0 + n >= lo && t0 + n < hi;
                dk_none = dk_none || seen;
                dv_none = dv_none || (seen && (of_weights >> n & 1) != 0);
            }
        }
    if (unexplained()) {
#pragma unroll
        for (int db = 0; db < NB; ++db) dk[db] = dv[db] = f32x16{};
#pragma unroll 1
        for (int h = kv_head * group; h < (kv_head + 1) * group; ++h)
#pragma unroll 1
            for (int t = wave_lo; t < wave_hi; ++t) {
                if (WK > 1 && ((t - row_begin) >> 5) % WK != wk) continue;
                const char* const q_row = a.q + (int64_t)t * a.q_row + (int64_t)h * a.q_head;
                const char* const o_row = w.dout + ((int64_t)t * a.heads + h) * a.dim * 2;
                const float dot = dot_row<T, DP>(k, q_row, a.dim, lane), dp = dot_row<T, DP>(v, o_row, a.dim, lane);
                if (t >= lo && t < hi) {
                    float add = 0.f;
                    if (a.bias != nullptr) {
                        const int d = a.bucket[min(max(place - t, -a.reach), a.reach) + a.reach];
                        const int b = d < 0 || d >= a.n_buckets ? 0 : d;
                        add = bias_of<T>(a, b, h);
                    }
                    const int64_t at = (int64_t)h * a.n_q + t;
                    const float p = exp2_fast(__builtin_fmaf(dot, c, add - w.lse2[at] + kWeightLift));
                    accumulate_row<T, DP>(dv, o_row, p, a.dim, g);
                    accumulate_row<T, DP>(dk, q_row, p * (dp - w.delta[at]) * up, a.dim, g);
                }
                if ((t & 31) == 31 && __all(!sees || (dk_none && all_nan(dv)))) {   // nothing is left to find
                    h = a.heads;
                    break;
                }
            }
#pragma unroll
        for (int db = 0; db < NB; ++db) dk[db] += dk_none ? NAN : 0.f;
    }
    if (WK > 1) {   // the second wave of a pair to the first (they have the same keys, and lifts)
        float* const there = reinterpret_cast<float*>(lds) + wr * 2 * NB * 16 * 64 + lane;   // [WR][2 NB 16][64]
        __syncthreads();
        if (wk == 1) {
#pragma unroll
            for (int db = 0; db < NB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    there[(db * 16 + i) * 64] = dk[db][i];
                    there[((NB + db) * 16 + i) * 64] = dv[db][i];
                }
        }
        __syncthreads();
        if (wk == 0) {
#pragma unroll
            for (int db = 0; db < NB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    dk[db][i] += there[(db * 16 + i) * 64];
                    dv[db][i] += there[((NB + db) * 16 + i) * 64];
                }
        }
        __syncthreads();
        if (wk == 1) return;
    }
    auto row_of_key = [&](char* rows) {
        return [=](int r) -> char* {
            const int there = key0 + r;
            return there < tile.last ? rows + ((int64_t)there * a.kv_heads + kv_head) * a.dim * 2 : nullptr;
        };
    };
    char* const mine = lds + wr * 32 * Tile<DP>::kRowBytes;
    store_rows<T, DP>(dk, ldexpf(a.scale, -lift), !sees, mine, a.dim, lane, row_of_key(w.dk));
    store_rows<T, DP>(dv, kWeightDown, !sees, mine, a.dim, lane, row_of_key(w.dv));
}

// One workgroup a head and bucket: the tiles' sums of all distances in it, in a fixed order.  By its trips to memory
// (8 heads of 2,048 tiles of 31 distances in 16 buckets 6 us, one head of 1,466 of 257 in 16 buckets 15, and with a workgroup for
// all buckets of a head 10 and 51).
constexpr int kBiasThreads = 1024;
template <class T>
__global__ __launch_bounds__(kBiasThreads) void attention_dbias_kernel(AttentionArgs a, GradArgs w) {
    __shared__ int bucket[2 * kMaxReach + 1];
    __shared__ int mine[2 * kMaxReach + 1];   // the bucket's distances
    __shared__ int n_mine;
    __shared__ float part[kBiasThreads / 64];
    const uint32_t number = block_number();
    const int width = 2 * a.reach + 1, head = number % a.heads, b = number / a.heads, tid = threadIdx.x;
    const int wave = tid >> 6, lane = tid & 63;
    if (b >= a.n_buckets) return;
    for (int d = tid; d < width; d += kBiasThreads) {
        const int x = a.bucket[d];
        bucket[d] = x < 0 || x >= a.n_buckets ? 0 : x;
    }
    __syncthreads();
    if (wave == 0) {
        int n = 0;
        for (int d0 = 0; d0 < width; d0 += 64) {
            const int d = d0 + lane;
            const bool hit = d < width && bucket[d] == b;
            const uint64_t hits = __ballot(hit);
            if (hit) mine[n + __popcll(hits & ((1ull << lane) - 1))] = d;
            n += __popcll(hits);
        }
        if (lane == 0) n_mine = n;
    }
    __syncthreads();
    // threads: as many distances as there are, up to 256 at a time, times slices of the tiles
    int across = 1;
    while (across < 256 && across < n_mine) across *= 2;
    const int slices = kBiasThreads / across, slice = tid / across;
    float sum = 0.f;
    for (int n = tid % across; n < n_mine; n += across) {
        const float* const from = w.by_distance + (int64_t)head * w.k_tiles * width + mine[n];
#pragma unroll 8
        for (int t = slice; t < w.k_tiles; t += slices) sum += from[(int64_t)t * width];
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    if (tid != 0) return;
    for (int n = 1; n < kBiasThreads / 64; ++n) sum += part[n];
    static_cast<typename T::elem*>(w.dbias)[(int64_t)b * a.heads + head] = (typename T::elem)sum;
}

struct GradPlan {
    bool across_q, across_k, twice;
    int keys;   // of a tile
    int64_t q_tiles, k_tiles;
};
GradPlan grad_plan(const AttentionArgs& a, int n_cu) {
    GradPlan p;
    const double mean_q = (double)a.n_q / a.n_seqs, mean_k = (double)a.n_k / a.n_seqs;
    // Tiles across sequences where these are short and alike (8,192 walks of 17 nodes 0.44 ms against 1.6, 2,048
    // sequences of 60 rows 0.40 against 0.51, 1,024 of 120 rows 0.43 against 0.44).  With a bias the rows (keys) of a tile have to
    // stand at neighbouring keys (rows), which those of several sequences do only where queries and keys lie alike.
    const bool may = a.bias == nullptr || a.q_off == a.k_off;
    p.across_q = may && mean_q < 128 && mean_k <= 256 && mean_k <= 2 * mean_q;
    p.across_k = may && mean_k < 128 && mean_q <= 256 && mean_q <= 2 * mean_k;
    // (8,192 walks of 17 nodes 456 us so and 503 with delta from out, which then has to be read; 800 sequences of
    // 250 rows 900 and 892; 200 of 700 rows 1,216 and 1,044)
    p.twice = mean_k <= 256;
    p.q_tiles = tiles_of_rows(a.n_seqs, a.n_q, 128, p.across_q);
    // Tiles of 64 keys where those of 128 are too few, or the longest of them too long: 4 causal sequences of 4,096 rows
    // with 16 heads of 128 elements to 4 of keys 1.32 ms against 1.57, 24 of 700 rows 0.48 both, but 200 of 700 rows
    // with 8 heads of their own 2.87 against 2.40.  Tiles of short sequences are all alike: 94 of them (1,000 of 12
    // rows, 128 elements) 36 us against 39, but 375 70 against 61, 1,500 228 against 174.
    const double full = a.kv_heads * ((double)a.n_k / 128 + (p.across_k ? 0 : 0.5 * a.n_seqs));
    p.keys = full < (p.across_k ? 1 : 8) * n_cu ? 64 : 128;
    p.k_tiles = tiles_of_rows(a.n_seqs, a.n_k, p.keys, p.across_k);
    return p;
}

int64_t blocks_of(const AttentionArgs& a, const GradPlan& p) {   // (buckets: below 2^28)
    return p.q_tiles * a.heads > p.k_tiles * a.kv_heads ? p.q_tiles * a.heads : p.k_tiles * a.kv_heads;
}

size_t aligned(size_t x) { return (x + 255) / 256 * 256; }

hipError_t allow_lds(const void* kernel, size_t bytes) {
    return bytes <= 65536 ? hipSuccess : hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <class T, int DP, int WR>
hipError_t launch_dkv(hipStream_t stream, const AttentionArgs& a, const GradArgs& w, const GradPlan& p, size_t bytes) {
    auto kernel = attention_dkv_kernel<T, DP, WR>;
    const hipError_t rc = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (rc != hipSuccess) return rc;
    hipLaunchKernelGGL(kernel, grid_of(p.k_tiles * a.kv_heads), dim3(kThreads), bytes, stream, a, w);
    return hipGetLastError();
}

template <class T, int DP>
hipError_t launch_width(hipStream_t stream, const AttentionArgs& a, const GradArgs& w, const GradPlan& p) {
    const size_t tiles = 4 * (size_t)kTileRows * Tile<DP>::kRowBytes;
    const size_t width = a.bias != nullptr ? 2 * (size_t)a.reach + 1 : 0;
    auto kernel = attention_dq_kernel<T, DP>;
    const size_t bytes = tiles + (width == 0 ? 0 : bias_width(a.reach) * sizeof(float));
    hipError_t rc = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (rc != hipSuccess) return rc;
    hipLaunchKernelGGL(kernel, grid_of(p.q_tiles * a.heads), dim3(kThreads), bytes, stream, a, w);
    if ((rc = hipGetLastError()) != hipSuccess) return rc;
    const size_t sums = width == 0 ? 0 : (4 * width + 4 * 16 * kDiagonals + bias_width(a.reach)) * sizeof(float);
    return p.keys == 64 ? launch_dkv<T, DP, 2>(stream, a, w, p, tiles + sums) : launch_dkv<T, DP, 4>(stream, a, w, p, tiles + sums);
}

template <class T>
hipError_t launch_type(hipStream_t stream, const AttentionArgs& a, const GradArgs& w, const GradPlan& p) {
    if (blocks_of(a, p) > 0x7FFFFFFF) return hipErrorInvalidValue;
    hipError_t rc = hipSuccess;
    if (!p.twice) {
        const int64_t blocks = ((int64_t)(a.n_q > a.n_k ? a.n_q : a.n_k) * a.heads + 63) / 64;
        hipLaunchKernelGGL(attention_grad_rows_kernel<T>, dim3((unsigned)(blocks < kRowBlocks ? blocks : kRowBlocks)), dim3(kThreads), 0,
                           stream, a, w);
        rc = hipGetLastError();
    }
    if (rc != hipSuccess) return rc;
    rc = a.dim <= 32   ? launch_width<T, 32>(stream, a, w, p)
         : a.dim <= 64 ? launch_width<T, 64>(stream, a, w, p)
         : a.dim <= 96 ? launch_width<T, 96>(stream, a, w, p)
                       : launch_width<T, 128>(stream, a, w, p);
    if (rc != hipSuccess || a.bias == nullptr) return rc;
    hipLaunchKernelGGL(attention_dbias_kernel<T>, grid_of((int64_t)a.heads * a.n_buckets), dim3(kBiasThreads), 0, stream, a, w);
    return hipGetLastError();
}

// Where the parts of the scratch lie; returns its size.
size_t lay_out(const AttentionArgs& a, const GradPlan& p, bool half, char* scratch, GradArgs* w) {
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* const here = scratch + at;
        at += aligned(bytes);
        return here;
    };
    const size_t rows = (size_t)a.n_q * a.heads * sizeof(float);
    const size_t width = a.bias != nullptr ? (2 * (size_t)a.reach + 1) * sizeof(float) : 0;
    w->lse2 = reinterpret_cast<float*>(take(rows));
    w->delta = reinterpret_cast<float*>(take(rows));
    w->dout_size = reinterpret_cast<float*>(take(half ? rows : 0));
    w->v_size = reinterpret_cast<float*>(take(half && !p.twice ? (size_t)a.n_k * a.kv_heads * sizeof(float) : 0));
    w->by_distance = reinterpret_cast<float*>(take((size_t)p.k_tiles * a.heads * width));
    return at;
}

}  // namespace

hipError_t launch_zero(hipStream_t stream, void* dst, int64_t n) {
    if (n <= 0) return hipSuccess;
    const int64_t blocks = (n + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(kThreads), 0, stream,
                       static_cast<uint16_t*>(dst), n);
    return hipGetLastError();
}

size_t attention_grad_scratch_bytes(int n_cu, const AttentionArgs& a, bool half) {
    GradArgs w;
    return lay_out(a, grad_plan(a, n_cu), half, nullptr, &w);
}

int64_t attention_grad_blocks(int n_cu, const AttentionArgs& a) { return blocks_of(a, grad_plan(a, n_cu)); }

hipError_t launch_attention_grad(hipStream_t stream, int n_cu, const AttentionArgs& a, bool half, const void* dout, const void* out,
                                 const float* lse, void* dq, void* dk, void* dv, void* dbias, void* scratch) {
    const GradPlan p = grad_plan(a, n_cu);
    GradArgs w;
    lay_out(a, p, half, static_cast<char*>(scratch), &w);
    w.dout = static_cast<const char*>(dout);
    w.out = static_cast<const char*>(out);
    w.lse = lse;
    w.dq = static_cast<char*>(dq);
    w.dk = static_cast<char*>(dk);
    w.dv = static_cast<char*>(dv);
    w.dbias = dbias;
    w.q_tiles = (int)p.q_tiles;
    w.k_tiles = (int)p.k_tiles;
    w.across_q = p.across_q;
    w.across_k = p.across_k;
    w.twice = p.twice;
    return half ? launch_type<Fp16>(stream, a, w, p) : launch_type<Bf16>(stream, a, w, p);
}

}  // namespace surel
