// Tiles of 16-bit rows for the matrix units (gfx950, wave64), shared by attention and loss.
//
// Every product here has the form C[32 x 32] += A[32 x 16] B[16 x 32] of one wavefront
// (v_mfma_f32_32x32x16): lane l holds the row (of A) or column (of B) l % 32 and eight of the 16
// inner values, those of half g = l / 32; of C it holds column l % 32 and, in register i, row
// 8 (i / 4) + 4 g + i % 4.
//
// The stationary side of a product (query rows, rows of a loss, ...) is always B and C's columns: one
// row of it belongs to one lane and its partner in the other half, so that sums over the streamed side run
// inside a lane.  C's registers, rounded to 16 bits, are then the B operand of the next product
// as they are: inner values 0..3 and 4..7 of half g are the streamed rows 4 g .. 4 g + 3 and
// 8 + 4 g .. 8 + 4 g + 3 of 16.  Its A operand, 16 streamed rows of a tile transposed, is read in the
// same order by two transposing LDS loads of 4 rows each.
//
// Rows lie in LDS in chunks of 16 bytes, permuted inside a row by the row's number so that neither
// kind of load meets a bank twice in a cycle (of 256 bytes, 64 banks): 16 rows' chunks of one column lie in 16
// places of 256 bytes, and 4 neighbouring rows' groups of 4 chunks in 4 different quarters of them.  (Permuted by
// the low 3 bits of the row alone, two thirds of the LDS cycles of rows of 128 elements were conflicts.)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_util.h"

namespace surel {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct Bf16 {
    typedef __bf16 elem;
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    static constexpr bool kNarrow = false;  // has the range of 32-bit floats
    static __device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
};

struct Fp16 {
    typedef _Float16 elem;
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    static constexpr bool kNarrow = true;  // 6e-8 .. 65504: sums of small factors are scaled first
    static __device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
};

// Runs turn(step, buffer) for step = begin, begin + by, ... < end, with buffers 0 and 1 in turn as constants: the places of
// tiles are then parts of the instructions that read them.
template <int N>
struct Constant {
    static constexpr int value = N;
};
template <class Turn>
__device__ __forceinline__ void alternate(int begin, int end, int by, Turn turn) {
#pragma unroll 1
    for (int step = begin; step < end; step += 2 * by) {
        turn(step, Constant<0>());
        if (step + by < end) turn(step + by, Constant<1>());
    }
}

// The thread's wave, and what is the same in all of its lanes, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform(float x) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(x)));
}

// Two 32-bit values rounded to nearest, in one word.
template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, typename T::x2));
}

template <class T>
__device__ __forceinline__ f32x2 unpack2(uint32_t w) {
    return __builtin_convertvector(__builtin_bit_cast(typename T::x2, w), f32x2);
}

// Registers 8 t .. 8 t + 7 of a product (16 streamed rows), as the B operand of the next one.
template <class T>
__device__ __forceinline__ u32x4 as_operand(const f32x16& c, int t) {
    u32x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = pack2<T>(c[8 * t + 2 * e], c[8 * t + 2 * e + 1]);
    return out;
}

// Streamed row (of 32) that register i of a product stands for.
__device__ __forceinline__ int row_of(int i, int g) { return 8 * (i >> 2) + 4 * g + (i & 3); }

// The other half's value of the same column.
__device__ __forceinline__ float from_other_half(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(lane_id() < 32 ? r[1] : r[0]);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// Rows of DP elements (a multiple of 32) in LDS, at byte offsets `at` from the start of dynamic LDS that are
// multiples of 256 (tiles, and 16 rows of them).
template <int DP>
struct Tile {
    static constexpr int kChunks = DP / 8;
    static constexpr int kRowBytes = 2 * DP;
    // What a chunk's number is xor-ed with.  Rows of a multiple of 256 bytes begin in one place of the banks: the
    // row's low bits choose the quarter.  Of 128 bytes, two rows share the 256; of 64, four lie in all quarters.
    static constexpr uint32_t kMixed = DP % 128 == 0 ? 15 : DP % 64 == 0 ? 7 : 3;   // the bits that change
    __device__ __forceinline__ static int permuted(int row) {
        const int high = DP % 128 == 0 ? (row & 3) << 2 : DP % 64 == 0 ? (row & 2) << 1 : 0;
        return high | ((row >> 2) & 3);
    }

    // A operand: the 32 rows at `at`, inner values 16 ks .. 16 ks + 15; lane_rows is the lane's place in rows
    // for ks = 0.  (For other ks it differs by an xor of constant bits; `at` is a constant where loops are unrolled
    // over buffers, and part of the instruction.)
    __device__ __forceinline__ static uint32_t lane_rows(int lane) {
        const int r = lane & 31;
        return r * kRowBytes + (((lane >> 5) ^ permuted(r)) * 16);
    }
    __device__ __forceinline__ static u32x4 rows(const char* lds, uint32_t at, uint32_t lane_rows, int ks) {
        const uint32_t c = 2 * ks;
        return *reinterpret_cast<const u32x4*>(lds + (lane_rows ^ ((c & kMixed) * 16)) + (at + (c & ~kMixed) * 16));
    }

    // A operand: columns 32 db .. 32 db + 31 as rows, the 16 rows at `at` as inner values, in the order that
    // as_operand gives its own; lane_columns as lane_rows above.
    __device__ __forceinline__ static uint32_t lane_columns(int lane) {
        const int i = lane & 15, r = 4 * (lane >> 5) + (i >> 2), c = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
        return r * kRowBytes + ((c ^ permuted(r)) * 16) + (i & 1) * 8;
    }
    __device__ __forceinline__ static u32x4 columns(const char* lds, uint32_t at, uint32_t lane_columns, int db) {
        typedef short v4i16 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) v4i16* lds_ptr;
        const uint32_t c = 4 * db;
        u32x4 out;
#pragma unroll
        for (int half = 0; half < 2; ++half) {   // 8 rows further down the permutation's second bit changes
            const char* const place = lds + (lane_columns ^ (((c & kMixed) ^ (2 * half)) * 16)) +
                                      (at + (c & ~kMixed) * 16 + half * 8 * kRowBytes);
            const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)place));
            out[2 * half] = x[0];
            out[2 * half + 1] = x[1];
        }
        return out;
    }
};

// Copies ROWS rows of global memory to a tile without passing through registers; the caller waits
// (tile_arrived) before the barrier behind which the tile is read.  A wave's 64 chunks lie behind
// one another in LDS, so it is the global chunks that are permuted.  Rows at or beyond `rows` (>= 1) repeat the
// last one and chunks at or beyond `dim` the first: what is there is finite where the rows are, and meets
// weights of zero or lands in columns that nobody reads.
template <int DP, int ROWS, int THREADS>
__device__ __forceinline__ void copy_tile(char* tile, const char* src, uint32_t row_bytes, int rows, int dim, int tid) {
    constexpr int kChunks = Tile<DP>::kChunks, kEach = (ROWS * kChunks + THREADS - 1) / THREADS;
    static_assert(ROWS * kChunks % 64 == 0, "the tile is not a multiple of a wave's chunks");
    typedef __attribute__((address_space(3))) void* lds_ptr;
    typedef const __attribute__((address_space(1))) void* global_ptr;
    const int wave = uniform(tid & ~63);
    char* const mine = tile + wave * 16;
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
        if (ROWS * kChunks % THREADS != 0 && n * THREADS + wave >= ROWS * kChunks) break;
        const int id = tid + n * THREADS, row = id / kChunks;
        const int c = (id % kChunks) ^ Tile<DP>::permuted(row);   // (below kMixed: stays inside the row)
        const uint32_t at = (uint32_t)min(row, rows - 1) * row_bytes + (c * 8 < dim ? c * 16 : 0);
        __builtin_amdgcn_global_load_lds((global_ptr)(src + at), (lds_ptr)(mine + n * THREADS * 16), 16, 0, 0);
    }
}
__device__ __forceinline__ void tile_arrived() { __builtin_amdgcn_s_waitcnt(0x0F70); }  // vmcnt(0)

// B operand: one row of global memory a lane (all of its DP elements over the two halves; zeros at
// and beyond `dim`, and everywhere if the row does not count).
template <int DP>
struct Stationary {
    u32x4 k[DP / 16];
    __device__ __forceinline__ void load(const char* row, bool counts, int dim, int lane) {
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) {
            const int c = 2 * ks + (lane >> 5);
            k[ks] = u32x4{0, 0, 0, 0};
            if (counts && c * 8 < dim) k[ks] = *reinterpret_cast<const u32x4*>(row + c * 16);
        }
    }
};

// C[32 streamed rows][32 stationary rows] of the rows at `at`, on top of c.
template <class T, int DP>
__device__ __forceinline__ f32x16 scores(const char* lds, uint32_t at, const Stationary<DP>& b, int lane, f32x16 c = {}) {
    const uint32_t mine = Tile<DP>::lane_rows(lane);
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) c = T::mma(Tile<DP>::rows(lds, at, mine, ks), b.k[ks], c);
    return c;
}

// What is one value a streamed row, 32 of them from LDS, as the start of a product.
__device__ __forceinline__ f32x16 by_row(const float* values, int g) {
    f32x16 c;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(values + 8 * n + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) c[4 * n + e] = x[e];
    }
    return c;
}

// acc[d][stationary row] += sum over the 32 streamed rows at `at` of row[d] w[row][stationary row].
template <class T, int DP>
__device__ __forceinline__ void accumulate(f32x16 (&acc)[DP / 32], const char* lds, uint32_t at, const f32x16& w, int lane) {
    const uint32_t mine = Tile<DP>::lane_columns(lane);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const u32x4 b = as_operand<T>(w, t);
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
            acc[db] = T::mma(Tile<DP>::columns(lds, at + 16 * t * Tile<DP>::kRowBytes, mine, db), b, acc[db]);
    }
}

// The same products one streamed row at a time, from global memory and in 32 bits throughout.  A tile's
// product also multiplies what a row does not see, by a weight of zero: that is NaN where it is not finite.  Who
// finds a sum that is not a number therefore goes over its rows again with these, and leaves out what they do
// not see; but not, or no further, where all that it would find is that they see it themselves.
template <class T, int DP>
__device__ __forceinline__ float dot_row(const Stationary<DP>& b, const char* row, int dim, int lane) {
    float sum = 0.f;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) {
        const int c = 2 * ks + (lane >> 5);
        if (c * 8 < dim) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(row + c * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x2 p = unpack2<T>(x[e]), q = unpack2<T>(b.k[ks][e]);
                sum = __builtin_fmaf(p[0], q[0], sum);
                sum = __builtin_fmaf(p[1], q[1], sum);
            }
        }
    }
    return sum + from_other_half(sum);
}
template <class T, int DP>
__device__ __forceinline__ void accumulate_row(f32x16 (&acc)[DP / 32], const char* row, float w, int dim, int g) {
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * db + row_of(i, g);
            if (d < dim) {
                const u32x2 x = *reinterpret_cast<const u32x2*>(row + d * 2);
                const f32x2 lo = unpack2<T>(x[0]), hi = unpack2<T>(x[1]);
                acc[db][i] = __builtin_fmaf(w, lo[0], acc[db][i]);
                acc[db][i + 1] = __builtin_fmaf(w, lo[1], acc[db][i + 1]);
                acc[db][i + 2] = __builtin_fmaf(w, hi[0], acc[db][i + 2]);
                acc[db][i + 3] = __builtin_fmaf(w, hi[1], acc[db][i + 3]);
            }
        }
}

// Sums of 32 stationary rows, times `scale` (a lane's own), rounded and written as rows of 16-bit
// elements.  They pass through 32 rows of LDS of the wave's own (of a tile that nobody reads any more), so that
// rows go out 16 bytes a lane in whole lines.  dst_of(row) is where row `row` of the 32 goes, or null.
template <class T, int DP, class Dst>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[DP / 32], float scale, bool zero, char* lds, int dim, int lane,
                                           Dst dst_of) {
    const int g = lane >> 5, col = lane & 31;
    wave_sync();
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * db + row_of(i, g);
            const u32x2 w = {pack2<T>(acc[db][i] * scale, acc[db][i + 1] * scale),
                             pack2<T>(acc[db][i + 2] * scale, acc[db][i + 3] * scale)};
            *reinterpret_cast<u32x2*>(lds + col * Tile<DP>::kRowBytes + (((d >> 3) ^ Tile<DP>::permuted(col)) * 16) +
                                      (d & 4) * 2) = zero ? u32x2{0, 0} : w;
        }
    wave_sync();
#pragma unroll
    for (int n = 0; n < DP / 16; ++n) {
        const int id = lane + 64 * n, r = id / Tile<DP>::kChunks, c = id % Tile<DP>::kChunks;
        char* const dst = dst_of(r);
        if (dst != nullptr && c * 8 < dim)
            *reinterpret_cast<u32x4*>(dst + c * 16) =
                *reinterpret_cast<const u32x4*>(lds + r * Tile<DP>::kRowBytes + ((c ^ Tile<DP>::permuted(r)) * 16));
    }
}

template <int NB>
__device__ __forceinline__ bool has_nan(const f32x16 (&acc)[NB]) {
    bool bad = false;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) bad = bad || acc[db][i] != acc[db][i];
    return bad;
}

// Whether nothing can change any more: what is not a number stays so.
template <int NB>
__device__ __forceinline__ bool all_nan(const f32x16 (&acc)[NB]) {
    bool bad = true;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) bad = bad && acc[db][i] != acc[db][i];
    return bad;
}

}  // namespace surel
