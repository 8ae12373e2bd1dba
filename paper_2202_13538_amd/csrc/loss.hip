// Softmax cross entropy of rows against a large table of classes (surel_softmax_loss).
#include <math.h>

#include "kernels.h"
#include "loss.h"

namespace surel {
namespace {

constexpr int kThreads = 256;
constexpr float kMost = 1e12f;

__device__ __forceinline__ float sum_of(const f32x16& s, float base) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += exp2_fast(__builtin_fmaf(s[i], kLog2e, -base));
    return sum;
}

struct LossOut {
    f32x4* part = nullptr;  // [n_rows][parts of rows]: maximum and sum (base 2), the label's score
    float *loss = nullptr, *lse = nullptr;
    int splits = 1;
    int row_parts = 1;      // splits times the waves that share a row
    uint32_t* turns = nullptr;  // [tiles] of zeros, or null: a launch of its own joins the parts
};

// Joining the parts of a row's classes: 64 lanes, then (where there are several) the waves.
struct Joined {
    float top = -INFINITY, sum = 0.f, hit = 0.f;
    __device__ __forceinline__ void add(float other, float other_sum, float other_hit) {
        const float now = fmaxf(top, other), base = now == -INFINITY ? 0.f : now;
        sum = sum * exp2_fast(top - base) + other_sum * exp2_fast(other - base);
        top = now;
        hit += other_hit;
    }
    __device__ __forceinline__ void add_lanes() {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) add(__shfl_xor(top, m), __shfl_xor(sum, m), __shfl_xor(hit, m));
    }
    __device__ __forceinline__ void write(const LossArgs& a, const LossOut& o, int row) const {
        const float lse = (top + log2_fast(sum)) * kLn2;
        const int label = a.labels[row];
        o.lse[row] = lse;
        o.loss[row] = label < 0 || label >= a.n_classes ? 0.f : lse - hit;
    }
};

// Words that workgroups on other XCDs read in the same launch: past the caches in between.
__device__ __forceinline__ void put(float* at, float x) { __hip_atomic_store(at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float get(const float* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

template <int DP, int WR>
struct LossShape {
    static constexpr int WK = 4 / WR;
    static constexpr int RB = WR == 1 ? 1 : 2;               // blocks of 32 rows a wave holds
    static constexpr int kRows = 32 * RB * WR;
    static constexpr int kKeys = WK == 1 ? 64 : 32;          // classes a wave takes at a time
    static constexpr int kTileKeys = kKeys * WK;
    static constexpr int kTileBytes = kTileKeys * Tile<DP>::kRowBytes;
};

// One workgroup: kRows rows against a part of the classes, which stream through LDS.  Waves hold their rows
// in registers and compute scores^T = W h^T: a row's scores lie in one lane and its partner, each of
// which keeps a running maximum and sum of its own until the end.  No logit leaves the registers.
//   WR = 4: 256 rows, every wave 64 of them and all classes of a tile;
//   WR = 1: 32 rows, the waves take different classes of a tile.
// What bounds it: 16 rows against 2,900,000 classes of 128 elements, reading these (120 us, 6.2 TB/s); 15,001 rows against
// 99,991 classes of 200 elements, the matrix units (0.54 ms, 1.11 PFLOP/s; 8,192 rows against 235,000 of 128 0.48 ms,
// 1.03); of 64 elements the exponentials between products that are as short as they (2,048 rows against 2,900,000
// 1.19 ms, 0.64 PFLOP/s).  (Of a warm device, as all times here: the first passes take up to an eighth longer.)
template <class T, int DP, int WR>
__global__ __launch_bounds__(kThreads, 2) void loss_kernel(LossArgs a, LossOut o) {
    using Shape = LossShape<DP, WR>;
    constexpr int RB = Shape::RB;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, g = lane >> 5, col = lane & 31;
    const int split = blockIdx.x % o.splits, row_tile = blockIdx.x / o.splits;
    const int first = row_tile * Shape::kRows + (WR == 1 ? 0 : wave * 32 * RB), wk = WR == 1 ? wave : 0;

    Stationary<DP> h[RB];
    int label[RB];
    float top[RB], sum[RB], hit[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int row = first + 32 * r + col;
        const bool counts = row < a.n_rows;
        h[r].load(a.h + (int64_t)row * a.dim * 2, counts, a.dim, lane);
        label[r] = counts ? label_of(a, row) : -1;
        top[r] = -INFINITY, sum[r] = 0.f, hit[r] = 0.f;
    }
    const int steps = (a.n_classes + Shape::kTileKeys - 1) / Shape::kTileKeys, each = (steps + o.splits - 1) / o.splits;
    const int begin = min(split * each, steps), end = min(begin + each, steps);
    const uint32_t row_bytes = (uint32_t)a.dim * 2;
    auto fetch = [&](int step, int buffer) {
        const int c0 = step * Shape::kTileKeys;
        copy_tile<DP, Shape::kTileKeys, kThreads>(lds + buffer * Shape::kTileBytes, a.w + (int64_t)c0 * row_bytes, row_bytes,
                                                  a.n_classes - c0, a.dim, tid);
    };
    if (begin < end) fetch(begin, 0);
    tile_arrived();
    __syncthreads();
    const bool works = first < a.n_rows;
    alternate(begin, end, 1, [&](int step, auto of) __attribute__((always_inline)) {
        constexpr int buffer = decltype(of)::value;
        if (step + 1 < end) fetch(step + 1, buffer ^ 1);
        if (works) {
#pragma unroll
            for (int b = 0; b < Shape::kKeys; b += 32) {
                const int c0 = step * Shape::kTileKeys + wk * Shape::kKeys + b;
                const uint32_t at = buffer * Shape::kTileBytes + (wk * Shape::kKeys + b) * Tile<DP>::kRowBytes;
                f32x16 s[RB] = {};
#pragma unroll
                for (int ks = 0; ks < DP / 16; ++ks) {
                    const u32x4 x = Tile<DP>::rows(lds, at, Tile<DP>::lane_rows(lane), ks);
#pragma unroll
                    for (int r = 0; r < RB; ++r) s[r] = T::mma(x, h[r].k[ks], s[r]);
                }
                if (c0 + 32 > a.n_classes) {
#pragma unroll
                    for (int r = 0; r < RB; ++r)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[r][i] = c0 + row_of(i, g) < a.n_classes ? s[r][i] : -INFINITY;
                }
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    if (__any((uint32_t)(label[r] - c0) < 32u)) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) hit[r] = label[r] - c0 == row_of(i, g) ? s[r][i] : hit[r];
                    }
                    // Relative to a maximum of earlier classes: as long as these add up to less than kMost,
                    // their own need not be known.
                    float part = sum_of(s[r], top[r] == -INFINITY ? 0.f : top[r]);
                    const bool again = top[r] == -INFINITY || !(part < kMost);   // (the row's own affair: no other row's
                    if (__any(again)) {                                          // result depends on it)
                        float most = s[r][0];
#pragma unroll
                        for (int i = 1; i < 16; ++i) most = fmaxf(most, s[r][i]);
                        const float now = again ? fmaxf(top[r], most * kLog2e) : top[r], base = now == -INFINITY ? 0.f : now;
                        sum[r] *= exp2_fast(top[r] - base);
                        top[r] = now;
                        part = sum_of(s[r], base);
                    }
                    sum[r] += part;
                }
            }
        }
        tile_arrived();
        __syncthreads();
    });
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const float other = from_other_half(top[r]), other_sum = from_other_half(sum[r]), other_hit = from_other_half(hit[r]);
        const float now = fmaxf(top[r], other), base = now == -INFINITY ? 0.f : now;
        const float total = sum[r] * exp2_fast(top[r] - base) + other_sum * exp2_fast(other - base);
        const int row = first + 32 * r + col;
        if (g == 0 && row < a.n_rows) {
            f32x4* const part = &o.part[(int64_t)row * o.row_parts + split * Shape::WK + wk];
            if (o.turns == nullptr) {
                *part = f32x4{now, total, hit[r] + other_hit, 0.f};
            } else {
                float* const word = reinterpret_cast<float*>(part);
                put(word, now), put(word + 1, total), put(word + 2, hit[r] + other_hit);
            }
        }
    }
    if (o.turns == nullptr) return;
    // the last workgroup of a tile's joins its rows' parts, in the same order whoever is last
    __shared__ bool last;
    wait_memory();
    __syncthreads();
    if (tid == 0) {
        const uint32_t before = __hip_atomic_fetch_add(&o.turns[row_tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = before == (uint32_t)o.splits - 1;
        if (last) __hip_atomic_store(&o.turns[row_tile], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!last) return;
    for (int row = row_tile * Shape::kRows + wave; row < min((row_tile + 1) * Shape::kRows, a.n_rows); row += kThreads / 64) {
        Joined x;
        for (int p = lane; p < o.row_parts; p += 64) {
            const float* const word = reinterpret_cast<const float*>(&o.part[(int64_t)row * o.row_parts + p]);
            x.add(get(word), get(word + 1), get(word + 2));
        }
        x.add_lanes();
        if (lane == 0) x.write(a, o, row);
    }
}

// The parts of a row's classes: a wave a row, or a workgroup where there are more than 64 parts.
template <int WAVES>
__global__ __launch_bounds__(kThreads) void loss_join_kernel(LossArgs a, LossOut o) {
    __shared__ float of_wave[3][kThreads / 64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t place = WAVES == 1 ? (int64_t)block_number() * (kThreads / 64) + wave : block_number();
    if (place >= a.n_rows) return;
    const int row = (int)place;
    Joined x;
#pragma unroll 4
    for (int p = WAVES == 1 ? lane : threadIdx.x; p < o.row_parts; p += 64 * WAVES) {
        const f32x4 y = o.part[(int64_t)row * o.row_parts + p];
        x.add(y[0], y[1], y[2]);
    }
    x.add_lanes();
    if (WAVES > 1) {
        if (lane == 0) of_wave[0][wave] = x.top, of_wave[1][wave] = x.sum, of_wave[2][wave] = x.hit;
        __syncthreads();
        x = Joined{of_wave[0][0], of_wave[1][0], of_wave[2][0]};
#pragma unroll
        for (int w = 1; w < WAVES; ++w) x.add(of_wave[0][w], of_wave[1][w], of_wave[2][w]);
    }
    if (lane == 0 && (WAVES == 1 || wave == 0)) x.write(a, o, row);
}

struct LossPlan {
    bool few, alone;   // alone: the last workgroup of a tile joins its parts
    int splits, row_parts;
    int64_t tiles;
};
LossPlan loss_plan(const LossArgs& a, int n_cu) {
    LossPlan p;
    // (tiles of 32 rows up to 128 of them: 64 rows against 1,000,000 classes of 64 elements 27 us, in one tile of 256 rows
    // 44; 128 rows 43 and 58, 192 both 60, 256 rows 71 and 62)
    p.few = a.n_rows <= 128;
    const int rows = p.few ? 32 : 256, keys = p.few ? 128 : 64;
    p.tiles = (a.n_rows + rows - 1) / rows;
    p.splits = parts_for(p.tiles, (a.n_classes + keys - 1) / keys, 2 * n_cu, 1024, 0.0);
    p.row_parts = p.splits * (p.few ? 4 : 1);
    // (one launch less: 7 rows against 4,096 classes 8.2 us instead of 11.8.  One workgroup joins all parts then, from past
    // the caches: 16 rows of 256 parts take 14.6 us, in a launch of their own 12.6, 32 rows 23 and 12.6.)
    p.alone = p.few && p.tiles == 1 && (int64_t)a.n_rows * p.row_parts <= 2048;
    return p;
}

template <class T, int DP, int WR>
hipError_t launch(hipStream_t stream, const LossArgs& a, const LossOut& o, const LossPlan& p) {
    const size_t bytes = 2 * LossShape<DP, WR>::kTileBytes;
    if (!fits_a_row(p.tiles * p.splits, kThreads)) return hipErrorInvalidValue;
    auto kernel = loss_kernel<T, DP, WR>;
    if (bytes > 65536) {
        const hipError_t rc = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                  hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (rc != hipSuccess) return rc;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p.tiles * p.splits)), dim3(kThreads), bytes, stream, a, o);
    return hipGetLastError();
}
template <class T, int DP>
hipError_t launch_rows(hipStream_t stream, const LossArgs& a, const LossOut& o, const LossPlan& p) {
    return p.few ? launch<T, DP, 1>(stream, a, o, p) : launch<T, DP, 4>(stream, a, o, p);
}
template <class T>
hipError_t launch_type(hipStream_t stream, const LossArgs& a, const LossOut& o, const LossPlan& p) {
    return a.dim <= 32    ? launch_rows<T, 32>(stream, a, o, p)
           : a.dim <= 64  ? launch_rows<T, 64>(stream, a, o, p)
           : a.dim <= 96  ? launch_rows<T, 96>(stream, a, o, p)
           : a.dim <= 128 ? launch_rows<T, 128>(stream, a, o, p)
           : a.dim <= 160 ? launch_rows<T, 160>(stream, a, o, p)
           : a.dim <= 192 ? launch_rows<T, 192>(stream, a, o, p)
           : a.dim <= 224 ? launch_rows<T, 224>(stream, a, o, p)
                          : launch_rows<T, 256>(stream, a, o, p);
}

}  // namespace

size_t loss_scratch_bytes(int n_cu, const LossArgs& a) {
    return (size_t)a.n_rows * loss_plan(a, n_cu).row_parts * sizeof(f32x4);
}

hipError_t launch_loss(hipStream_t stream, int n_cu, const LossArgs& a, bool half, float* loss, float* lse, void* scratch,
                       uint32_t* turns) {
    const LossPlan p = loss_plan(a, n_cu);
    LossOut o;
    o.part = static_cast<f32x4*>(scratch);
    o.loss = loss;
    o.lse = lse;
    o.splits = p.splits;
    o.row_parts = p.row_parts;
    o.turns = p.alone ? turns : nullptr;
    const hipError_t rc = half ? launch_type<Fp16>(stream, a, o, p) : launch_type<Bf16>(stream, a, o, p);
    if (rc != hipSuccess || p.alone) return rc;
    if (p.row_parts > 64) hipLaunchKernelGGL(loss_join_kernel<4>, grid_of(a.n_rows), dim3(kThreads), 0, stream, a, o);
    else hipLaunchKernelGGL(loss_join_kernel<1>, grid_of(((int64_t)a.n_rows + 3) / 4), dim3(kThreads), 0, stream, a, o);
    return hipGetLastError();
}

}  // namespace surel
