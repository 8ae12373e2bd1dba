// The gradients of the softmax loss (surel_softmax_loss_grad).
//
// With z = h w^T and g_nc = dloss_n (exp(z_nc - lse_n) - [c = label_n]):  dh = g w,  dw = g^T h.
// Logits are made again where they are needed, in the registers of the workgroup that needs them: once for
// dh (rows stay, classes stream by) and once for dw (classes stay, rows stream by).  For rows of up to 256
// elements that is less than to write g, 16 bits a row and class, and read it twice: 4 dim operations against
// 6 bytes, 0.4 against 1.2 ps at 128 elements and the rates of a large product and a large copy.
//
// What bounds them: the matrix units, at the 1.7 to 1.8 GHz that they leave of the clock.  dh: 8,192 rows against 235,000
// classes of 128 elements 0.81 ms (1.22 PFLOP/s), 15,001 against 99,991 of 200 1.02 ms (1.18), 2,048 against 2,900,000
// of 64 1.58 ms (0.97, exponentials).  dw: 0.99 ms (1.00), 1.38 ms (0.87) and 1.53 ms (0.99).
#include <math.h>

#include "kernels.h"
#include "loss.h"

namespace surel {
namespace {

constexpr int kThreads = 256;
constexpr int kStep = 64;  // streamed rows or classes of a tile
// fp16 only: weights (of at most 1) are multiplied by 2^12 before they are rounded, so that a class's share
// of 1.5e-8 still has all its bits.
constexpr int kLift = 12;
constexpr int kMaxima = 256;  // workgroups that look for the largest |dloss|, at most

struct LossGradArgs {
    const float *dloss = nullptr, *lse = nullptr;
    void *dh = nullptr, *dw = nullptr;
    float *part_h = nullptr, *part_w = nullptr;  // [split][rows][dim], where there are several
    float* maxima = nullptr;                     // [n_maxima], of parts of |dloss| (fp16 only)
    int n_maxima = 0;
    int splits_h = 1, splits_w = 1;
};

__global__ __launch_bounds__(kThreads) void largest_kernel(LossArgs a, LossGradArgs w) {
    __shared__ float most_of[kThreads / 64];
    float most = 0.f;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < a.n_rows; i += (int64_t)gridDim.x * kThreads)
        if (a.labels[i] >= 0) most = fmaxf(most, fabsf(w.dloss[i]));
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    if ((threadIdx.x & 63) == 0) most_of[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x == 0) w.maxima[blockIdx.x] = fmaxf(fmaxf(most_of[0], most_of[1]), fmaxf(most_of[2], most_of[3]));
}

// The power of two that dloss is multiplied by before weights are rounded to fp16: the largest becomes 2^11 .. 2^12.
template <class T>
__device__ __forceinline__ int lift_of(const LossGradArgs& w, int lane) {
    if (!T::kNarrow) return 0;
    float most = 0.f;
    for (int i = lane; i < w.n_maxima; i += 64) most = fmaxf(most, w.maxima[i]);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    if (!(most > 0.f) || !(most < INFINITY)) return 0;
    return min(max(kLift - 1 - ilogbf(most), -100), 100);
}

// dh of 128 rows, 32 a wave, from a part of the classes.
template <class T, int DP>
__global__ __launch_bounds__(kThreads, DP > 224 ? 1 : 2) void loss_dh_kernel(LossArgs a, LossGradArgs w) {
    constexpr int NB = DP / 32, kTileBytes = kStep * Tile<DP>::kRowBytes;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, g = lane >> 5, col = lane & 31;
    const int split = blockIdx.x % w.splits_h, first = blockIdx.x / w.splits_h * 128 + wave * 32, row = first + col;
    const bool in = row < a.n_rows, works = first < a.n_rows;
    Stationary<DP> h;
    h.load(a.h + (int64_t)row * a.dim * 2, in, a.dim, lane);
    const int label = in ? label_of(a, row) : -1;
    const float lift = T::kNarrow ? (float)kLift : 0.f, one = T::kNarrow ? (float)(1 << kLift) : 1.f;
    const float base = (in ? w.lse[row] * kLog2e : 0.f) - lift;
    const float scale = label >= 0 ? w.dloss[row] / one : 0.f;

    f32x16 acc[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db) acc[db] = f32x16{};
    const int steps = (a.n_classes + kStep - 1) / kStep, each = (steps + w.splits_h - 1) / w.splits_h;
    const int begin = min(split * each, steps), end = min(begin + each, steps);
    const uint32_t row_bytes = (uint32_t)a.dim * 2;
    auto fetch = [&](int step, int buffer) {
        const int c0 = step * kStep;
        copy_tile<DP, kStep, kThreads>(lds + buffer * kTileBytes, a.w + (int64_t)c0 * row_bytes, row_bytes,
                                       a.n_classes - c0, a.dim, tid);
    };
    if (begin < end) fetch(begin, 0);
    tile_arrived();
    __syncthreads();
    alternate(begin, end, 1, [&](int step, auto of) __attribute__((always_inline)) {
        constexpr int buffer = decltype(of)::value;
        if (step + 1 < end) fetch(step + 1, buffer ^ 1);
        constexpr uint32_t tile = buffer * kTileBytes;
        if (works) {
#pragma unroll
            for (int b = 0; b < kStep; b += 32) {
                const int c0 = step * kStep + b;
                f32x16 s = scores<T, DP>(lds, tile + b * Tile<DP>::kRowBytes, h, lane);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = exp2_fast(__builtin_fmaf(s[i], kLog2e, -base));
                if (__any((uint32_t)(label - c0) < 32u)) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] -= label - c0 == row_of(i, g) ? one : 0.f;
                }
                if (c0 + 32 > a.n_classes) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = c0 + row_of(i, g) < a.n_classes ? s[i] : 0.f;
                }
                accumulate<T, DP>(acc, lds, tile + b * Tile<DP>::kRowBytes, s, lane);   // (weights rounded to the inputs' 16 bits)
            }
        }
        tile_arrived();
        __syncthreads();
    });
    if (w.splits_h > 1) {
        if (!in) return;
        float* const dst = w.part_h + ((int64_t)split * a.n_rows + row) * a.dim;
        const bool zero = scale == 0.f;
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * db + row_of(i, g);
                const f32x4 x = {acc[db][i] * scale, acc[db][i + 1] * scale, acc[db][i + 2] * scale, acc[db][i + 3] * scale};
                if (d < a.dim) *reinterpret_cast<f32x4*>(dst + d) = zero ? f32x4{0.f, 0.f, 0.f, 0.f} : x;
            }
        return;
    }
    store_rows<T, DP>(acc, scale, scale == 0.f, lds + wave * 32 * Tile<DP>::kRowBytes, a.dim, lane, [&](int r) -> char* {
        return first + r < a.n_rows ? static_cast<char*>(w.dh) + (int64_t)(first + r) * a.dim * 2 : nullptr;
    });
}

// dw of 128 classes, 32 a wave, from a part of the rows.
template <class T, int DP>
__global__ __launch_bounds__(kThreads, DP > 224 ? 1 : 2) void loss_dw_kernel(LossArgs a, LossGradArgs w) {
    constexpr int NB = DP / 32, kTileBytes = kStep * Tile<DP>::kRowBytes;
    extern __shared__ __align__(16) char lds[];
    __shared__ __align__(16) float start[2][kStep];   // [buffer][row]: log |dloss| - lse
    __shared__ __align__(16) float dloss[2][kStep];
    __shared__ __align__(16) int labels[2][kStep];
    __shared__ int negative[2];                       // [buffer]: some dloss of the tile is
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, g = lane >> 5, col = lane & 31;
    const int split = blockIdx.x % w.splits_w, first = blockIdx.x / w.splits_w * 128 + wave * 32, cls = first + col;
    const bool in = cls < a.n_classes, works = first < a.n_classes;
    Stationary<DP> c;
    c.load(a.w + (int64_t)cls * a.dim * 2, in, a.dim, lane);
    const int lift = lift_of<T>(w, lane);
    const float up = ldexpf(1.f, lift);

    f32x16 acc[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db) acc[db] = f32x16{};
    const int steps = (a.n_rows + kStep - 1) / kStep, each = (steps + w.splits_w - 1) / w.splits_w;
    const int begin = min(split * each, steps), end = min(begin + each, steps);
    const uint32_t row_bytes = (uint32_t)a.dim * 2;
    // Products start from log |dloss| - lse of their rows: the exponential of that is a weight with dloss in it, and only
    // a tile with negative ones has to be multiplied by signs.  A row that does not count starts from minus infinity.
    float dl = 0.f, lse = 0.f;
    int label = -1;
    auto fetch = [&](int step, int buffer) {
        const int r0 = step * kStep, n = r0 + tid;
        copy_tile<DP, kStep, kThreads>(lds + buffer * kTileBytes, a.h + (int64_t)r0 * row_bytes, row_bytes, a.n_rows - r0,
                                       a.dim, tid);
        if (tid < kStep) {
            label = n < a.n_rows ? a.labels[n] : -1;
            if (label >= a.n_classes) label = -1;
            dl = label < 0 ? 0.f : w.dloss[n] * up;
            lse = label < 0 ? 0.f : w.lse[n];
        }
    };
    auto keep = [&](int buffer) {
        if (tid < kStep) {
            start[buffer][tid] = dl == 0.f ? -INFINITY : log2_fast(fabsf(dl)) * kLn2 - lse;
            dloss[buffer][tid] = dl;
            labels[buffer][tid] = label;
            const bool any = __any(dl < 0.f);
            if (tid == 0) negative[buffer] = any;
        }
    };
    if (begin < end) {
        fetch(begin, 0);
        keep(0);
    }
    tile_arrived();
    __syncthreads();
    alternate(begin, end, 1, [&](int step, auto of) __attribute__((always_inline)) {
        constexpr int buffer = decltype(of)::value;
        const bool more = step + 1 < end;
        if (more) fetch(step + 1, buffer ^ 1);
        constexpr uint32_t tile = buffer * kTileBytes;
        if (works) {
#pragma unroll
            for (int b = 0; b < kStep; b += 32) {
                f32x16 s = scores<T, DP>(lds, tile + b * Tile<DP>::kRowBytes, c, lane, by_row(&start[buffer][b], g));
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = exp2_fast(s[i] * kLog2e);
                if (negative[buffer]) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = dloss[buffer][b + row_of(i, g)] < 0.f ? -s[i] : s[i];
                }
                if (__any((uint32_t)(labels[buffer][b + col] - first) < 32u)) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int n = b + row_of(i, g);
                        s[i] -= labels[buffer][n] == cls ? dloss[buffer][n] : 0.f;
                    }
                }
                accumulate<T, DP>(acc, lds, tile + b * Tile<DP>::kRowBytes, s, lane);   // (weights rounded to the inputs' 16 bits)
            }
        }
        if (more) keep(buffer ^ 1);
        tile_arrived();
        __syncthreads();
    });
    // Once more, without the rows that do not count: unless one that does has no numbers, which no class's sum survives.
    auto has_numbers = [&] {
        bool none = false;
#pragma unroll 1
        for (int n = begin * kStep + lane; n < min(end * kStep, a.n_rows); n += 64)
            none = none || (a.labels[n] >= 0 && a.labels[n] < a.n_classes && (w.lse[n] != w.lse[n] || w.dloss[n] != w.dloss[n]));
        return !__any(none);
    };
    if (__any(has_nan(acc)) && has_numbers()) {
#pragma unroll
        for (int db = 0; db < NB; ++db) acc[db] = f32x16{};
#pragma unroll 1
        for (int n = begin * kStep; n < min(end * kStep, a.n_rows); ++n) {
            const int label_n = a.labels[n];
            if (label_n < 0 || label_n >= a.n_classes) continue;
            const char* const row = a.h + (int64_t)n * row_bytes;
            const float z = dot_row<T, DP>(c, row, a.dim, lane);
            const float p = exp2_fast(__builtin_fmaf(z, kLog2e, -w.lse[n] * kLog2e)) - (label_n == cls ? 1.f : 0.f);
            accumulate_row<T, DP>(acc, row, p * w.dloss[n] * up, a.dim, g);
        }
    }
    const float down = ldexpf(1.f, -lift);
    if (w.splits_w > 1) {
        if (!in) return;
        float* const dst = w.part_w + ((int64_t)split * a.n_classes + cls) * a.dim;
#pragma unroll
        for (int db = 0; db < NB; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * db + row_of(i, g);
                if (d < a.dim)
                    *reinterpret_cast<f32x4*>(dst + d) = f32x4{acc[db][i] * down, acc[db][i + 1] * down,
                                                               acc[db][i + 2] * down, acc[db][i + 3] * down};
            }
        return;
    }
    store_rows<T, DP>(acc, down, false, lds + wave * 32 * Tile<DP>::kRowBytes, a.dim, lane, [&](int r) -> char* {
        return first + r < a.n_classes ? static_cast<char*>(w.dw) + (int64_t)(first + r) * a.dim * 2 : nullptr;
    });
}

// The parts of every element, in order, four elements a thread, eight loads at a time (48 parts of 863 rows of 224 elements
// 6.8 us, one load at a time 15.6).
template <class T>
__global__ __launch_bounds__(kThreads) void add_parts_kernel(const float* part, int splits, int64_t n4, void* out) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= n4) return;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < splits; ++s) sum += reinterpret_cast<const f32x4*>(part)[s * n4 + i];
    static_cast<u32x2*>(out)[i] = u32x2{pack2<T>(sum[0], sum[1]), pack2<T>(sum[2], sum[3])};
}

struct LossGradPlan {
    int64_t tiles_h, tiles_w;
    int splits_h, splits_w;
};
LossGradPlan loss_grad_plan(const LossArgs& a, int n_cu) {
    LossGradPlan p;
    p.tiles_h = (a.n_rows + 127) / 128;
    p.tiles_w = ((int64_t)a.n_classes + 127) / 128;
    const int slots = a.dim > 224 ? n_cu : 2 * n_cu;
    // A part's sums are written and read again, 8 bytes an element; a step is 4 * 64 * 128 operations an
    // element of a row on one of the slots: at 4.5 TB/s and 1.1 PFLOP/s 0.06 / slots of a step a row of sums.
    const double cost = 0.06 / slots;
    p.splits_h = parts_for(p.tiles_h, (a.n_classes + kStep - 1) / kStep, slots, 256, cost * a.n_rows);
    p.splits_w = parts_for(p.tiles_w, (a.n_rows + kStep - 1) / kStep, slots, 64, cost * a.n_classes);
    return p;
}

size_t lay_out(const LossArgs& a, const LossGradPlan& p, char* scratch, LossGradArgs* w) {
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* const here = scratch + at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    w->maxima = reinterpret_cast<float*>(take(kMaxima * sizeof(float)));
    // one after the other in one place: dh's parts are added up before dw's are written
    const size_t h = p.splits_h > 1 ? (size_t)p.splits_h * a.n_rows * a.dim * sizeof(float) : 0;
    const size_t c = p.splits_w > 1 ? (size_t)p.splits_w * a.n_classes * a.dim * sizeof(float) : 0;
    w->part_h = w->part_w = reinterpret_cast<float*>(take(h > c ? h : c));
    return at;
}

template <class T>
hipError_t add_parts(hipStream_t stream, const float* part, int splits, int64_t elements, void* out) {
    const int64_t n4 = elements / 4;
    if (!fits_a_row((n4 + kThreads - 1) / kThreads, kThreads)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(add_parts_kernel<T>, dim3((unsigned)((n4 + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, part,
                       splits, n4, out);
    return hipGetLastError();
}

template <class T, int DP>
hipError_t launch_width(hipStream_t stream, const LossArgs& a, const LossGradArgs& w, const LossGradPlan& p) {
    const size_t bytes = 2 * (size_t)kStep * Tile<DP>::kRowBytes;   // 64 KB at most
    if (!fits_a_row(p.tiles_h * p.splits_h, kThreads) || !fits_a_row(p.tiles_w * p.splits_w, kThreads)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((loss_dh_kernel<T, DP>), dim3((unsigned)(p.tiles_h * p.splits_h)), dim3(kThreads), bytes, stream, a, w);
    hipError_t rc = hipGetLastError();
    if (rc == hipSuccess && p.splits_h > 1)
        rc = add_parts<T>(stream, w.part_h, p.splits_h, (int64_t)a.n_rows * a.dim, w.dh);
    if (rc != hipSuccess) return rc;
    hipLaunchKernelGGL((loss_dw_kernel<T, DP>), dim3((unsigned)(p.tiles_w * p.splits_w)), dim3(kThreads), bytes, stream, a, w);
    rc = hipGetLastError();
    if (rc == hipSuccess && p.splits_w > 1)
        rc = add_parts<T>(stream, w.part_w, p.splits_w, (int64_t)a.n_classes * a.dim, w.dw);
    return rc;
}

template <class T>
hipError_t launch_type(hipStream_t stream, const LossArgs& a, const LossGradArgs& w, const LossGradPlan& p) {
    if (T::kNarrow) {
        hipLaunchKernelGGL(largest_kernel, dim3((unsigned)w.n_maxima), dim3(kThreads), 0, stream, a, w);
        const hipError_t rc = hipGetLastError();
        if (rc != hipSuccess) return rc;
    }
    return a.dim <= 32    ? launch_width<T, 32>(stream, a, w, p)
           : a.dim <= 64  ? launch_width<T, 64>(stream, a, w, p)
           : a.dim <= 96  ? launch_width<T, 96>(stream, a, w, p)
           : a.dim <= 128 ? launch_width<T, 128>(stream, a, w, p)
           : a.dim <= 160 ? launch_width<T, 160>(stream, a, w, p)
           : a.dim <= 192 ? launch_width<T, 192>(stream, a, w, p)
           : a.dim <= 224 ? launch_width<T, 224>(stream, a, w, p)
                          : launch_width<T, 256>(stream, a, w, p);
}

}  // namespace

size_t loss_grad_scratch_bytes(int n_cu, const LossArgs& a) {
    LossGradArgs w;
    return lay_out(a, loss_grad_plan(a, n_cu), nullptr, &w);
}

hipError_t launch_loss_grad(hipStream_t stream, int n_cu, const LossArgs& a, bool half, const float* dloss, const float* lse,
                            void* dh, void* dw, void* scratch) {
    const LossGradPlan p = loss_grad_plan(a, n_cu);
    LossGradArgs w;
    lay_out(a, p, static_cast<char*>(scratch), &w);
    w.dloss = dloss;
    w.lse = lse;
    w.dh = dh;
    w.dw = dw;
    w.splits_h = p.splits_h;
    w.splits_w = p.splits_w;
    const int blocks = (a.n_rows + kThreads - 1) / kThreads;
    w.n_maxima = blocks < kMaxima ? blocks : kMaxima;
    return half ? launch_type<Fp16>(stream, a, w, p) : launch_type<Bf16>(stream, a, w, p);
}

}  // namespace surel
