// Attention of one row a sequence to its keys in a paged cache, where few query heads share a key head: by the vector
// units, without LDS.
//
// A matrix product's 16 columns would hold one or two heads.  Here lanes hold 16 bytes of a key's row each, 64 / LPK keys at a
// time, as they come from memory: products of pairs of elements, sums over the LPK lanes of a key, and every group
// of lanes keeps the softmax and the sum over its own keys.  Groups are joined at a pair's end: halves of what two lanes hold
// are exchanged, so that each then adds half as much.
// What bounds it: memory.  16,384 caches of 1 to 64 keys, 8 heads of 64 elements, with a bias: 243 us, 4.7 TB/s read and
// written (by 32-column products 1,221, by 16-column ones 317); 512 of 100 to 8,192, 4 heads of 128: 741, 5.9 TB/s.  With three and
// four heads a key head the products are faster (12 heads to 4 of 104 elements 147 us here, 132 there; two of 128: 140, 150).
#include "cache_attention.h"
#include "kernels.h"

namespace surel {
namespace {

constexpr int kThreads = 256;
constexpr int kMostTable = 4096;   // biases of all heads by distance that are kept in LDS

__device__ __forceinline__ float dot2(Bf16, uint32_t x, uint32_t y, float c) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Bf16::x2, x), __builtin_bit_cast(Bf16::x2, y), c, false);
}
__device__ __forceinline__ float dot2(Fp16, uint32_t x, uint32_t y, float c) {
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(Fp16::x2, x), __builtin_bit_cast(Fp16::x2, y), c, false);
}

// Lanes of 16, moved: 1 and 2 inside four, 7 and 15 mirrors of eight and sixteen.
template <int CTRL>
__device__ __forceinline__ float moved(float x) { return __uint_as_float(dpp_permute<CTRL>(__float_as_uint(x))); }
template <int LPK>
__device__ __forceinline__ float sum_of_key(float x) {
    if constexpr (LPK >= 2) x += moved<0xB1>(x);
    if constexpr (LPK >= 4) x += moved<0x4E>(x);
    if constexpr (LPK >= 8) x += moved<0x141>(x);
    if constexpr (LPK >= 16) x += moved<0x140>(x);
    return x;
}
// Over the groups of lanes that are LPK apart.
template <int LPK, class Op>
__device__ __forceinline__ float over_rows_of_16(float x, Op op) {
    if constexpr (LPK <= 8) x = op(x, moved<0x128>(x));   // rotated by 8, 4, 2
    if constexpr (LPK <= 4) x = op(x, moved<0x124>(x));
    if constexpr (LPK <= 2) x = op(x, moved<0x122>(x));
    return x;
}
template <int LPK, class Op>
__device__ __forceinline__ float over_groups(float x, Op op) {
    x = over_rows_of_16<LPK>(x, op);
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t w = __float_as_uint(x);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// Sums of x and y over lanes 32 (16) apart: x's in the lower of both, y's in the upper.
__device__ __forceinline__ float halves_of_32(float x, float y) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halves_of_16(float x, float y) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Waves of a SIMD: what two tiles of keys and values and the sums of G heads leave room for in its registers.
constexpr int waves_of_a_simd(int lpk, int g) { return lpk == 16 ? 2 : lpk == 8 ? 3 : 4; }

template <class T, int LPK, int G>
__global__ __launch_bounds__(kThreads, waves_of_a_simd(LPK, G)) void cache_lanes_kernel(CacheAttention a, Share o, int in_table) {
    constexpr int kKeys = 64 / LPK, kSteps = kCacheTile / kKeys;
    extern __shared__ float table[];   // biases, see Biases
    const int lane = threadIdx.x & 63, wave = uniform((int)block_number() * (kThreads / 64) + (int)(threadIdx.x >> 6));
    const int chunk = lane % LPK, in_step = lane / LPK, col = lane & 31;
    const Biases<T> biases = {a, in_table ? table : nullptr, farthest(a)};
    if (in_table) {
        biases.fill(table);
        __syncthreads();
    }
    const int far = biases.far;
    if (wave >= o.waves) return;
    const int unit = wave % o.units, group = a.heads / a.kv_heads;   // (a unit is a key head here)
    write_empty(a, o, wave);
    const Course course = course_of(a, o, wave);
    if (course.tiles <= 0) return;

    const float c = a.scale * kLog2e;   // scores in units of log 2
    const bool mine = chunk * 8 < a.dim;
    auto look_up = [&](const Place& p) {   // the page of the tile's key of number `col`
        const int key = p.tile * kCacheTile + col;
        return key < p.length ? a.pages[(int64_t)p.seq * a.width + a.page_rows.of((uint32_t)key)] : 0;
    };
    auto fetch = [&](const Place& p, int page, u32x4 (&k)[kSteps], u32x4 (&v)[kSteps]) {
        const int key = p.tile * kCacheTile + col;
        const bool bad = page < 0 || page >= a.n_pages;
        raise_error(a.err, bad, kDevBadPage);
        const uint32_t in_page = (uint32_t)key - a.page_rows.of((uint32_t)key) * a.page_rows.d;
        const int64_t from = bad || key >= p.length ? -1 : page * a.page + (int64_t)in_page * a.row;
        const uint32_t lo = (uint32_t)from, hi = (uint32_t)(from >> 32);
        const int64_t head = (int64_t)unit * a.head + chunk * 16;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int src = s * kKeys + in_step;
            const int64_t at = (int64_t)((uint64_t)(uint32_t)__shfl((int)hi, src) << 32 | (uint32_t)__shfl((int)lo, src));
            k[s] = v[s] = u32x4{0, 0, 0, 0};
            if (mine && at >= 0) {
                k[s] = *reinterpret_cast<const u32x4*>(a.k_pages + at + head);
                v[s] = *reinterpret_cast<const u32x4*>(a.v_pages + at + head);
            }
        }
        // (which keys there are: a bit each)
        return (uint32_t)__ballot(from >= 0);
    };
    auto load_q = [&](const Place& p, u32x4 (&q)[G]) {
#pragma unroll
        for (int h = 0; h < G; ++h) {
            q[h] = u32x4{0, 0, 0, 0};
            if (mine && h < group)
                q[h] = *reinterpret_cast<const u32x4*>(a.q + (int64_t)p.seq * a.q_row + (int64_t)(unit * group + h) * a.q_head + chunk * 16);
        }
    };

    float top[G], sum[G], acc[G][8];
    u32x4 k[2][kSteps], v[2][kSteps], q[G], q_next[G];
    Place now = course.at, next = now, after;
    int64_t left = course.tiles;
    uint32_t there[2] = {0, 0};
    int page = look_up(now), page_next = 0, first_tile = 0;
    if (left > 1) next = following(a, o, now), page_next = look_up(next);
    load_q(now, q_next);
    there[0] = fetch(now, page, k[0], v[0]);
    page = page_next;
    after = next;
    bool fresh = true;

    auto turn = [&](auto of) __attribute__((always_inline)) {
        constexpr int buffer = decltype(of)::value;
        if (fresh) {
            first_tile = now.tile;
#pragma unroll
            for (int h = 0; h < G; ++h) {
                q[h] = q_next[h], top[h] = -INFINITY, sum[h] = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[h][i] = 0.f;
            }
        }
        if (left > 1) {
            if (left > 2) after = following(a, o, next), page_next = look_up(after);
            if (next.tile == 0) load_q(next, q_next);
            there[buffer ^ 1] = fetch(next, page, k[buffer ^ 1], v[buffer ^ 1]);
        }

        const uint32_t seen = there[buffer];
        const int nearest = now.length - 1 - now.tile * kCacheTile;   // distance of the tile's first key
        const bool all_far = nearest - (kCacheTile - 1) >= far;
        float p[G][kSteps];
#pragma unroll
        for (int h = 0; h < G; ++h) {
            if (h >= group) break;
            const int head = unit * group + h;
            float most = -INFINITY;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) x = dot2(T(), k[buffer][s][i], q[h][i], x);
                p[h][s] = sum_of_key<LPK>(x) * c;
            }
            if (a.bias != nullptr) {
                if (all_far) {
                    const float x = biases.at(head, far);
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) p[h][s] += x;
                } else {
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        const int d = min(max(nearest - (s * kKeys + in_step), 0), far);
                        p[h][s] += biases.at(head, d);
                    }
                }
            }
            if (seen != ~0u) {
#pragma unroll
                for (int s = 0; s < kSteps; ++s) p[h][s] = seen >> (s * kKeys + in_step) & 1 ? p[h][s] : -INFINITY;
            }
#pragma unroll
            for (int s = 0; s < kSteps; ++s) most = fmaxf(most, p[h][s]);
            if (__any(most > top[h])) {
                const float to = fmaxf(top[h], most), shrink = to == top[h] ? 1.f : exp2_fast(top[h] - to);
                top[h] = to;
                sum[h] *= shrink;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[h][i] *= shrink;
            }
            const float base = top[h] == -INFINITY ? 0.f : top[h];
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                p[h][s] = exp2_fast(p[h][s] - base);
                sum[h] += p[h][s];
            }
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x2 y = unpack2<T>(v[buffer][s][i]);
                x[2 * i] = y[0], x[2 * i + 1] = y[1];
            }
#pragma unroll
            for (int h = 0; h < G; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (h < group) acc[h][i] = __builtin_fmaf(p[h][s], x[i], acc[h][i]);
        }

        const bool ends = now.tile + 1 == now.tiles || left == 1;
        if (ends) {
            const bool part = first_tile > 0 || now.tile + 1 < now.tiles;
#pragma unroll
            for (int h = 0; h < G; ++h) {
                if (h >= group) break;
                const float most = over_groups<LPK>(top[h], [](float x, float y) { return fmaxf(x, y); });
                const float weight = top[h] == most ? 1.f : exp2_fast(top[h] - most);   // of this group's sums
                const float all = over_groups<LPK>(sum[h] * weight, [](float x, float y) { return x + y; });
                float y[4], z[2];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = halves_of_32(acc[h][i] * weight, acc[h][i + 4] * weight);
#pragma unroll
                for (int i = 0; i < 2; ++i) z[i] = over_rows_of_16<LPK>(halves_of_16(y[i], y[i + 2]), [](float x, float y) { return x + y; });
                // this lane has elements 4 (lane / 32) + 2 (lane / 16 % 2) and the next one of its chunk's
                const int d = 8 * chunk + 4 * (lane >> 5) + 2 * ((lane >> 4) & 1);
                const bool writes = mine && (lane & 15) < LPK;
                const int64_t row = (int64_t)now.seq * a.heads + unit * group + h;
                if (part) {
                    const int64_t at = ((int64_t)wave * 2 + (first_tile > 0 ? 0 : 1)) * o.columns + h;
                    if (lane == 0) o.part_ml[2 * at] = most, o.part_ml[2 * at + 1] = all;
                    if (writes) *reinterpret_cast<f32x2*>(o.part_o + at * a.dim + d) = f32x2{z[0], z[1]};
                } else {
                    if (lane == 0) a.lse[row] = (most + log2_fast(all)) * kLn2;
                    const float scale = all == 0.f ? 0.f : 1.f / all;   // all that it sees is masked by a bias, or in no page
                    if (writes)
                        static_cast<uint32_t*>(a.out)[(row * a.dim + d) / 2] = all == 0.f ? 0u : pack2<T>(z[0] * scale, z[1] * scale);
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

int lanes_a_key(int dim) { return dim <= 16 ? 2 : dim <= 32 ? 4 : dim <= 64 ? 8 : 16; }

template <class T, int LPK, int G>
hipError_t launch(hipStream_t stream, const CacheAttention& a, const Share& o) {
    const int64_t entries = a.bias == nullptr ? 0 : (int64_t)a.heads * (farthest(a) + 1);
    const bool in_table = entries > 0 && entries <= kMostTable;
    hipLaunchKernelGGL((cache_lanes_kernel<T, LPK, G>), grid_of((o.waves + kThreads / 64 - 1) / (kThreads / 64)), dim3(kThreads),
                       in_table ? entries * sizeof(float) : 0, stream, a, o, in_table ? 1 : 0);
    return hipGetLastError();
}
template <class T, int LPK>
hipError_t launch_group(hipStream_t stream, const CacheAttention& a, const Share& o) {
    const int group = a.heads / a.kv_heads;
    return group == 1 ? launch<T, LPK, 1>(stream, a, o) : launch<T, LPK, 2>(stream, a, o);
}

}  // namespace

bool lanes_serve(int group) { return group <= 2; }
int lanes_waves(int group, int dim) { return 4 * waves_of_a_simd(lanes_a_key(dim), group); }

template <class T>
hipError_t launch_lanes(hipStream_t stream, const CacheAttention& a, const Share& o) {
    switch (lanes_a_key(a.dim)) {
        case 2: return launch_group<T, 2>(stream, a, o);
        case 4: return launch_group<T, 4>(stream, a, o);
        case 8: return launch_group<T, 8>(stream, a, o);
        default: return launch_group<T, 16>(stream, a, o);
    }
}
template hipError_t launch_lanes<Bf16>(hipStream_t, const CacheAttention&, const Share&);
template hipError_t launch_lanes<Fp16>(hipStream_t, const CacheAttention&, const Share&);

}  // namespace surel
