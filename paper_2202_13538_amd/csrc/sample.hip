// Drawing a class for every row of logits (surel_sample_classes).
//
// With x_c = (max z - z_c) / T a class has the weight exp(-x_c).  What is kept of a row is the beginning of its classes
// in the order of their logits, so that a border says it all: a logit, and how many of the classes that have it (the first of
// them).  It is found without sorting.  Classes are counted, and their weights added up, in 4,095 bins of equal width in x
// (up to 64 or to the row's smallest logit); the bin that the border falls into is then looked at by its logits alone.
// Within a bin of at most 1/64 a weight is that of the bin's beginning times a short polynomial, in 64 bits, and
// weights relative to their bin's beginning are added up as whole numbers of 44 bits and more: sums are the same in whatever
// order they are made, and err by 2^-44 of a weight.  The draw itself adds weights up in 64 bits in the order of classes: by
// chunks of 512 times 16 bytes, then inside the one that u falls into.
#include "sample.h"

#include "kernels.h"
#include "matrix_tile.h"

namespace surel {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kBins = 4096;        // the last takes what counts as zero
constexpr double kFar = 64.0;      // in x: e^-64 of 2^28 classes is 2^-64 of the largest weight
constexpr int kSub = 1024;         // bins of logits inside a bin
constexpr int kList = 4096;        // logits of a bin that are kept beside one another, at most
constexpr int kChunkSlots = 512;   // 16-byte parts of a row whose weights are added up together
constexpr int kMostChunks = 1024;  // of a row that one workgroup draws from alone

struct Bf16Logit {
    static constexpr int kPer = 8, kKeyShift = 16;
    static constexpr uint32_t kNone = 0xFF80FF80u;   // minus infinity
    static __device__ __forceinline__ float at(const u32x4& x, int e) {
        return __uint_as_float(e & 1 ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16);
    }
};
struct Fp16Logit {
    static constexpr int kPer = 8, kKeyShift = 13;
    static constexpr uint32_t kNone = 0xFC00FC00u;
    static __device__ __forceinline__ float at(const u32x4& x, int e) { return unpack2<Fp16>(x[e >> 1])[e & 1]; }
};
struct Fp32Logit {
    static constexpr int kPer = 4, kKeyShift = 0;
    static constexpr uint32_t kNone = 0xFF800000u;
    static __device__ __forceinline__ float at(const u32x4& x, int e) { return __uint_as_float(x[e]); }
};

// Logits as whole numbers of the same order (both zeros alike), as narrow as their type allows, and back.
template <class L>
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);
    return (u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) >> L::kKeyShift;
}
template <class L>
__device__ __forceinline__ float logit_of(uint32_t key) {
    const uint32_t u = key << L::kKeyShift;
    return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~(u | ((1u << L::kKeyShift) - 1u)));
}

// A row in slots of 16 bytes that lie on 16-byte boundaries; its first and last slot may be filled in part.  What is not
// the row's is minus infinity.
template <class L>
struct RowOf {
    const char* base;
    int skip, end, slots, chunks;
    __device__ __forceinline__ RowOf(const SampleArgs& a, int row) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(a.logits + row * a.row);
        base = reinterpret_cast<const char*>(at & ~(uintptr_t)15);
        skip = (int)(at & 15) / (16 / L::kPer);
        end = skip + a.n_classes;
        slots = (end + L::kPer - 1) / L::kPer;
        chunks = (slots + kChunkSlots - 1) / kChunkSlots;
    }
    __device__ __forceinline__ u32x4 load(int slot) const {
        const char* const at = base + (int64_t)slot * 16;
        const int first = slot * L::kPer;
        if (first >= skip && first + L::kPer <= end) return *reinterpret_cast<const u32x4*>(at);
        u32x4 x = {L::kNone, L::kNone, L::kNone, L::kNone};
#pragma unroll
        for (int e = 0; e < L::kPer; ++e) {
            if (first + e < skip || first + e >= end) continue;
            if constexpr (L::kPer == 4) {
                x[e] = reinterpret_cast<const uint32_t*>(at)[e];
            } else {
                const uint32_t z = reinterpret_cast<const uint16_t*>(at)[e];
                x[e >> 1] = e & 1 ? (x[e >> 1] & 0xFFFFu) | z << 16 : (x[e >> 1] & 0xFFFF0000u) | z;
            }
        }
        return x;
    }
};

// The least and largest of a row's logits above minus infinity, and whether any is NaN or plus infinity.
struct Ends {
    float most, least;
    uint32_t bad;
    static __device__ __forceinline__ Ends none() { return Ends{-INFINITY, INFINITY, 0}; }
    __device__ __forceinline__ void add(float z) {
        most = fmaxf(most, z);
        least = z > -INFINITY ? fminf(least, z) : least;
        bad |= !(z < INFINITY);
    }
    __device__ __forceinline__ void add(const Ends& o) {
        most = fmaxf(most, o.most), least = fminf(least, o.least), bad |= o.bad;
    }
};

// How a row is drawn from.
struct How {
    int draws;               // 0: not at all, see `wrong`
    int wrong;
    float most;              // largest logit
    double inv_t, width, bins;   // 1 / T; a bin's, and bins of a unit of logit
    uint32_t k;              // 0: all
    double p, min_p, u;      // p of 1: all
    bool first;              // the first of the largest logits, nothing else
};

__device__ __forceinline__ How how_of(const SampleArgs& a, int row, const Ends& e) {
    How h;
    const float u = a.u[row], t = a.temperature == nullptr ? 1.f : a.temperature[row];
    const int k = a.top_k == nullptr ? 0 : a.top_k[row];
    const float p = a.top_p == nullptr ? 1.f : a.top_p[row], floor = a.min_p == nullptr ? 0.f : a.min_p[row];
    const bool fine = u >= 0.f && u < 1.f && t >= 0.f && t < INFINITY && p >= 0.f && floor >= 0.f && floor <= 1.f;
    h.wrong = !fine || e.bad;
    h.draws = !h.wrong && e.most > -INFINITY;
    h.first = t == 0.f || k == 1;
    h.most = e.most;
    h.inv_t = h.first ? 1.0 : 1.0 / (double)t;
    const double range = ((double)e.most - (double)e.least) * h.inv_t;
    h.width = range > 0.0 ? fmin(range, kFar) / (kBins - 2) : 1.0 / 64;
    h.bins = h.inv_t / h.width;
    h.k = k < 1 || k >= a.n_classes ? 0 : (uint32_t)k;
    h.p = h.first || p >= 1.f ? 1.0 : (double)p;
    h.min_p = h.first ? 0.0 : (double)floor;
    h.u = (double)u;
    return h;
}

// What a workgroup keeps of its row in LDS.
struct Bench {
    How how;
    double tens[64], ones[64];      // exp(-64 width i), exp(-width i)
    Ends ends[kWaves];
    double of_wave[kWaves];
    uint32_t counts_of_wave[kWaves];
    int hit, last;                  // what a search found, or the last that is not empty
    uint32_t before;                // counts and weights before it, and its own
    double mass_before;
    uint32_t lo, hi;
    int n_list, is_last;
};
struct Bins {
    uint64_t mass[kBins];
    uint32_t count[kBins];
};
struct SubBins {
    uint64_t mass[kSub];
    uint32_t count[kSub];
    uint32_t list[kList];
};

// What is known of a row's border.
struct Border {
    int open;                // 0: found (or there is none), 1: of the first k, 2: of p
    int alone;               // its bin has too many logits: one workgroup looks for it
    int bin;
    uint32_t before;         // classes before the bin, and their weights
    double mass_before, target;
    uint32_t key, ties;      // kept: logits above, and the first `ties` of this one
    uint32_t k_key, k_ties;  // the same of the first k alone
};

__device__ __forceinline__ double bin_weight(const Bench& l, int bin) { return l.tens[bin >> 6] * l.ones[bin & 63]; }

// exp(y), -1/64 <= y <= 0 (and a little beyond both): the next term is 2^-54.
__device__ __forceinline__ double exp_short(double y) {
    double e = __builtin_fma(y, 1.0 / 720, 1.0 / 120);
    e = __builtin_fma(e, y, 1.0 / 24);
    e = __builtin_fma(e, y, 1.0 / 6);
    e = __builtin_fma(e, y, 0.5);
    e = __builtin_fma(e, y, 1.0);
    return __builtin_fma(e, y, 1.0);
}
__device__ __forceinline__ int bin_of(const How& h, float z) {
    return (int)fmin(((double)h.most - (double)z) * h.bins, (double)(kBins - 1));
}
__device__ __forceinline__ double in_bin(const How& h, float z, int bin) {   // the weight relative to its bin's beginning
    return exp_short(__builtin_fma((double)bin, h.width, ((double)z - (double)h.most) * h.inv_t));
}
__device__ __forceinline__ double weight_of(const Bench& l, const How& h, float z) {
    const int bin = bin_of(h, z);
    return bin == kBins - 1 ? 0.0 : bin_weight(l, bin) * in_bin(h, z, bin);
}

// Weights relative to their bin's beginning as whole numbers: 2^unit of them are one.  A bin's sum stays below 2^63.
__device__ __forceinline__ int unit_of(int n_classes) { return min(62 - (32 - __clz(n_classes)), 50); }
__device__ __forceinline__ uint64_t whole(double w, double one) {   // rounded, by a sum whose last place is 1
    return (uint64_t)__double_as_longlong(__builtin_fma(w, one, 0x1p52)) - 0x4330000000000000ull;
}

__device__ __forceinline__ void add_count(uint32_t* at, uint32_t n) {
    (void)__hip_atomic_fetch_add(at, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
__device__ __forceinline__ void add_mass(uint64_t* at, uint64_t x) {
    (void)__hip_atomic_fetch_add(at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// Sums over the workgroup of what its threads before this one have; *all: of all threads.
__device__ __forceinline__ uint32_t counts_before(Bench& l, uint32_t mine, uint32_t* all) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint32_t x = wave_incl_sum(mine);
    __syncthreads();
    if (lane == 63) l.counts_of_wave[wave] = x;
    __syncthreads();
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t y = l.counts_of_wave[w];
        before += w < wave ? y : 0;
        total += y;
    }
    *all = total;
    return before + x - mine;
}
__device__ __forceinline__ double masses_before(Bench& l, double mine, double* all) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    double x = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    const double till = __shfl_up(x, 1);
    __syncthreads();
    if (lane == 63) l.of_wave[wave] = x;
    __syncthreads();
    double before = 0.0, total = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const double y = l.of_wave[w];
        if (w < wave) before += y;
        total += y;
    }
    *all = total;
    return before + (lane == 0 ? 0.0 : till);
}

// The workgroup's bench for a row whose ends every thread has a part of.
__device__ __forceinline__ void set_up(Bench& l, const SampleArgs& a, int row, Ends e) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        Ends o;
        o.most = __shfl_xor(e.most, m), o.least = __shfl_xor(e.least, m), o.bad = __shfl_xor(e.bad, m);
        e.add(o);
    }
    if ((threadIdx.x & 63) == 0) l.ends[threadIdx.x >> 6] = e;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) e.add(l.ends[w]);
        l.how = how_of(a, row, e);
    }
    __syncthreads();
    const int i = threadIdx.x;
    if (i < 64) l.tens[i] = exp(-64.0 * l.how.width * i);
    else if (i < 128) l.ones[i - 64] = exp(-l.how.width * (i - 64));
    __syncthreads();
}

// The first of BINS bins up to which counts reach k, or (by_mass) weights reach the target.  Leaves in l.hit which, or -1,
// and in l.before and l.mass_before what comes before it, on top of what is given.  mass null: weights are not asked for.
template <int BINS, class Factor>
__device__ __forceinline__ void search(Bench& l, const uint32_t* count, const uint64_t* mass, bool by_mass, uint32_t k, double target,
                                       uint32_t before, double mass_before, double* total, Factor factor) {
    constexpr int kEach = BINS / kThreads;
    const int first = threadIdx.x * kEach;
    uint32_t n = 0, all;
    double w = 0.0, all_w = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        n += count[first + e];
        if (mass != nullptr) w += (double)mass[first + e] * factor(first + e);
    }
    if (threadIdx.x == 0) l.hit = 0x7FFFFFFF, l.last = -1;
    uint32_t till = before + counts_before(l, n, &all);
    double till_w = mass == nullptr ? 0.0 : mass_before + masses_before(l, w, &all_w);
    if (total != nullptr) *total = mass_before + all_w;
    uint32_t my_till = till;
    double my_till_w = till_w;
    int mine = -1, full = -1;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint32_t c = count[first + e];
        const double m = mass == nullptr ? 0.0 : (double)mass[first + e] * factor(first + e);
        const bool there = by_mass ? till_w + m >= target : till + c >= k;
        if (c != 0) full = first + e;
        if (mine < 0 && there && c != 0) mine = first + e, my_till = till, my_till_w = till_w;
        till += c, till_w += m;
    }
    if (mine >= 0) atomicMin(&l.hit, mine);
    if (by_mass && full >= 0) atomicMax(&l.last, full);
    __syncthreads();
    if (l.hit == 0x7FFFFFFF) {   // (sums in another order: the weights' last places)
        if (full >= 0 && full == l.last) {
            mine = full;
            my_till = till, my_till_w = till_w;   // up to the thread's end, from where empty bins and the last one go off again
            my_till -= count[full], my_till_w -= mass == nullptr ? 0.0 : (double)mass[full] * factor(full);
        }
    } else if (mine != l.hit) {
        mine = -1;
    }
    __syncthreads();
    if (mine >= 0) l.hit = mine, l.before = my_till, l.mass_before = my_till_w;
    if (threadIdx.x == 0 && l.hit == 0x7FFFFFFF && l.last < 0) l.hit = -1;
    __syncthreads();
}

// Where the border lies among the bins: of the first k, then of p.
__device__ __forceinline__ void start_border(Border* b) {
    b->open = 0, b->alone = 0, b->bin = -1, b->before = 0, b->mass_before = b->target = 0.0;
    b->key = b->k_key = 0, b->ties = b->k_ties = 0xFFFFFFFFu;
}
__device__ __forceinline__ void open_p(Bench& l, const Bins& bins, Border* b, double of, double one) {
    const double target = l.how.p * of;
    search<kBins>(l, bins.count, bins.mass, true, 0, target, 0, 0.0, nullptr, [&](int i) { return bin_weight(l, i) * one; });
    if (threadIdx.x == 0) b->open = 2, b->bin = l.hit, b->before = l.before, b->mass_before = l.mass_before, b->target = target;
    __syncthreads();
}
__device__ __forceinline__ void open_border(Bench& l, const Bins& bins, Border* b, int n_classes) {
    const double one = ldexp(1.0, -unit_of(n_classes));
    const bool by_p = l.how.p < 1.0;
    auto factor = [&](int i) { return bin_weight(l, i) * one; };
    if (threadIdx.x == 0) start_border(b);
    __syncthreads();
    double total = 0.0;
    // (without a k no count reaches it: the weights' sum is what is asked for)
    search<kBins>(l, bins.count, by_p ? bins.mass : nullptr, false, l.how.k != 0 ? l.how.k : 0xFFFFFFFFu, 0.0, 0, 0.0, &total, factor);
    const int hit = l.hit;
    __syncthreads();
    if (hit >= 0) {
        if (threadIdx.x == 0) b->open = 1, b->bin = hit, b->before = l.before, b->mass_before = l.mass_before;
        __syncthreads();
    } else if (by_p) {
        open_p(l, bins, b, total, one);
    }
}

// The border among the logits of its bin, which each() goes through; every thread takes some.
template <class L, class Each>
__device__ __forceinline__ void find_border(Bench& l, SubBins& sub, Border* b, int n_classes, Each each) {
    const How& how = l.how;
    const int unit = unit_of(n_classes);
    const double one = ldexp(1.0, unit), back = ldexp(1.0, -unit);
    const bool by_p = b->open == 2, masses = how.p < 1.0;
    const int bin = b->bin;
    const double of_bin = bin_weight(l, bin) * back;
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    each([&](uint32_t key) { lo = min(lo, key), hi = max(hi, key); });
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) lo = min(lo, (uint32_t)__shfl_xor((int)lo, m)), hi = max(hi, (uint32_t)__shfl_xor((int)hi, m));
    if (threadIdx.x == 0) l.lo = 0xFFFFFFFFu, l.hi = 0;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) atomicMin(&l.lo, lo), atomicMax(&l.hi, hi);
    __syncthreads();
    lo = l.lo, hi = l.hi;
    uint32_t before = b->before;
    double mass_before = b->mass_before;
    const double target = b->target;
    for (;;) {
        const int shift = max(32 - (int)__clz(hi - lo) - 10, 0);   // (hi - lo) >> shift is below kSub
        for (int i = threadIdx.x; i < kSub; i += kThreads) sub.count[i] = 0, sub.mass[i] = 0;
        __syncthreads();
        each([&](uint32_t key) {
            if (key < lo || key > hi) return;
            const uint32_t i = (hi - key) >> shift;
            add_count(&sub.count[i], 1);
            if (masses) add_mass(&sub.mass[i], whole(in_bin(how, logit_of<L>(key), bin), one));
        });
        __syncthreads();
        search<kSub>(l, sub.count, masses ? sub.mass : nullptr, by_p, how.k, target, before, mass_before, nullptr, [&](int) { return of_bin; });
        if (l.hit < 0) break;   // (of a bin that has logits, one is found)
        before = l.before, mass_before = l.mass_before;
        const uint32_t top = hi - ((uint32_t)l.hit << shift);
        if (shift == 0) {
            if (threadIdx.x == 0) {
                const uint32_t n = sub.count[l.hit];
                const double w = weight_of(l, how, logit_of<L>(top));
                b->key = top;
                if (by_p) {
                    const double need = ceil((target - mass_before) / w);
                    b->ties = (uint32_t)fmin(fmax(need, 1.0), (double)n);
                    if (b->key == b->k_key) b->ties = min(b->ties, b->k_ties);
                } else {
                    b->ties = how.k - before;
                    b->k_key = b->key, b->k_ties = b->ties;
                    b->target = mass_before + (double)b->ties * w;   // what the first k weigh
                }
            }
            break;
        }
        hi = top;
        lo = max(lo, top - ((1u << shift) - 1u));
        __syncthreads();
    }
    if (threadIdx.x == 0) b->open = 0;
    __syncthreads();
}

// Weights of a chunk above the border, and how many classes lie on it.  One wave.
struct Drawn {
    float at;          // the border's logit
    double floor;      // least weight that is kept
};
__device__ __forceinline__ double kept_weight(const Bench& l, const How& h, const Drawn& d, float z) {
    if (!(z > d.at)) return 0.0;
    const double w = weight_of(l, h, z);
    return w >= d.floor ? w : 0.0;
}
template <class L>
__device__ __forceinline__ void chunk_sums(const Bench& l, const How& h, const RowOf<L>& r, const Drawn& d, int chunk, double* mass,
                                           uint32_t* ties) {
    const int lane = threadIdx.x & 63;
    double w = 0.0;
    uint32_t n = 0;
#pragma unroll 2
    for (int i = 0; i < kChunkSlots / 64; ++i) {
        const int slot = chunk * kChunkSlots + i * 64 + lane;
        if (slot >= r.slots) break;
        const u32x4 x = r.load(slot);
#pragma unroll
        for (int e = 0; e < L::kPer; ++e) {
            const float z = L::at(x, e);
            w += kept_weight(l, h, d, z);
            n += z == d.at;
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) w += __shfl_xor(w, m), n += __shfl_xor((int)n, m);
    *mass = w, *ties = n;
}

// The class, from the chunks' sums.
template <class L, class Mass, class Ties>
__device__ __forceinline__ void choose(Bench& l, const SampleArgs& a, int row, const RowOf<L>& r, const Drawn& d, uint32_t most_ties,
                                       Mass mass_of, Ties ties_of) {
    const How& h = l.how;
    const double on = weight_of(l, h, d.at);         // of a class on the border
    const uint32_t kept = on >= d.floor ? most_ties : 0;
    const int per = (r.chunks + kThreads - 1) / kThreads, first = threadIdx.x * per, end = min(first + per, r.chunks);
    uint32_t n = 0, all_n;
    for (int c = first; c < end; ++c) n += ties_of(c);
    uint32_t ties = counts_before(l, n, &all_n);
    auto of_chunk = [&](int c, uint32_t before) {
        const uint32_t n = min(before + ties_of(c), kept) - min(before, kept);
        return __builtin_fma((double)n, on, mass_of(c));
    };
    double w = 0.0, total;
    uint32_t t = ties;
    for (int c = first; c < end; ++c) w += of_chunk(c, t), t += ties_of(c);
    double till = masses_before(l, w, &total);
    const double target = h.u * total;
    if (threadIdx.x == 0) l.hit = 0x7FFFFFFF, l.last = -1;
    __syncthreads();
    double my_till = 0.0;
    uint32_t my_ties = 0;
    int mine = -1, full = -1;
    double full_till = 0.0;
    uint32_t full_ties = 0;
    for (int c = first; c < end; ++c) {
        const double m = of_chunk(c, ties);
        if (m > 0.0) {
            full = c, full_till = till, full_ties = ties;
            if (mine < 0 && till + m > target) mine = c, my_till = till, my_ties = ties;
        }
        till += m, ties += ties_of(c);
    }
    if (mine >= 0) atomicMin(&l.hit, mine);
    if (full >= 0) atomicMax(&l.last, full);
    __syncthreads();
    const int chunk = l.hit != 0x7FFFFFFF ? l.hit : l.last;   // (by the sums' last places u may lie behind them all)
    __syncthreads();
    if (mine == chunk) l.mass_before = my_till, l.before = my_ties;
    else if (full == chunk) l.mass_before = full_till, l.before = full_ties;
    if (threadIdx.x == 0) l.hit = 0x7FFFFFFF, l.last = -1;
    __syncthreads();
    till = l.mass_before;
    const uint32_t ties0 = l.before;
    if (chunk < 0) return;   // (the largest logit is always kept)

    // inside the chunk, a slot a thread
    const int slot = chunk * kChunkSlots + threadIdx.x;
    const u32x4 x = slot < r.slots ? r.load(slot) : u32x4{L::kNone, L::kNone, L::kNone, L::kNone};
    uint32_t on_it = 0, unused;
#pragma unroll
    for (int e = 0; e < L::kPer; ++e) on_it += L::at(x, e) == d.at;
    ties = ties0 + counts_before(l, on_it, &unused);
    double each[L::kPer], mass = 0.0, unused_mass;
#pragma unroll
    for (int e = 0; e < L::kPer; ++e) {
        const float z = L::at(x, e);
        each[e] = kept_weight(l, h, d, z);
        if (z == d.at) each[e] = ties++ < kept ? on : 0.0;
        mass += each[e];
    }
    till += masses_before(l, mass, &unused_mass);
    int found = -1, last = -1;
    double found_w = 0.0, last_w = 0.0;
#pragma unroll
    for (int e = 0; e < L::kPer; ++e) {
        till += each[e];
        if (each[e] > 0.0) {
            last = slot * L::kPer + e, last_w = each[e];
            if (found < 0 && till > target) found = last, found_w = each[e];
        }
    }
    if (found >= 0) atomicMin(&l.hit, found);
    if (last >= 0) atomicMax(&l.last, last);
    __syncthreads();
    const int chosen = l.hit != 0x7FFFFFFF ? l.hit : l.last;
    if (chosen >= 0 && (found == chosen || (l.hit == 0x7FFFFFFF && last == chosen))) {
        a.chosen[row] = chosen - r.skip;
        a.logp[row] = (float)log((found == chosen ? found_w : last_w) / total);
    }
}

__device__ __forceinline__ void no_class(const Bench& l, const SampleArgs& a, int row) {
    if (threadIdx.x != 0) return;
    a.chosen[row] = -1;
    a.logp[row] = -INFINITY;
    if (l.how.wrong) atomicOr(a.err, kDevBadChoice);
}
__device__ __forceinline__ bool has_border(const How& h) { return !h.first && (h.k != 0 || h.p < 1.0); }

// Goes through the slots begin .. end - 1 of a row.
template <class L, class Do>
__device__ __forceinline__ void each_logit(const RowOf<L>& r, int begin, int end, Do act) {
#pragma unroll 2
    for (int s = begin + (int)threadIdx.x; s < end; s += kThreads) {
        const u32x4 x = r.load(s);
#pragma unroll
        for (int e = 0; e < L::kPer; ++e) act(L::at(x, e));
    }
}
template <class L>
__device__ __forceinline__ void count_bins(const Bench& l, Bins& bins, const RowOf<L>& r, int begin, int end, double one) {
    const How how = l.how;
    const bool masses = how.p < 1.0;
    each_logit<L>(r, begin, end, [&](float z) {
        const int b = bin_of(how, z);
        if (b == kBins - 1) return;
        add_count(&bins.count[b], 1);
        if (masses) add_mass(&bins.mass[b], whole(in_bin(how, z, b), one));
    });
}
// Keys of a bin's logits, kept at `put(key)`.
template <class L, class Put>
__device__ __forceinline__ void bin_keys(const How& how, const RowOf<L>& r, int begin, int end, int bin, Put put) {
    each_logit<L>(r, begin, end, [&](float z) {
        if (bin_of(how, z) == bin) put(key_of<L>(z));
    });
}

// A row's border once its bin is known, by one workgroup: from a list of the bin's logits if that holds them, or by the row.
template <class L>
__device__ __forceinline__ void find_in_row(Bench& l, SubBins& sub, Border* b, const RowOf<L>& r, int n_classes) {
    if (threadIdx.x == 0) l.n_list = 0;
    __syncthreads();
    const int bin = b->bin;
    const How how = l.how;
    bin_keys<L>(how, r, 0, r.slots, bin, [&](uint32_t key) {
        const int at = atomicAdd(&l.n_list, 1);
        if (at < kList) sub.list[at] = key;
    });
    __syncthreads();
    const int n = l.n_list;
    if (n <= kList) {
        find_border<L>(l, sub, b, n_classes, [&](auto act) {
            for (int i = threadIdx.x; i < n; i += kThreads) act(sub.list[i]);
        });
    } else {
        find_border<L>(l, sub, b, n_classes, [&](auto act) { bin_keys<L>(how, r, 0, r.slots, bin, act); });
    }
}
template <class L>
__device__ __forceinline__ void find_all_in_row(Bench& l, Bins& bins, SubBins& sub, Border* b, const RowOf<L>& r, int n_classes) {
    const int open = b->open;
    if (open == 0) return;
    find_in_row<L>(l, sub, b, r, n_classes);
    if (open == 1 && l.how.p < 1.0) {
        open_p(l, bins, b, b->target, ldexp(1.0, -unit_of(n_classes)));
        find_in_row<L>(l, sub, b, r, n_classes);
    }
}

template <class L>
__device__ __forceinline__ Drawn drawn_by(const How& h, const Border& b) {
    Drawn d;
    d.at = h.first ? h.most : b.key == 0 ? -INFINITY : logit_of<L>(b.key);
    d.floor = h.min_p;
    return d;
}

// One workgroup a row, all of it.
struct RowLds {
    Bench bench;
    Border border;
    double mass[kMostChunks];
    uint32_t ties[kMostChunks];
};
template <class L>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(SampleArgs a) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ RowLds l;
    const int64_t place = block_number();
    if (place >= a.n_rows) return;
    const int row = (int)place;
    const RowOf<L> r(a, row);
    Ends ends = Ends::none();
    each_logit<L>(r, 0, r.slots, [&](float z) { ends.add(z); });
    set_up(l.bench, a, row, ends);
    const How how = l.bench.how;
    if (!how.draws) {
        no_class(l.bench, a, row);
        return;
    }
    if (threadIdx.x == 0) start_border(&l.border);
    if (has_border(how)) {
        Bins& bins = *reinterpret_cast<Bins*>(dynamic);
        SubBins& sub = *reinterpret_cast<SubBins*>(dynamic + sizeof(Bins));
        for (int i = threadIdx.x; i < kBins; i += kThreads) bins.count[i] = 0, bins.mass[i] = 0;
        __syncthreads();
        count_bins<L>(l.bench, bins, r, 0, r.slots, ldexp(1.0, unit_of(a.n_classes)));
        __syncthreads();
        open_border(l.bench, bins, &l.border, a.n_classes);
        find_all_in_row<L>(l.bench, bins, sub, &l.border, r, a.n_classes);
    }
    __syncthreads();
    const Drawn d = drawn_by<L>(how, l.border);
    for (int c = threadIdx.x >> 6; c < r.chunks; c += kWaves) {
        double mass;
        uint32_t ties;
        chunk_sums<L>(l.bench, how, r, d, c, &mass, &ties);
        if ((threadIdx.x & 63) == 0) l.mass[c] = mass, l.ties[c] = ties;
    }
    __syncthreads();
    choose<L>(l.bench, a, row, r, d, how.first ? 1u : l.border.ties, [&](int c) { return l.mass[c]; }, [&](int c) { return l.ties[c]; });
}

// Rows in parts.
struct Parts {
    int parts = 1, chunks = 0, each = 0;   // of a row: workgroups, chunks at most, chunks of a part
    Ends* ends = nullptr;                  // [rows][parts]
    uint32_t* turns = nullptr;             // [rows][4]: workgroups of a step that are done, and how long the list is
    Border* border = nullptr;              // [rows]
    Bins* bins = nullptr;                  // [rows]
    uint32_t* list = nullptr;              // [rows][kList]
    uint64_t* mass = nullptr;              // [rows][chunks]
    uint32_t* ties = nullptr;              // [rows][chunks]
};
enum { kBinTurn = 0, kListTurn = 1, kDrawTurn = 2, kListed = 3 };

// Words that other workgroups read or write in the same launch: past the caches in between.
template <class X>
__device__ __forceinline__ void put(X* at, X x) { __hip_atomic_store(at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <class X>
__device__ __forceinline__ X get(const X* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <class X>
__device__ __forceinline__ X add_far(X* at, X x) { return __hip_atomic_fetch_add(at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Whether this workgroup is the last of its row's to come here.
__device__ __forceinline__ bool last_of(Bench& l, uint32_t* turn, int parts) {
    wait_memory();
    __syncthreads();
    if (threadIdx.x == 0) l.is_last = add_far(turn, 1u) == (uint32_t)parts - 1;
    __syncthreads();
    return l.is_last != 0;
}

struct Part {
    int row, part, begin, end, chunk_begin, chunk_end;   // slots; chunks
};
template <class L>
__device__ __forceinline__ Part part_of(const Parts& p, const RowOf<L>& r, int row, int part) {
    Part x;
    x.row = row, x.part = part;
    x.chunk_begin = min(part * p.each, r.chunks), x.chunk_end = min(x.chunk_begin + p.each, r.chunks);
    x.begin = min(x.chunk_begin * kChunkSlots, r.slots), x.end = min(x.chunk_end * kChunkSlots, r.slots);
    return x;
}
__device__ __forceinline__ void set_up_from_parts(Bench& l, const SampleArgs& a, const Parts& p, int row) {
    Ends e = Ends::none();
    for (int i = threadIdx.x; i < p.parts; i += kThreads) e.add(p.ends[(int64_t)row * p.parts + i]);
    set_up(l, a, row, e);
}

template <class L>
__global__ __launch_bounds__(kThreads) void sample_ends_kernel(SampleArgs a, Parts p) {
    __shared__ Ends ends[kWaves];
    const int64_t block = block_number();
    const int row = (int)(block / p.parts), part = (int)(block % p.parts);
    if (row >= a.n_rows) return;
    const RowOf<L> r(a, row);
    const Part x = part_of(p, r, row, part);
    if (part == 0 && threadIdx.x < 4) p.turns[4 * row + threadIdx.x] = 0;
    if (p.bins != nullptr)
        for (int i = part * kThreads + threadIdx.x; i < kBins; i += p.parts * kThreads) p.bins[row].count[i] = 0, p.bins[row].mass[i] = 0;
    Ends e = Ends::none();
    each_logit<L>(r, x.begin, x.end, [&](float z) { e.add(z); });
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        Ends o;
        o.most = __shfl_xor(e.most, m), o.least = __shfl_xor(e.least, m), o.bad = __shfl_xor(e.bad, m);
        e.add(o);
    }
    if ((threadIdx.x & 63) == 0) ends[threadIdx.x >> 6] = e;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kWaves; ++w) e.add(ends[w]);
    p.ends[(int64_t)row * p.parts + part] = e;
}

template <class L>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a, Parts p) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ Bench l;
    const int64_t block = block_number();
    const int row = (int)(block / p.parts), part = (int)(block % p.parts);
    if (row >= a.n_rows) return;
    set_up_from_parts(l, a, p, row);
    if (!l.how.draws || !has_border(l.how)) {
        if (part == 0 && threadIdx.x == 0) start_border(&p.border[row]);
        return;
    }
    const RowOf<L> r(a, row);
    const Part x = part_of(p, r, row, part);
    Bins& bins = *reinterpret_cast<Bins*>(dynamic);
    for (int i = threadIdx.x; i < kBins; i += kThreads) bins.count[i] = 0, bins.mass[i] = 0;
    __syncthreads();
    count_bins<L>(l, bins, r, x.begin, x.end, ldexp(1.0, unit_of(a.n_classes)));
    __syncthreads();
    const bool masses = l.how.p < 1.0;
    Bins& all = p.bins[row];
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
        if (bins.count[i] == 0) continue;
        (void)add_far(&all.count[i], bins.count[i]);
        if (masses) (void)add_far(&all.mass[i], bins.mass[i]);
    }
    if (!last_of(l, &p.turns[4 * row + kBinTurn], p.parts)) return;
    for (int i = threadIdx.x; i < kBins; i += kThreads) bins.count[i] = get(&all.count[i]), bins.mass[i] = get(&all.mass[i]);
    __syncthreads();
    open_border(l, bins, &p.border[row], a.n_classes);
}

// The border among its bin's logits, which all parts put into a list; the last part looks through it.
template <class L>
__global__ __launch_bounds__(kThreads) void sample_list_kernel(SampleArgs a, Parts p) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ Bench l;
    __shared__ Border b;
    const int64_t block = block_number();
    const int row = (int)(block / p.parts), part = (int)(block % p.parts);
    if (row >= a.n_rows) return;
    const int open = p.border[row].open;
    if (open == 0 || p.border[row].alone != 0) return;   // (no part of the row has changed that yet)
    set_up_from_parts(l, a, p, row);
    const RowOf<L> r(a, row);
    const Part x = part_of(p, r, row, part);
    const int bin = p.border[row].bin;
    uint32_t* const list = p.list + (int64_t)row * kList;
    bin_keys<L>(l.how, r, x.begin, x.end, bin, [&](uint32_t key) {
        const uint32_t at = add_far(&p.turns[4 * row + kListed], 1u);
        if (at < kList) put(&list[at], key);
    });
    if (!last_of(l, &p.turns[4 * row + kListTurn], p.parts)) return;
    const uint32_t n = get(&p.turns[4 * row + kListed]);
    if (threadIdx.x == 0) b = p.border[row];
    __syncthreads();
    if (n > (uint32_t)kList) {
        if (threadIdx.x == 0) p.border[row].alone = 1;
        return;
    }
    Bins& bins = *reinterpret_cast<Bins*>(dynamic);
    SubBins& sub = *reinterpret_cast<SubBins*>(dynamic + sizeof(Bins));
    for (int i = threadIdx.x; i < (int)n; i += kThreads) sub.list[i] = get(&list[i]);
    __syncthreads();
    find_border<L>(l, sub, &b, a.n_classes, [&](auto act) {
        for (int i = threadIdx.x; i < (int)n; i += kThreads) act(sub.list[i]);
    });
    if (open == 1 && l.how.p < 1.0) {
        const Bins& all = p.bins[row];
        for (int i = threadIdx.x; i < kBins; i += kThreads) bins.count[i] = all.count[i], bins.mass[i] = all.mass[i];
        __syncthreads();
        open_p(l, bins, &b, b.target, ldexp(1.0, -unit_of(a.n_classes)));
    }
    if (threadIdx.x == 0) {
        p.border[row] = b;
        p.turns[4 * row + kListTurn] = 0, p.turns[4 * row + kListed] = 0;
    }
}

// Rows whose bin holds more logits than the list: a workgroup each.
template <class L>
__global__ __launch_bounds__(kThreads) void sample_alone_kernel(SampleArgs a, Parts p) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ Bench l;
    __shared__ Border b;
    const int64_t place = block_number();
    if (place >= a.n_rows || p.border[place].alone == 0) return;
    const int row = (int)place;
    set_up_from_parts(l, a, p, row);
    const RowOf<L> r(a, row);
    Bins& bins = *reinterpret_cast<Bins*>(dynamic);
    SubBins& sub = *reinterpret_cast<SubBins*>(dynamic + sizeof(Bins));
    for (int i = threadIdx.x; i < kBins; i += kThreads) bins.count[i] = p.bins[row].count[i], bins.mass[i] = p.bins[row].mass[i];
    if (threadIdx.x == 0) b = p.border[row];
    __syncthreads();
    find_all_in_row<L>(l, bins, sub, &b, r, a.n_classes);
    if (threadIdx.x == 0) p.border[row] = b;
}

template <class L>
__global__ __launch_bounds__(kThreads) void sample_draw_kernel(SampleArgs a, Parts p) {
    __shared__ Bench l;
    const int64_t block = block_number();
    const int row = (int)(block / p.parts), part = (int)(block % p.parts);
    if (row >= a.n_rows) return;
    set_up_from_parts(l, a, p, row);
    const How how = l.how;
    if (!how.draws) {
        if (part == 0) no_class(l, a, row);
        return;
    }
    const RowOf<L> r(a, row);
    const Part x = part_of(p, r, row, part);
    Border b;
    if (has_border(how)) b = p.border[row];
    else start_border(&b);
    const Drawn d = drawn_by<L>(how, b);
    uint64_t* const masses = p.mass + (int64_t)row * p.chunks;
    uint32_t* const ties = p.ties + (int64_t)row * p.chunks;
    for (int c = x.chunk_begin + (threadIdx.x >> 6); c < x.chunk_end; c += kWaves) {
        double mass;
        uint32_t n;
        chunk_sums<L>(l, how, r, d, c, &mass, &n);
        if ((threadIdx.x & 63) == 0) put(&masses[c], (uint64_t)__double_as_longlong(mass)), put(&ties[c], n);
    }
    if (!last_of(l, &p.turns[4 * row + kDrawTurn], p.parts)) return;
    choose<L>(l, a, row, r, d, how.first ? 1u : b.ties, [&](int c) { return __longlong_as_double((long long)get(&masses[c])); },
              [&](int c) { return get(&ties[c]); });
}

struct Plan {
    Parts p;
    bool in_rows = false, borders = false;
    int lists = 0;
    size_t at[8] = {}, bytes = 0;
};
Plan plan_of(int n_cu, const SampleArgs& a, int type) {
    Plan x;
    const int per = type == 2 ? 4 : 8;
    x.p.chunks = ((a.n_classes + per - 1) / per + 1 + kChunkSlots - 1) / kChunkSlots;   // (one slot more where a row starts inside one)
    x.borders = a.top_k != nullptr || a.top_p != nullptr;
    x.lists = (a.top_k != nullptr ? 1 : 0) + (a.top_p != nullptr ? 1 : 0);
    // A workgroup a row where rows fill the device, or are so short that one goes over them as soon as several would.
    x.in_rows = x.p.chunks <= kMostChunks && (a.n_rows >= n_cu || x.p.chunks <= 8);
    if (x.in_rows) return x;
    const int64_t wanted = (3 * (int64_t)n_cu + a.n_rows - 1) / a.n_rows;
    x.p.parts = (int)(wanted < x.p.chunks ? wanted : x.p.chunks);
    x.p.each = (x.p.chunks + x.p.parts - 1) / x.p.parts;
    x.p.parts = (x.p.chunks + x.p.each - 1) / x.p.each;
    const size_t rows = (size_t)a.n_rows;
    const size_t sizes[7] = {rows * x.p.parts * sizeof(Ends), rows * 16, x.borders ? rows * sizeof(Border) : 0,
                             x.borders ? rows * sizeof(Bins) : 0, x.borders ? rows * kList * 4 : 0, rows * x.p.chunks * 8,
                             rows * x.p.chunks * 4};
    for (int i = 0; i < 7; ++i) x.at[i + 1] = x.at[i] + (sizes[i] + 255) / 256 * 256;
    x.bytes = x.at[7];
    return x;
}

template <class Kernel>
hipError_t allow(Kernel kernel, size_t bytes) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <class L>
hipError_t launch_type(hipStream_t stream, const SampleArgs& a, const Plan& x) {
    const size_t lds = sizeof(Bins) + sizeof(SubBins);
    hipError_t rc = hipSuccess;
    if (x.in_rows) {
        if ((rc = allow(sample_row_kernel<L>, lds)) != hipSuccess) return rc;
        hipLaunchKernelGGL(sample_row_kernel<L>, grid_of(a.n_rows), dim3(kThreads), x.borders ? lds : 0, stream, a);
        return hipGetLastError();
    }
    const dim3 grid = grid_of((int64_t)a.n_rows * x.p.parts);
    hipLaunchKernelGGL(sample_ends_kernel<L>, grid, dim3(kThreads), 0, stream, a, x.p);
    if ((rc = hipGetLastError()) != hipSuccess) return rc;
    if (x.borders) {
        if ((rc = allow(sample_bins_kernel<L>, sizeof(Bins))) != hipSuccess || (rc = allow(sample_list_kernel<L>, lds)) != hipSuccess ||
            (rc = allow(sample_alone_kernel<L>, lds)) != hipSuccess)
            return rc;
        hipLaunchKernelGGL(sample_bins_kernel<L>, grid, dim3(kThreads), sizeof(Bins), stream, a, x.p);
        for (int i = 0; i < x.lists; ++i) hipLaunchKernelGGL(sample_list_kernel<L>, grid, dim3(kThreads), lds, stream, a, x.p);
        hipLaunchKernelGGL(sample_alone_kernel<L>, grid_of(a.n_rows), dim3(kThreads), lds, stream, a, x.p);
        if ((rc = hipGetLastError()) != hipSuccess) return rc;
    }
    hipLaunchKernelGGL(sample_draw_kernel<L>, grid, dim3(kThreads), 0, stream, a, x.p);
    return hipGetLastError();
}

}  // namespace

size_t sample_scratch_bytes(int n_cu, const SampleArgs& a, int type) { return plan_of(n_cu, a, type).bytes; }

hipError_t launch_sample(hipStream_t stream, int n_cu, const SampleArgs& a, int type, void* scratch) {
    Plan x = plan_of(n_cu, a, type);
    char* const s = static_cast<char*>(scratch);
    if (!x.in_rows) {
        x.p.ends = reinterpret_cast<Ends*>(s + x.at[0]);
        x.p.turns = reinterpret_cast<uint32_t*>(s + x.at[1]);
        x.p.border = x.borders ? reinterpret_cast<Border*>(s + x.at[2]) : nullptr;
        x.p.bins = x.borders ? reinterpret_cast<Bins*>(s + x.at[3]) : nullptr;
        x.p.list = x.borders ? reinterpret_cast<uint32_t*>(s + x.at[4]) : nullptr;
        x.p.mass = reinterpret_cast<uint64_t*>(s + x.at[5]);
        x.p.ties = reinterpret_cast<uint32_t*>(s + x.at[6]);
    }
    return type == 0 ? launch_type<Bf16Logit>(stream, a, x) : type == 1 ? launch_type<Fp16Logit>(stream, a, x)
                                                                        : launch_type<Fp32Logit>(stream, a, x);
}

}  // namespace surel
