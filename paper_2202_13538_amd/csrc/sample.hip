// Drawing a class for every row of logits (surel_sample_classes).
//
// With x_c = (max z - z_c) / T a class has the weight exp(-x_c).  What is kept of a row is the beginning of its classes
// in the order of their logits, so that a border says it all: a logit, and how many of the classes that have it (the first of
// them).  It is found without sorting.  Classes are counted in 4,095 bins of equal width in x (up to 64 or to the row's smallest
// logit), and how far they lie inside them is added up.  Counts say which bin the k-th class is in; a bin's weights, by their
// expansion up to that first moment, are known to h^2 of them (h its width, 1/64 at most), so that the border of top_p lies
// in one of few bins.  The logits of these are put into a list, the weights before
// them added up, and the border found in the list.  There weights are whole numbers of two words relative to the list's
// largest, so that their sums are the same in whatever order they are made.
// The draw adds weights up in 64 bits in the order of classes: by chunks, then inside the one that u falls into.
// What bounds it: for many rows the exponentials of what is kept and the barriers of a row (4,096 rows of 10,001 classes by
// min-p 73 us); for few long ones four to six passes over the row, of which a bare one takes 9 us for 64 rows of 235,000 in 16 bits
// and each of the others 20 to 35 more: it begins with what is known of the row, and ends with one workgroup's sums, some
// 15 us of barriers and trips to memory that nothing runs beside (in all 123 us, by top-p); 16 rows of 2.9 million in 32 bits, whose
// passes run at memory's speed, 225.
#include "sample.h"

#include "kernels.h"
#include "matrix_tile.h"
#include "wave_sums.h"

namespace surel {
namespace {

constexpr int kThreads = 512, kFewThreads = 256, kMostWaves = kThreads / 64;   // of a workgroup; of one for a short row
constexpr int kBins = 4096;        // the last takes what counts as zero
constexpr double kFar = 64.0;      // in x: e^-64 of 2^28 classes is 2^-64 of the largest weight
constexpr int kSub = 1024;         // bins of logits of a list
constexpr int kList = 4096;        // logits of a list, at most
constexpr int kMostChunks = 1024;  // of a row that one workgroup draws from alone
constexpr int kMostParted = 2048;  // and of one that several do

__device__ __forceinline__ int threads() { return (int)blockDim.x; }

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
    int skip, end, slots, chunk, chunks;   // chunk: slots whose weights are added up together
    __device__ __forceinline__ RowOf(const SampleArgs& a, int row, int of_chunk) : chunk(of_chunk) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(a.logits + row * a.row);
        base = reinterpret_cast<const char*>(at & ~(uintptr_t)15);
        skip = (int)(at & 15) / (16 / L::kPer);
        end = skip + a.n_classes;
        slots = (end + L::kPer - 1) / L::kPer;
        chunks = (slots + chunk - 1) / chunk;
    }
    __device__ __forceinline__ u32x4 load(int slot) const {
        const char* const at = base + (int64_t)slot * 16;
        const int first = slot * L::kPer;
        if (first >= skip && first + L::kPer <= end) return *reinterpret_cast<const u32x4*>(at);
        // (a loop, as this is in many places: one workgroup's first pass over code that nobody has read yet is what a small
        // row waits for)
        u32x4 x = {L::kNone, L::kNone, L::kNone, L::kNone};
#pragma unroll 1
        for (int e = max(skip - first, 0); e < min(end - first, L::kPer); ++e) {
            constexpr int kBits = 128 / L::kPer, kOfWord = 32 / kBits;
            const uint32_t z = kBits == 32 ? reinterpret_cast<const uint32_t*>(at)[e] : reinterpret_cast<const uint16_t*>(at)[e];
            const int shift = e % kOfWord * kBits, word = e / kOfWord;
            const uint32_t mask = (kBits == 32 ? ~0u : 0xFFFFu) << shift;
#pragma unroll
            for (int w = 0; w < 4; ++w) x[w] = w == word ? (x[w] & ~mask) | z << shift : x[w];
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
    float bins;              // bins of a unit of half a logit
    float cut;               // logits below it have weights below min_p
    double inv_t, width;     // 1 / T; a bin's, in x
    uint32_t k;              // 0: all
    double p, min_p, u;      // p of 1: all
    bool first;              // the first of the largest logits, nothing else
};

// What a row is given beside its logits.
struct Given {
    float u, t, p, floor;
    int k;
};
__device__ __forceinline__ Given given_for(const SampleArgs& a, int row) {
    return Given{a.u[row], a.temperature == nullptr ? 1.f : a.temperature[row], a.top_p == nullptr ? 1.f : a.top_p[row],
                 a.min_p == nullptr ? 0.f : a.min_p[row], a.top_k == nullptr ? 0 : a.top_k[row]};
}
__device__ __forceinline__ How how_of(const SampleArgs& a, const Given& given, const Ends& e) {
    How h;
    const float u = given.u, t = given.t, p = given.p, floor = given.floor;
    const int k = given.k;
    const bool fine = u >= 0.f && u < 1.f && t >= 0.f && t < INFINITY && p >= 0.f && floor >= 0.f && floor <= 1.f;
    h.wrong = !fine || e.bad;
    h.draws = !h.wrong && e.most > -INFINITY;
    h.first = t == 0.f || k == 1;
    h.most = e.most;
    const double temperature = h.first ? 1.0 : (double)t;
    h.inv_t = 1.0 / temperature;
    // a range of logits, not of x: a division less, and T may be any
    const double range = fmin((double)e.most - (double)e.least, kFar * temperature);
    const double bins = range > 0.0 ? 2.0 * (kBins - 2) / range : 0.0;
    h.bins = bins < 0x1p126 ? (float)bins : 0.f;   // 0: one bin of all
    h.width = range * h.inv_t / (kBins - 2);
    h.k = k < 1 || k >= a.n_classes ? 0 : (uint32_t)k;
    h.p = h.first || p >= 1.f ? 1.0 : (double)p;
    h.min_p = h.first ? 0.0 : (double)floor;
    h.cut = -INFINITY;
    if (h.min_p > 0.0) {     // a little below, for what is rounded here; the weights themselves decide
        const double down = log(h.min_p) * temperature;
        h.cut = (float)((double)e.most + down * (1.0 + 0x1p-20) - fabs((double)e.most) * 0x1p-20);
    }
    h.u = (double)u;
    return h;
}

// What a workgroup keeps of its row in LDS.
struct Bench {
    How how;
    double roots[16];
    Ends ends[kMostWaves];
    double of_wave[16];
    uint32_t counts_of_wave[16];
    int hit, last;                  // what a search found, or the last that is not empty
    uint32_t before;                // counts and weights before it
    double mass_before;
    uint32_t lo, hi;
    int n_list, is_last;
};
struct SubBins {
    uint64_t mass[kSub];
    uint32_t count[kSub];
    uint32_t list[kList];
};

// What is known of a row's border.
struct Border {
    int open;                // 0: found (or there is none), 1: of the first k, 2: of p
    int alone;               // its bins have too many logits: one workgroup looks for it
    int from, to;            // it lies in these bins
    uint32_t before;         // classes before them
    double whole;            // what p is of, or -1: the sum of all weights
    uint32_t key, ties;      // kept: logits above, and the first `ties` of this one
    uint32_t k_key, k_ties;  // the same of the first k alone
};

// 2^(j / 16).
__constant__ const double kRoots[16] = {0x1.0000000000000p+0, 0x1.0b5586cf9890fp+0, 0x1.172b83c7d517bp+0, 0x1.2387a6e756238p+0, 0x1.306fe0a31b715p+0, 0x1.3dea64c123422p+0, 0x1.4bfdad5362a27p+0, 0x1.5ab07dd485429p+0, 0x1.6a09e667f3bcdp+0, 0x1.7a11473eb0187p+0, 0x1.8ace5422aa0dbp+0, 0x1.9c49182a3f090p+0, 0x1.ae89f995ad3adp+0, 0x1.c199bdd85529cp+0, 0x1.d5818dcfba487p+0, 0x1.ea4afa2a490dap+0};

// exp(y), -64 <= y <= 0, in 64 bits; 0 below.  2^(n / 16) exp(r) with |r| <= ln(2) / 32, whose next term is 2^-59.  roots: kRoots in
// LDS (16 addresses meet no bank twice; without them 13 terms are needed, twice the instructions).
__device__ __forceinline__ double exp64(const double* roots, double y) {
    const double n = rint(y * 0x1.71547652b82fep+4);
    double r = __builtin_fma(n, -0x1.62e42fefa39efp-5, y);
    r = __builtin_fma(n, -0x1.abc9e3b39803fp-60, r);   // (what ln(2) / 16 in 64 bits leaves out)
    double e = __builtin_fma(r, 1.0 / 5040.0, 1.0 / 720.0);
    e = __builtin_fma(e, r, 1.0 / 120.0);
    e = __builtin_fma(e, r, 1.0 / 24.0);
    e = __builtin_fma(e, r, 1.0 / 6.0);
    e = __builtin_fma(e, r, 0.5);
    e = __builtin_fma(e, r, 1.0);
    e = __builtin_fma(e, r, 1.0);
    const int i = (int)n;
    return y >= -kFar ? ldexp(e * roots[i & 15], i >> 4) : 0.0;
}
__device__ __forceinline__ double weight_of(const Bench& l, const How& h, float z) {
    return exp64(l.roots, fmax(((double)z - (double)h.most) * h.inv_t, -2.0 * kFar));
}
// Where a logit lies, in bins: never before a larger one.  (Halves: their difference has the range of 32-bit floats.)
__device__ __forceinline__ float place_of(const How& h, float z) {
    return fminf((0.5f * h.most - 0.5f * z) * h.bins, (float)(kBins - 1));
}
__device__ __forceinline__ int bin_of(const How& h, float z) { return (int)place_of(h, z); }
// A bin's number of classes, 30 bits, and the sum of how far they lie in it, 34, in parts of 2^-inside_bits of its width
// (31 bits at most: a class's is a 32-bit word).
constexpr int kInside = 34;
__device__ __forceinline__ int inside_bits(int n_classes) { return min(kInside - (32 - __clz(n_classes)), 31); }
__device__ __forceinline__ uint32_t count_in(uint64_t bin) { return (uint32_t)(bin >> kInside); }

// Weights relative to a list's largest as whole numbers of two words: `one` = 2^unit of the first are one, and as many of the
// second, which is signed, one of the first.  Their sums stay below 2^63, and what is left out of a weight is at most
// 2^-(2 unit + 1): of all of a row's 2^-39 in the longest rows, 2^-60 in those of 2.9 million.  (One word left out up to 2^-41 of each
// there: of a tail of classes of 2^-33 of the largest some thousands too many were kept, of 20 million of 2^-38 a quarter too few.)
__device__ __forceinline__ int unit_of(int n_classes) { return min(62 - (32 - __clz(n_classes)), 50); }

__device__ __forceinline__ void add_count(uint32_t* at, uint32_t n) {
    (void)__hip_atomic_fetch_add(at, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
__device__ __forceinline__ void add_mass(uint64_t* at, uint64_t x) {
    (void)__hip_atomic_fetch_add(at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// Sums over the workgroup of what its threads before this one have; *all: of all threads.
__device__ __forceinline__ uint32_t counts_before(Bench& l, uint32_t mine, uint32_t* all) {
    return before_in_group(mine, l.counts_of_wave, all);
}
__device__ __forceinline__ double masses_before(Bench& l, double mine, double* all) { return before_in_group(mine, l.of_wave, all); }

__device__ __forceinline__ void add_weight(uint64_t* first, uint64_t* second, double w, double one) {
    const double near = __builtin_fma(w, one, 0x1p52);   // rounded, by a sum whose last place is 1
    add_mass(first, (uint64_t)__double_as_longlong(near) - 0x4330000000000000ull);
    const double rest = __builtin_fma(w, one, -(near - 0x1p52));
    add_mass(second, (uint64_t)__double_as_longlong(__builtin_fma(rest, one, 0x1.8p52)) - 0x4338000000000000ull);
}

// The workgroup's bench for a row whose ends every thread has a part of.
__device__ __forceinline__ Ends over_lanes(Ends e) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        Ends o;
        o.most = __shfl_xor(e.most, m), o.least = __shfl_xor(e.least, m), o.bad = __shfl_xor(e.bad, m);
        e.add(o);
    }
    return e;
}
__device__ __forceinline__ void set_up(Bench& l, const SampleArgs& a, const Given& given, Ends e) {
    e = over_lanes(e);
    if (threadIdx.x < 16) l.roots[threadIdx.x] = kRoots[threadIdx.x];
    if ((threadIdx.x & 63) == 0) l.ends[threadIdx.x >> 6] = e;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < threads() / 64; ++w) e.add(l.ends[w]);
        l.how = how_of(a, given, e);
    }
    __syncthreads();
}

// The first of n bins that is not empty and up to which counts reach k, or (by_mass) weights reach the target; count and mass
// of a bin by its number, at most n / threads of them a thread.  Leaves in l.hit which, or where none is the last that is not
// empty (by_mass: sums in another order may differ in their last places), or -1, and in l.before and l.mass_before what
// comes before it, on top of what is given.  masses: weights are asked for.
template <class Count, class Mass>
__device__ __forceinline__ void search(Bench& l, int bins, bool by_mass, bool masses, uint32_t k, double target, uint32_t before, double mass_before,
                                       Count count, Mass mass) {
    const int each = (bins + threads() - 1) / threads(), first = threadIdx.x * each, end = min(first + each, bins);
    uint32_t n = 0, all;
    double w = 0.0, all_w;
    for (int i = first; i < end; ++i) n += count(i), w += mass(i);
    if (threadIdx.x == 0) l.hit = 0x7FFFFFFF, l.last = -1;
    uint32_t till = before + counts_before(l, n, &all);
    double till_w = masses ? mass_before + masses_before(l, w, &all_w) : 0.0;
    uint32_t my_till = 0, full_till = 0;
    double my_till_w = 0.0, full_till_w = 0.0;
    int mine = -1, full = -1;
    for (int i = first; i < end; ++i) {
        const uint32_t c = count(i);
        const double m = mass(i);
        if (c != 0) {
            full = i, full_till = till, full_till_w = till_w;
            if (mine < 0 && (by_mass ? till_w + m >= target : till + c >= k)) mine = i, my_till = till, my_till_w = till_w;
        }
        till += c, till_w += m;
    }
    if (mine >= 0) atomicMin(&l.hit, mine);
    if (by_mass && full >= 0) atomicMax(&l.last, full);
    __syncthreads();
    const int hit = l.hit != 0x7FFFFFFF ? l.hit : l.last;
    __syncthreads();
    if (hit >= 0 && mine == hit) l.before = my_till, l.mass_before = my_till_w;
    else if (hit >= 0 && full == hit) l.before = full_till, l.mass_before = full_till_w;
    if (threadIdx.x == 0) l.hit = hit;
    __syncthreads();
}

// Between which bins the border lies: of the first k, then of p.
__device__ __forceinline__ void start_border(Border* b) {
    b->open = 0, b->alone = 0, b->from = b->to = -1, b->before = 0, b->whole = -1.0;
    b->key = b->k_key = 0, b->ties = b->k_ties = 0xFFFFFFFFu;
}
// `whole`: what p is of, if that is known.  A bin's c classes, places f_j of its width h behind its beginning i h, weigh
// exp(-i h) (c - h sum f) and up to exp(-i h) c h^2 / 2 more; what is rounded is less than 2^-16 of it.
__device__ __forceinline__ void open_p(Bench& l, const uint64_t* bins, Border* b, int n_classes, double whole) {
    const double h = l.how.width, p = l.how.p, step = exp64(l.roots, -h), part = ldexp(h, -inside_bits(n_classes));
    const double off = 1.0 + h * h + part + 0x1p-16;
    const int each = kBins / threads(), first = threadIdx.x * each;   // (the last bin does not count)
    auto mass = [&](uint64_t x, double at) { return at * ((double)count_in(x) - part * (double)(x & ((1ull << kInside) - 1))); };
    uint32_t n = 0, unused;
    double w = 0.0, all, at = exp64(l.roots, fmax(-h * first, -kFar));
    for (int i = first; i < min(first + each, kBins - 1); ++i, at *= step) n += count_in(bins[i]), w += mass(bins[i], at);
    if (threadIdx.x == 0) l.hit = l.hi = 0x7FFFFFFF, l.last = -1;
    uint32_t till = counts_before(l, n, &unused);
    double till_w = masses_before(l, w, &all);
    const double low = p * (whole >= 0.0 ? whole / off : all / (off * off)), high = p * (whole >= 0.0 ? whole * off : all * off * off);
    int from = -1, to = -1, full = -1;
    uint32_t from_till = 0, full_till = 0;
    at = exp64(l.roots, fmax(-h * first, -kFar));
    for (int i = first; i < min(first + each, kBins - 1); ++i, at *= step) {
        const uint32_t c = count_in(bins[i]);
        if (c != 0) {
            till_w += mass(bins[i], at);
            full = i, full_till = till;
            if (from < 0 && till_w >= low) from = i, from_till = till;
            if (to < 0 && till_w >= high) to = i;
        }
        till += c;
    }
    if (from >= 0) atomicMin(&l.hit, from);
    if (to >= 0) atomicMin(&l.hi, (uint32_t)to);
    if (full >= 0) atomicMax(&l.last, full);
    __syncthreads();
    const int begin = l.hit != 0x7FFFFFFF ? l.hit : l.last, end = l.hi != 0x7FFFFFFFu ? (int)l.hi : l.last;
    if (from == begin || full == begin) b->before = from == begin ? from_till : full_till;
    if (threadIdx.x == 0) b->open = 2, b->from = begin, b->to = end, b->whole = whole;
    __syncthreads();
}
__device__ __forceinline__ void open_border(Bench& l, const uint64_t* bins, Border* b, int n_classes) {
    if (threadIdx.x == 0) start_border(b);
    __syncthreads();
    int hit = -1;
    if (l.how.k != 0) {
        search(l, kBins, false, false, l.how.k, 0.0, 0, 0.0, [&](int i) { return i < kBins - 1 ? count_in(bins[i]) : 0u; }, [](int) { return 0.0; });
        hit = l.hit;
        if (hit >= 0 && threadIdx.x == 0) b->open = 1, b->from = b->to = hit, b->before = l.before;
        __syncthreads();
    }
    if (hit < 0 && l.how.p < 1.0) open_p(l, bins, b, n_classes, -1.0);   // (no k, or fewer classes of any weight)
}

// The border among the logits of its bins, which each() goes through; every thread takes some.  mass_before: the weights
// before them, total: all there are.  rest: kSub words of LDS, weights' second ones.
template <class L, class Each>
__device__ __forceinline__ void find_border(Bench& l, SubBins& sub, uint64_t* rest, Border* b, int n_classes, double mass_before, double total, Each each) {
    const How how = l.how;
    const int unit = unit_of(n_classes);
    const double one = ldexp(1.0, unit), back = ldexp(1.0, -unit);
    const bool by_p = b->open == 2, masses = how.p < 1.0;
    const double target = how.p * (b->whole >= 0.0 ? b->whole : total);
    uint32_t lo = 0xFFFFFFFFu, hi = 0, before = b->before;
    each([&](uint32_t key) { lo = min(lo, key), hi = max(hi, key); });
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) lo = min(lo, (uint32_t)__shfl_xor((int)lo, m)), hi = max(hi, (uint32_t)__shfl_xor((int)hi, m));
    if (threadIdx.x == 0) l.lo = 0xFFFFFFFFu, l.hi = 0;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) atomicMin(&l.lo, lo), atomicMax(&l.hi, hi);
    __syncthreads();
    lo = l.lo, hi = l.hi;
    const float top = logit_of<L>(hi);
    const double of_top = weight_of(l, how, top) * back;
    for (;;) {
        const int shift = max(32 - (int)__clz(hi - lo) - 10, 0);   // (hi - lo) >> shift is below kSub
        const bool add = masses && shift > 0;   // (bins of one logit: their counts say what they weigh)
        for (int i = threadIdx.x; i < kSub; i += threads()) sub.count[i] = 0, sub.mass[i] = rest[i] = 0;
        __syncthreads();
        each([&](uint32_t key) {
            if (key < lo || key > hi) return;
            const uint32_t i = (hi - key) >> shift;
            add_count(&sub.count[i], 1);
            if (add) add_weight(&sub.mass[i], &rest[i], exp64(l.roots, fmax(((double)logit_of<L>(key) - (double)top) * how.inv_t, -2.0 * kFar)), one);
        });
        __syncthreads();
        if (masses && shift == 0) {
            for (int i = threadIdx.x; i < kSub; i += threads())
                if (const uint32_t n = sub.count[i]; n != 0) sub.mass[i] = (uint64_t)__double_as_longlong((double)n * weight_of(l, how, logit_of<L>(hi - i)));
            __syncthreads();
        }
        search(l, kSub, by_p, masses, how.k, target, before, mass_before, [&](int i) { return sub.count[i]; },
               [&](int i) {
                   return !add ? __longlong_as_double((long long)sub.mass[i])
                               : __builtin_fma((double)(int64_t)rest[i], back, (double)sub.mass[i]) * of_top;
               });
        const int hit = l.hit;
        if (hit < 0) break;   // (of a list that is not empty one is found)
        before = l.before, mass_before = l.mass_before;
        const uint32_t upper = hi - ((uint32_t)hit << shift);
        if (shift == 0) {
            if (threadIdx.x == 0) {
                const uint32_t n = sub.count[hit];
                const double w = weight_of(l, how, logit_of<L>(upper));
                b->key = upper;
                if (by_p) {
                    const double need = w > 0.0 ? ceil((target - mass_before) / w) : (double)n;
                    b->ties = (uint32_t)fmin(fmax(need, 1.0), (double)n);
                    if (b->key == b->k_key) b->ties = min(b->ties, b->k_ties);
                } else {
                    b->ties = how.k - before;
                    b->k_key = b->key, b->k_ties = b->ties;
                    b->whole = mass_before + (double)b->ties * w;   // what the first k weigh
                }
            }
            break;
        }
        hi = upper;
        lo = max(lo, upper - ((1u << shift) - 1u));
        __syncthreads();
    }
    if (threadIdx.x == 0) b->open = 0;
    __syncthreads();
}

// What is kept of a row.
struct Drawn {
    float at;          // the border's logit
    float from;        // below it no logit counts
    double floor;      // least weight that is kept
};
__device__ __forceinline__ double kept_weight(const Bench& l, const How& h, const Drawn& d, float z) {
    const double w = weight_of(l, h, z);
    return z > d.at && w >= d.floor ? w : 0.0;
}
// Weights of a chunk above the border, and how many classes lie on it.  One wave.
template <class L>
__device__ __forceinline__ void chunk_sums(const Bench& l, const How& h, const RowOf<L>& r, const Drawn& d, int chunk, double* mass, uint32_t* ties) {
    const int lane = threadIdx.x & 63, end = min((chunk + 1) * r.chunk, r.slots);
    double w = 0.0;
    uint32_t n = 0;
    const u32x4 none = {L::kNone, L::kNone, L::kNone, L::kNone};
    int slot = chunk * r.chunk + lane;
    u32x4 next = slot < end ? r.load(slot) : none;
#pragma unroll 1
    for (; slot - lane < end; slot += 64) {
        const u32x4 x = next;
        next = slot + 64 < end ? r.load(slot + 64) : none;
        float most = L::at(x, 0);
#pragma unroll
        for (int e = 1; e < L::kPer; ++e) most = fmaxf(most, L::at(x, e));
        if (!__any(most >= d.from)) continue;
#pragma unroll
        for (int e = 0; e < L::kPer; ++e) {
            const float z = L::at(x, e);
            w += kept_weight(l, h, d, z);
            n += z == d.at;
        }
    }
    *mass = of_lane(sum_till(w), 63), *ties = wave_bcast_u32(wave_incl_sum(n), 63);
}

__device__ __forceinline__ void no_class(const Bench& l, const SampleArgs& a, int row) {
    if (threadIdx.x != 0) return;
    a.chosen[row] = -1;
    a.logp[row] = -INFINITY;
    if (l.how.wrong) atomicOr(a.err, kDevBadChoice);
}
// The class, from the chunks' sums.
template <class L, class Mass, class Ties>
__device__ __forceinline__ void choose(Bench& l, const SampleArgs& a, int row, const RowOf<L>& r, const Drawn& d, uint32_t most_ties,
                                       Mass mass_of, Ties ties_of) {
    const How h = l.how;
    const double on = weight_of(l, h, d.at);            // of a class on the border
    const uint32_t kept = on >= d.floor ? most_ties : 0;
    // chunks: how many of their classes on the border are kept, then their weights
    const int per = (r.chunks + threads() - 1) / threads(), first = threadIdx.x * per, end = min(first + per, r.chunks);
    uint32_t n = 0, unused;
    for (int c = first; c < end; ++c) n += ties_of(c);
    uint32_t ties = counts_before(l, n, &unused);
    double w = 0.0, total;
    uint32_t t = ties;
    auto of_chunk = [&](int c, uint32_t before) {
        const uint32_t n = min(before + ties_of(c), kept) - min(before, kept);
        return __builtin_fma((double)n, on, mass_of(c));
    };
    for (int c = first; c < end; ++c) w += of_chunk(c, t), t += ties_of(c);
    double till = masses_before(l, w, &total);
    const double target = h.u * total;
    // the first whose sum passes the target; where by the sums' last places none does, the last that weighs anything
    struct Found {
        int at;
        double till, w;
        uint32_t ties;
    };
    Found mine = {-1, 0.0, 0.0, 0}, full = {-1, 0.0, 0.0, 0};
    auto take = [&](int at, double m, uint32_t before) {
        if (m > 0.0) {
            full = Found{at, till, m, before};
            if (mine.at < 0 && till + m > target) mine = full;
        }
        till += m;
    };
    auto agree = [&] {   // returns whether it is this thread's, in `mine`
        if (threadIdx.x == 0) l.hit = 0x7FFFFFFF, l.last = -1;
        __syncthreads();
        if (mine.at >= 0) atomicMin(&l.hit, mine.at);
        if (full.at >= 0) atomicMax(&l.last, full.at);
        __syncthreads();
        const int at = l.hit != 0x7FFFFFFF ? l.hit : l.last;
        __syncthreads();
        if (mine.at != at) mine = full;
        return at >= 0 && mine.at == at;
    };
    for (int c = first; c < end; ++c) {
        take(c, of_chunk(c, ties), ties);
        ties += ties_of(c);
    }
    if (agree()) l.mass_before = mine.till, l.before = mine.ties;
    __syncthreads();
    const int chunk = l.hit != 0x7FFFFFFF ? l.hit : l.last;
    if (chunk < 0) {   // (the largest logit is always kept; but a row that changes under the call is not to lead anywhere)
        no_class(l, a, row);
        return;
    }
    till = l.mass_before;
    ties = l.before;

    // inside the chunk, some slots a thread.  (Loops that are not unrolled: one workgroup a row comes here, and reads this code
    // for the first time.  With three loops of eight elements it took 17 us, of 43 for 64 rows of 235,000.)
    const int each = (r.chunk + threads() - 1) / threads(), begin = chunk * r.chunk + (int)threadIdx.x * each;
    const int stop = min(min(begin + each, (chunk + 1) * r.chunk), r.slots);
    n = 0;
#pragma unroll 1
    for (int s = begin; s < stop; ++s) {
        const u32x4 x = r.load(s);
#pragma unroll
        for (int e = 0; e < L::kPer; ++e) n += L::at(x, e) == d.at;
    }
    ties += counts_before(l, n, &unused);
    auto weight_in = [&](float z, uint32_t& t) { return z == d.at ? (t++ < kept ? on : 0.0) : kept_weight(l, h, d, z); };
    auto each_weight = [&](auto act) {
        uint32_t t = ties;
#pragma unroll 1
        for (int s = begin; s < stop; ++s) {
            const u32x4 x = r.load(s);
#pragma unroll 1
            for (int e = 0; e < L::kPer; ++e) act(s * L::kPer + e, weight_in(L::at(x, e), t));
        }
    };
    w = 0.0;
    each_weight([&](int, double m) { w += m; });
    double unused_mass;
    till += masses_before(l, w, &unused_mass);
    mine.at = full.at = -1;
    each_weight([&](int at, double m) { take(at, m, 0); });
    if (agree()) {
        a.chosen[row] = mine.at - r.skip;
        a.logp[row] = (float)log(mine.w / total);
    }
}

__device__ __forceinline__ bool has_border(const How& h) { return !h.first && (h.k != 0 || h.p < 1.0); }

// Goes through the slots begin .. end - 1 of a row.
template <class L, class Do>
__device__ __forceinline__ void each_logit(const RowOf<L>& r, int begin, int end, Do act) {
#pragma unroll 2
    for (int s = begin + (int)threadIdx.x; s < end; s += threads()) {
        const u32x4 x = r.load(s);
#pragma unroll
        for (int e = 0; e < L::kPer; ++e) act(L::at(x, e));
    }
}
template <class L>
__device__ __forceinline__ void count_bins(const Bench& l, uint64_t* bins, const RowOf<L>& r, int begin, int end, int n_classes) {
    const How how = l.how;
    const float parts = (float)(1u << inside_bits(n_classes));
    each_logit<L>(r, begin, end, [&](float z) {
        const float at = place_of(how, z), b = floorf(at);
        if (b < (float)(kBins - 1)) add_mass(&bins[(int)b], (1ull << kInside) + (uint32_t)((at - b) * parts));
    });
}
// Goes through a border's logits, put(key); returns the thread's share of the weights before them (if these are asked for) and
// of all weights (if p is of them).
struct Masses {
    double before, all;
};
template <class L, class Put>
__device__ __forceinline__ Masses border_logits(const Bench& l, const How& how, const Border& b, const RowOf<L>& r, int begin, int end, Put put) {
    const int from = b.from, to = b.to;
    const bool masses = how.p < 1.0, all = masses && b.open == 2 && b.whole < 0.0;
    Masses m = {0.0, 0.0};
    const u32x4 none = {L::kNone, L::kNone, L::kNone, L::kNone};
    int s = begin + (int)threadIdx.x;
    u32x4 next = s < end ? r.load(s) : none;
#pragma unroll 1
    for (; s < end; s += threads()) {
        const u32x4 x = next;
        next = s + threads() < end ? r.load(s + threads()) : none;
        int bin[L::kPer], first = kBins;
#pragma unroll
        for (int e = 0; e < L::kPer; ++e) {
            bin[e] = bin_of(how, L::at(x, e));
            first = min(first, bin[e]);
        }
        if (all || __any(first <= to)) {
#pragma unroll
            for (int e = 0; e < L::kPer; ++e) {
                const float z = L::at(x, e);
                if (bin[e] >= from && bin[e] <= to) put(key_of<L>(z));
                if (masses) {
                    const double w = weight_of(l, how, z);
                    m.before += bin[e] < from ? w : 0.0;
                    m.all += w;
                }
            }
        }
    }
    return m;
}

// A row's border once its bins are known, by one workgroup: from a list of their logits if that holds them, or by the row.
template <class L>
__device__ __forceinline__ void find_in_row(Bench& l, SubBins& sub, uint64_t* rest, Border* b, const RowOf<L>& r, int n_classes) {
    if (threadIdx.x == 0) l.n_list = 0;
    __syncthreads();
    const How how = l.how;
    const Border now = *b;
    const Masses m = border_logits<L>(l, how, now, r, 0, r.slots, [&](uint32_t key) {
        const int at = atomicAdd(&l.n_list, 1);
        if (at < kList) sub.list[at] = key;
    });
    double before = 0.0, all = 0.0;
    if (how.p < 1.0) {
        (void)masses_before(l, m.before, &before);
        (void)masses_before(l, m.all, &all);
    }
    __syncthreads();
    const int n = l.n_list;
    find_border<L>(l, sub, rest, b, n_classes, before, all, [&](auto act) {
        if (n <= kList) {
            for (int i = threadIdx.x; i < n; i += threads()) act(sub.list[i]);
        } else {
            // (equal logits on the border, or rows of so many classes that bins beside it hold more than the list: 2.9 million by
            // top_p alone.  Loops that keep the code short)
#pragma unroll 1
            for (int s = threadIdx.x; s < r.slots; s += threads()) {
                const u32x4 x = r.load(s);
#pragma unroll 1
                for (int e = 0; e < L::kPer; ++e) {
                    const float z = L::at(x, e);
                    const int bin = bin_of(how, z);
                    if (bin >= now.from && bin <= now.to) act(key_of<L>(z));
                }
            }
        }
    });
}
template <class L>
__device__ __forceinline__ void find_all_in_row(Bench& l, const uint64_t* bins, SubBins& sub, uint64_t* rest, Border* b, const RowOf<L>& r, int n_classes) {
#pragma unroll 1
    for (int open = b->open; open != 0; open = b->open) {
        find_in_row<L>(l, sub, rest, b, r, n_classes);
        if (open == 1 && l.how.p < 1.0) open_p(l, bins, b, n_classes, b->whole);
    }
}

template <class L>
__device__ __forceinline__ Drawn drawn_by(const How& h, const Border& b) {
    Drawn d;
    d.at = h.first ? h.most : b.key == 0 ? -INFINITY : logit_of<L>(b.key);
    d.from = fmaxf(d.at, h.cut);
    d.floor = h.min_p;
    return d;
}

// One workgroup a row, all of it.
struct RowLds {
    Bench bench;
    Border border;
    union {
        double mass[kMostChunks];
        uint64_t rest[kSub];        // (while the border is looked for.  With 8 KB more one row fits a compute unit, not two)
    };
    uint32_t ties[kMostChunks];
};
struct BorderLds {
    SubBins sub;
    uint64_t bins[kBins];
};
// Rows without a border need half the registers, and twice as many of them are on their way.
template <class L, bool BORDERS>
__global__ __launch_bounds__(kThreads, BORDERS ? 4 : 6) void sample_row_kernel(SampleArgs a, int chunk) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ RowLds l;
    const int64_t place = block_number();
    if (place >= a.n_rows) return;
    const int row = (int)place;
    const RowOf<L> r(a, row, chunk);
    const Given given = given_for(a, row);
    Ends ends = Ends::none();
    each_logit<L>(r, 0, r.slots, [&](float z) { ends.add(z); });
    set_up(l.bench, a, given, ends);
    const How how = l.bench.how;
    if (!how.draws) {
        no_class(l.bench, a, row);
        return;
    }
    if (threadIdx.x == 0) start_border(&l.border);
    if (BORDERS && has_border(how)) {
        BorderLds& w = *reinterpret_cast<BorderLds*>(dynamic);
        for (int i = threadIdx.x; i < kBins; i += threads()) w.bins[i] = 0;
        __syncthreads();
        count_bins<L>(l.bench, w.bins, r, 0, r.slots, a.n_classes);
        __syncthreads();
        open_border(l.bench, w.bins, &l.border, a.n_classes);
        find_all_in_row<L>(l.bench, w.bins, w.sub, l.rest, &l.border, r, a.n_classes);
    }
    __syncthreads();
    const Drawn d = drawn_by<L>(how, l.border);
    for (int c = threadIdx.x >> 6; c < r.chunks; c += threads() / 64) {
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
    int parts = 1, chunk = 0, chunks = 0, each = 0;   // of a row: workgroups, slots of a chunk, chunks at most, chunks of a part
    Ends* ends = nullptr;                  // [rows][parts]
    uint32_t* turns = nullptr;             // [rows][4]: workgroups of a step that are done, and how long the list is
    Border* border = nullptr;              // [rows]
    uint64_t* bins = nullptr;              // [rows][kBins]
    uint32_t* list = nullptr;              // [rows][kList]
    uint64_t* masses = nullptr;            // [rows][parts][2]
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
__device__ __forceinline__ void put(uint64_t* at, double x) { put(at, (uint64_t)__double_as_longlong(x)); }
__device__ __forceinline__ double get_mass(const uint64_t* at) { return __longlong_as_double((long long)get(at)); }

// Whether this workgroup is the last of its row's to come here.
__device__ __forceinline__ bool last_of(Bench& l, uint32_t* turn, int parts) {
    wait_memory();
    __syncthreads();
    if (threadIdx.x == 0) l.is_last = add_far(turn, 1u) == (uint32_t)parts - 1;
    __syncthreads();
    return l.is_last != 0;
}

struct Part {
    int begin, end, chunk_begin, chunk_end;   // slots; chunks
};
template <class L>
__device__ __forceinline__ Part part_of(const Parts& p, const RowOf<L>& r, int part) {
    Part x;
    x.chunk_begin = min(part * p.each, r.chunks), x.chunk_end = min(x.chunk_begin + p.each, r.chunks);
    x.begin = min(x.chunk_begin * r.chunk, r.slots), x.end = min(x.chunk_end * r.chunk, r.slots);
    return x;
}
__device__ __forceinline__ void set_up_from_parts(Bench& l, const SampleArgs& a, const Parts& p, int row) {
    const Given given = given_for(a, row);
    Ends e = Ends::none();
    for (int i = threadIdx.x; i < p.parts; i += threads()) e.add(p.ends[(int64_t)row * p.parts + i]);
    set_up(l, a, given, e);
}

template <class L>
__global__ __launch_bounds__(kThreads) void sample_ends_kernel(SampleArgs a, Parts p) {
    __shared__ Ends ends[kMostWaves];
    const int64_t block = block_number();
    const int row = (int)(block / p.parts), part = (int)(block % p.parts);
    if (row >= a.n_rows) return;
    const RowOf<L> r(a, row, p.chunk);
    const Part x = part_of(p, r, part);
    if (part == 0 && threadIdx.x < 4) p.turns[4 * row + threadIdx.x] = 0;
    if (p.bins != nullptr)
        for (int i = part * kThreads + threadIdx.x; i < kBins; i += p.parts * kThreads) p.bins[(int64_t)row * kBins + i] = 0;
    Ends e = Ends::none();
    each_logit<L>(r, x.begin, x.end, [&](float z) { e.add(z); });
    e = over_lanes(e);
    if ((threadIdx.x & 63) == 0) ends[threadIdx.x >> 6] = e;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kMostWaves; ++w) e.add(ends[w]);
    p.ends[(int64_t)row * p.parts + part] = e;
}

template <class L>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a, Parts p) {
    __shared__ uint64_t bins[kBins];
    __shared__ Bench l;
    const int64_t block = block_number();
    const int row = (int)(block / p.parts), part = (int)(block % p.parts);
    if (row >= a.n_rows) return;
    set_up_from_parts(l, a, p, row);
    if (!l.how.draws || !has_border(l.how)) {
        if (part == 0 && threadIdx.x == 0) start_border(&p.border[row]);
        return;
    }
    const RowOf<L> r(a, row, p.chunk);
    const Part x = part_of(p, r, part);
    for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
    __syncthreads();
    count_bins<L>(l, bins, r, x.begin, x.end, a.n_classes);
    __syncthreads();
    uint64_t* const all = p.bins + (int64_t)row * kBins;
    for (int i = threadIdx.x; i < kBins; i += kThreads)
        if (bins[i] != 0) (void)add_far(&all[i], bins[i]);
    if (!last_of(l, &p.turns[4 * row + kBinTurn], p.parts)) return;
    for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = get(&all[i]);
    __syncthreads();
    open_border(l, bins, &p.border[row], a.n_classes);
}

// The border among its bins' logits, which all parts put into a list; the last part looks through it.
template <class L>
__global__ __launch_bounds__(kThreads) void sample_list_kernel(SampleArgs a, Parts p) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ Bench l;
    __shared__ Border b;
    __shared__ uint64_t rest[kSub];
    const int64_t block = block_number();
    const int row = (int)(block / p.parts), part = (int)(block % p.parts);
    if (row >= a.n_rows) return;
    const Border now = p.border[row];
    if (now.open == 0 || now.alone != 0) return;   // (no part of the row has changed that yet)
    set_up_from_parts(l, a, p, row);
    const RowOf<L> r(a, row, p.chunk);
    const Part x = part_of(p, r, part);
    uint32_t* const list = p.list + (int64_t)row * kList;
    const Masses m = border_logits<L>(l, l.how, now, r, x.begin, x.end, [&](uint32_t key) {
        const uint32_t at = add_far(&p.turns[4 * row + kListed], 1u);
        if (at < kList) put(&list[at], key);
    });
    double before, all;
    (void)masses_before(l, m.before, &before);
    (void)masses_before(l, m.all, &all);
    uint64_t* const masses = p.masses + 2 * (int64_t)row * p.parts;
    if (threadIdx.x == 0) put(&masses[2 * part], before), put(&masses[2 * part + 1], all);
    if (!last_of(l, &p.turns[4 * row + kListTurn], p.parts)) return;
    const uint32_t n = get(&p.turns[4 * row + kListed]);
    if (threadIdx.x == 0) b = now;
    __syncthreads();
    if (n > (uint32_t)kList) {
        if (threadIdx.x == 0) p.border[row].alone = 1;
        return;
    }
    BorderLds& w = *reinterpret_cast<BorderLds*>(dynamic);
    for (int i = threadIdx.x; i < (int)n; i += kThreads) w.sub.list[i] = get(&list[i]);
    double my_before = 0.0, my_all = 0.0;
    for (int i = threadIdx.x; i < p.parts; i += kThreads) my_before += get_mass(&masses[2 * i]), my_all += get_mass(&masses[2 * i + 1]);
    (void)masses_before(l, my_before, &before);
    (void)masses_before(l, my_all, &all);
    __syncthreads();
    find_border<L>(l, w.sub, rest, &b, a.n_classes, before, all, [&](auto act) {
        for (int i = threadIdx.x; i < (int)n; i += kThreads) act(w.sub.list[i]);
    });
    if (now.open == 1 && l.how.p < 1.0) {
        for (int i = threadIdx.x; i < kBins; i += kThreads) w.bins[i] = p.bins[(int64_t)row * kBins + i];
        __syncthreads();
        open_p(l, w.bins, &b, a.n_classes, b.whole);
    }
    if (threadIdx.x == 0) {
        p.border[row] = b;
        p.turns[4 * row + kListTurn] = 0, p.turns[4 * row + kListed] = 0;
    }
}

// Rows whose bins hold more logits than the list: a workgroup each, whatever their length.  16 rows of 2.9 million by a top_p of
// 0.95 alone take 3 to 6 ms so, where a list that holds them takes 0.2.
template <class L>
__global__ __launch_bounds__(kThreads) void sample_alone_kernel(SampleArgs a, Parts p) {
    extern __shared__ __align__(16) char dynamic[];
    __shared__ Bench l;
    __shared__ Border b;
    __shared__ uint64_t rest[kSub];
    const int64_t place = block_number();
    if (place >= a.n_rows || p.border[place].alone == 0) return;
    const int row = (int)place;
    set_up_from_parts(l, a, p, row);
    const RowOf<L> r(a, row, p.chunk);
    BorderLds& w = *reinterpret_cast<BorderLds*>(dynamic);
    for (int i = threadIdx.x; i < kBins; i += kThreads) w.bins[i] = p.bins[(int64_t)row * kBins + i];
    if (threadIdx.x == 0) b = p.border[row];
    __syncthreads();
    find_all_in_row<L>(l, w.bins, w.sub, rest, &b, r, a.n_classes);
    if (threadIdx.x == 0) p.border[row] = b;
}

template <class L>
__global__ __launch_bounds__(kThreads) void sample_draw_kernel(SampleArgs a, Parts p) {
    __shared__ Bench l;
    __shared__ double chunk_mass[kMostParted];
    __shared__ uint32_t chunk_ties[kMostParted];
    const int64_t block = block_number();
    const int row = (int)(block / p.parts), part = (int)(block % p.parts);
    if (row >= a.n_rows) return;
    set_up_from_parts(l, a, p, row);
    const How how = l.how;
    if (!how.draws) {
        if (part == 0) no_class(l, a, row);
        return;
    }
    const RowOf<L> r(a, row, p.chunk);
    const Part x = part_of(p, r, part);
    Border b;
    if (has_border(how)) b = p.border[row];
    else start_border(&b);
    const Drawn d = drawn_by<L>(how, b);
    uint64_t* const masses = p.mass + (int64_t)row * p.chunks;
    uint32_t* const ties = p.ties + (int64_t)row * p.chunks;
    for (int c = x.chunk_begin + (threadIdx.x >> 6); c < x.chunk_end; c += kThreads / 64) {
        double mass;
        uint32_t n;
        chunk_sums<L>(l, how, r, d, c, &mass, &n);
        if ((threadIdx.x & 63) == 0) put(&masses[c], mass), put(&ties[c], n);
    }
    if (!last_of(l, &p.turns[4 * row + kDrawTurn], p.parts)) return;
    for (int c = threadIdx.x; c < r.chunks; c += kThreads) chunk_mass[c] = get_mass(&masses[c]), chunk_ties[c] = get(&ties[c]);
    __syncthreads();
    choose<L>(l, a, row, r, d, how.first ? 1u : b.ties, [&](int c) { return chunk_mass[c]; }, [&](int c) { return chunk_ties[c]; });
}

struct Plan {
    Parts p;
    bool in_rows = false, borders = false;
    int lists = 0, row_threads = kThreads;
    size_t at[9] = {}, bytes = 0;
};
Plan plan_of(int n_cu, const SampleArgs& a, int type) {
    Plan x;
    const int per = type == 2 ? 4 : 8, slots = (a.n_classes + per - 1) / per + 1;   // (one more where a row starts inside one)
    x.borders = a.top_k != nullptr || a.top_p != nullptr;
    x.lists = (a.top_k != nullptr ? 1 : 0) + (a.top_p != nullptr ? 1 : 0);
    // A workgroup a row where rows fill the device, or are so short that one goes over them as soon as several would.
    x.p.chunk = slots <= 64 * kMostChunks ? 64 : 512;
    x.p.chunks = (slots + x.p.chunk - 1) / x.p.chunk;
    x.in_rows = x.p.chunks <= kMostChunks && (a.n_rows >= n_cu || slots <= 4096);
    if (x.in_rows) {
        x.row_threads = slots <= 2048 && a.n_rows >= n_cu ? kFewThreads : kThreads;
        return x;
    }
    x.p.chunk = 512;
    while ((slots + x.p.chunk - 1) / x.p.chunk > kMostParted) x.p.chunk *= 2;
    x.p.chunks = (slots + x.p.chunk - 1) / x.p.chunk;
    const int64_t wanted = (2 * (int64_t)n_cu + a.n_rows - 1) / a.n_rows;   // (two fit a compute unit)
    x.p.parts = (int)(wanted < x.p.chunks ? wanted : x.p.chunks);
    x.p.each = (x.p.chunks + x.p.parts - 1) / x.p.parts;
    x.p.parts = (x.p.chunks + x.p.each - 1) / x.p.each;
    const size_t rows = (size_t)a.n_rows;
    const size_t sizes[8] = {rows * x.p.parts * sizeof(Ends), rows * 16, x.borders ? rows * sizeof(Border) : 0,
                             x.borders ? rows * kBins * 8 : 0, x.borders ? rows * kList * 4 : 0, x.borders ? rows * x.p.parts * 16 : 0,
                             rows * x.p.chunks * 8, rows * x.p.chunks * 4};
    for (int i = 0; i < 8; ++i) x.at[i + 1] = x.at[i] + (sizes[i] + 255) / 256 * 256;
    x.bytes = x.at[8];
    return x;
}

template <class Kernel>
hipError_t allow(Kernel kernel) {   // (more LDS than a launch has without asking)
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(BorderLds));
}

template <class L>
hipError_t launch_type(hipStream_t stream, const SampleArgs& a, const Plan& x) {
    const size_t lds = sizeof(BorderLds);
    hipError_t rc = hipSuccess;
    if (x.in_rows) {
        if (x.borders) {
            if ((rc = allow(sample_row_kernel<L, true>)) != hipSuccess) return rc;
            hipLaunchKernelGGL((sample_row_kernel<L, true>), grid_of(a.n_rows), dim3(x.row_threads), lds, stream, a, x.p.chunk);
        } else {
            hipLaunchKernelGGL((sample_row_kernel<L, false>), grid_of(a.n_rows), dim3(x.row_threads), 0, stream, a, x.p.chunk);
        }
        return hipGetLastError();
    }
    const dim3 grid = grid_of((int64_t)a.n_rows * x.p.parts);
    hipLaunchKernelGGL(sample_ends_kernel<L>, grid, dim3(kThreads), 0, stream, a, x.p);
    if ((rc = hipGetLastError()) != hipSuccess) return rc;
    if (x.borders) {
        if ((rc = allow(sample_list_kernel<L>)) != hipSuccess || (rc = allow(sample_alone_kernel<L>)) != hipSuccess) return rc;
        hipLaunchKernelGGL(sample_bins_kernel<L>, grid, dim3(kThreads), 0, stream, a, x.p);
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
        x.p.bins = x.borders ? reinterpret_cast<uint64_t*>(s + x.at[3]) : nullptr;
        x.p.list = x.borders ? reinterpret_cast<uint32_t*>(s + x.at[4]) : nullptr;
        x.p.masses = x.borders ? reinterpret_cast<uint64_t*>(s + x.at[5]) : nullptr;
        x.p.mass = reinterpret_cast<uint64_t*>(s + x.at[6]);
        x.p.ties = reinterpret_cast<uint32_t*>(s + x.at[7]);
    }
    return type == 0 ? launch_type<Bf16Logit>(stream, a, x) : type == 1 ? launch_type<Fp16Logit>(stream, a, x)
                                                                        : launch_type<Fp32Logit>(stream, a, x);
}

}  // namespace surel
