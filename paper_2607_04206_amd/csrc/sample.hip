// A token and a confidence for every row of logits, for gfx950, with its C ABI
// entry point (include/sangam_sample.h).
//
// All filters and the draw are places on one axis, the ranks: a prefix of them
// is kept, and the draw falls at a share u of the prefix's weight. What is
// needed of a row is therefore how many tokens and how much weight lie above a
// logit. With t = -64 log2(e) x / T (and a constant), a token weighs 2^(-t / 64);
// bin b holds those with floor(t) = b, as a count and the sum of what their
// weights miss of the bin's largest, y = 1 - 2^(-frac(t) / 64) in whole steps of
// 2^-33. Whole numbers, so the order of LDS atomics changes nothing, and 4096
// bins reach down to 2^-64 of the largest weight. A place inside a bin is found
// among the bin's own tokens, which a further look at the row collects: sorted
// in LDS where they fit (some hundred at most in a row of a language model's
// logits), else by digits of their logits.
//
// The bins do not hang on the row's largest logit, so one look fills them: they
// lie in a circle, and where a chunk of the row has a larger logit than all
// before, the bins that fall out at the far end are cleared for it.
//
// Logits in bf16 take few values: from 2^-24 to 2^8 there are 4096 of either
// sign. There a row is counted by its values themselves, six instructions a
// logit and no exponential but one a value; rows that reach beyond (an
// infinity, a place among the tiny ones) go the way of the others.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <string>

#include "../../include/sangam_sample.h"
#include "entry.h"
#include "exact_sum.h"
#include "wave_sum.h"

namespace sangam {
void set_error(const std::string& msg);
void clear_error();
}  // namespace sangam

using namespace sangam;

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 4096;
constexpr int kEach = kBins / kThreads;  // bins of a thread
constexpr int kList = kThreads;          // tokens of a bin that are sorted
constexpr int kMaxVocab = 1 << 18;
// Logits of a thread in a chunk, all on their way together: where a work-group
// takes a whole row, and where it takes a part of one.
template <typename T>
constexpr int kWhole = 128 / int(sizeof(T));
constexpr int kPart = 16;

// t's constant. From 2^20 to 2^21 a double's upper word ends in its whole part
// (|x / T| up to 5,600), and its fraction has steps of 2^-32.
constexpr double kOrigin = 0x1.8p20, kLowest = 0x1p20, kHighest = 0x1p21;

// A bin or digit: the sum over its tokens of 2^52 + 2^45 + y, y what the weight
// misses in units of 2^-33 of the bin's largest weight, as the bits of that double:
// the bits from 45 on add up an odd number a token modulo 2^19, those below y
// (2^18 tokens miss under 2^44.5 units). So what is added is what the last step of
// the polynomial gives, without a further instruction.
constexpr int kMissBits = 45;
constexpr double kCounted = 0x1p52 + 0x1p45;
constexpr uint64_t kOne = uint64_t(1) << 33;
constexpr uint32_t kCode = 0x43302000u >> 13;  // of a token
constexpr uint32_t inverse(uint32_t x) {       // modulo 2^32
    uint32_t y = x;
    for (int k = 0; k < 5; ++k) y *= 2 - x * y;
    return y;
}
static_assert(kCode * inverse(kCode) == 1);
__device__ __forceinline__ int tokens_in(uint64_t bin) { return int((uint32_t(bin >> kMissBits) * inverse(kCode)) & 0x7FFFFu); }
__device__ __forceinline__ uint64_t weight_in(uint64_t bin) {  // in units of 2^-33
    return tokens_in(bin) * kOne - (bin & ((uint64_t(1) << kMissBits) - 1));
}

struct SampleArgs {
    const void* logits;
    int64_t row_stride;
    const float* u;
    const int32_t* params_of;
    int64_t num_params;
    const float* temperatures;
    const int32_t* top_ks;
    const float* top_ps;
    const float* min_ps;
    float temperature;
    int32_t top_k;
    float top_p, min_p;
    int32_t vocab, confidence, forbid;
    int32_t* tokens;
    float* conf;
};

// Values of bf16 by the bits without the sign: those up to kTiny count as 0, those
// from kHuge on have no value (infinities and what is no number among them).
constexpr int kTiny = (127 - 24) * 128 - 1, kHuge = (127 + 8) * 128;
constexpr int kSide = kHuge - kTiny + 1;  // counts of a sign: tiny, the values, huge
constexpr int kValues = kSide - 2;        // of a sign
constexpr int kRanked = 2 * kValues;      // values in rank order; the tiny ones lie in the middle, without a place

// What a look at a row or a part of it gives.
struct Counts {
    union {
        struct {
            uint64_t bins[kBins];  // of floor(t) mod kBins
            uint64_t beyond;       // where what is too low for a bin goes
        };
        uint32_t counts[2 * kSide];
    };
    float wave_top[2][kWaves];
    double wave_sums[2 * kWaves];
    int32_t first_token;
};

// E: logits of a thread in a chunk.
template <int E>
struct Shared : Counts {
    static constexpr int kTops = kMaxVocab / E;
    union {
        struct {
            uint64_t list[kList];    // key and index; then the weight up to each
            union {
                uint64_t sorted[kList];
                uint16_t queue[4 * kList];  // entries of tops to be looked at again
            };
        };
        uint64_t digits[256];
    };
    alignas(16) uint16_t tops[kTops];  // the largest logit of a thread's chunk (rounded up to 16 bits); entry chunk * kThreads + thread
    uint64_t part[2 * kWaves];
    uint64_t block_mass[64];  // of a 64th of the bins or values
    int32_t block_tokens[64];
    double sums[2 * kWaves];
    uint64_t found_mass, found_bin;
    int found, found_tokens, found_last, listed, queued;
    int32_t index;
    double powers[64];  // 2^(-k / 64)

    // The largest weight of the row's b-th bin.
    __device__ __forceinline__ double bin_weight(int b) const { return __builtin_ldexp(powers[b & 63], -(b >> 6)); }
    // Units of 2^-33 of a bin's largest weight as units of 2^-44 of the first bin's.
    __device__ __forceinline__ uint64_t mass_of(int b, uint64_t v) const { return uint64_t(__builtin_rint(bin_weight(b) * double(v) * 2048.0)); }
    // And back.
    __device__ __forceinline__ double inside(int b, double mass) const { return mass / (bin_weight(b) * 2048.0); }
};

// Keys of 32 bits in rank order: the larger the logit, the smaller the key.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);  // -0 equals 0
    return (b >> 31) ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float((key >> 31) ? key : ~key & 0x7FFFFFFFu); }

// The upper 16 bits of the least such number not below x (no number: +inf).
__device__ __forceinline__ uint16_t rounded_up(float x) {
    const uint32_t b = __float_as_uint(x);
    if (!(x == x)) return 0x7F80;
    return uint16_t(((b >> 31) ? b : b + 0xFFFFu) >> 16);
}
__device__ __forceinline__ float from_upper(uint16_t h) { return __uint_as_float(uint32_t(h) << 16); }

// What a token at a fraction f of a bin adds to it: y = 2^33 (1 - 2^(-f / 64)) by
// a cubic without constant, fitted over [0, 1) and off by 5.3e-12 = 0.05 units.
// (Written as instructions: the compiler copies constants for the shorter v_fmac.)
__device__ __forceinline__ uint64_t added_at(double f) {
    constexpr double q1 = 0x1.62e42fb615b67p-7 * 0x1p33, q2 = -0x1.ebfa827a93283p-15 * 0x1p33, q3 = 0x1.c454fdc63ddabp-23 * 0x1p33;
    double y;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(y) : "v"(f), "s"(q3), "v"(q2));
    asm("v_fma_f64 %0, %1, %0, %2" : "+v"(y) : "v"(f), "v"(q1));
    asm("v_fma_f64 %0, %1, %0, %2" : "+v"(y) : "v"(f), "v"(kCounted));
    return __builtin_bit_cast(uint64_t, y);
}
__device__ __forceinline__ uint32_t miss_at(double f) { return uint32_t(added_at(f)); }

// A value that all lanes hold, in scalar registers.
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float scalar(float x) { return __uint_as_float(uint32_t(scalar(int(__float_as_uint(x))))); }
__device__ __forceinline__ uint64_t scalar(uint64_t x) { return uint64_t(uint32_t(scalar(int(x >> 32)))) << 32 | uint32_t(scalar(int(x))); }
__device__ __forceinline__ double scalar(double x) { return __builtin_bit_cast(double, scalar(__builtin_bit_cast(uint64_t, x))); }

__device__ __forceinline__ void add_to(uint64_t* bin, uint64_t more) { atomicAdd(reinterpret_cast<unsigned long long*>(bin), more); }

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

__device__ __forceinline__ int lane_of(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ uint64_t lane_of(uint64_t x, int lane) {
    return uint64_t(uint32_t(lane_of(int(x >> 32), lane))) << 32 | uint32_t(lane_of(int(x), lane));
}

__device__ __forceinline__ double lane_of(double x, int lane) { return __builtin_bit_cast(double, lane_of(__builtin_bit_cast(uint64_t, x), lane)); }

// Sum over the threads before this one, and over all.
template <int E>
__device__ __forceinline__ uint64_t sum_before(Shared<E>& sh, uint64_t x, uint64_t* total) {
    const int wave = threadIdx.x / 64;
    const uint64_t up_to = wave_up_to(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh.part[wave] = up_to;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint64_t p = sh.part[w];
        if (w < wave) before += p;
        all += p;
    }
    *total = scalar(all);
    return before + up_to - x;
}

// The same for two at once: before becomes what lies before this thread, all the sums.
template <int E>
__device__ __forceinline__ void sums_before(Shared<E>& sh, uint64_t x, uint64_t y, uint64_t (&before)[2], uint64_t (&all)[2]) {
    const int wave = threadIdx.x / 64;
    const uint64_t up_to[2] = {wave_up_to(x), wave_up_to(y)};
    __syncthreads();
    if ((threadIdx.x & 63) == 63) {
        sh.part[wave] = up_to[0];
        sh.part[kWaves + wave] = up_to[1];
    }
    __syncthreads();
    before[0] = up_to[0] - x;
    before[1] = up_to[1] - y;
    uint64_t total[2] = {0, 0};
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint64_t p = sh.part[k * kWaves + w];
            if (w < wave) before[k] += p;
            total[k] += p;
        }
    all[0] = scalar(total[0]);
    all[1] = scalar(total[1]);
}

// Sums over all threads, in a fixed order.
template <int E>
__device__ __forceinline__ void sum_all(Shared<E>& sh, double& x, double& y) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        x += __shfl_xor(x, d);
        y += __shfl_xor(y, d);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        sh.sums[threadIdx.x / 64] = x;
        sh.sums[kWaves + threadIdx.x / 64] = y;
    }
    __syncthreads();
    x = y = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        x += sh.sums[w];
        y += sh.sums[kWaves + w];
    }
}

// A row of logits, or a part of one: vectors [first, last) of it, and with the
// first part the elements outside all vectors.
template <typename T, int E>
struct Row {
    static constexpr int V = 16 / int(sizeof(T));
    static constexpr int kLoads = E / V;
    static constexpr int kChunk = kThreads * kLoads;  // vectors of a chunk
    typedef T Vec __attribute__((ext_vector_type(V)));
    const T* p;
    int vocab, forbid;
    int head, vectors;  // elements before the first aligned vector; vectors of the row
    int first, last;
    bool infinite;      // some logit is +inf: those count as 0, all others as -inf
    bool wide;          // t is relative to the largest logit, as x / T is large
    double top, scale;  // wide: t = (top - x) scale, else kOrigin - x scale
    int base;           // floor(t) of the largest logit

    __device__ __forceinline__ float adjusted(float x, int i) const {
        if (i == forbid) x = -INFINITY;
        if (infinite) x = x == INFINITY ? 0.0f : -INFINITY;
        return x;
    }
    __device__ __forceinline__ float at(int i) const { return adjusted(float(p[i]), i); }
    __device__ __forceinline__ double t_of(float x) const { return wide ? (top - double(x)) * scale : __builtin_fma(-double(x), scale, kOrigin); }
    __device__ __forceinline__ const Vec* body() const { return reinterpret_cast<const Vec*>(p + head); }
    __device__ __forceinline__ void unpack(const Vec& w, int i0, float (&x)[V]) const {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = float(w[e]);
        if (unsigned(forbid - i0) < unsigned(V)) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (i0 + e == forbid) x[e] = -INFINITY;
        }
        if (infinite) {
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = x[e] == INFINITY ? 0.0f : -INFINITY;
        }
    }
    // the part's vectors, a chunk after the other: f(number of the chunk in the row, first vector of the chunk, vectors)
    template <typename F>
    __device__ __forceinline__ void each_chunk(F f) const {
        const Vec* const v = body();
#pragma unroll 1
        for (int v0 = first; v0 < last; v0 += kChunk) {
            Vec w[kLoads];
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int k = v0 + j * kThreads + int(threadIdx.x);
                if (k < last) w[j] = v[k];
            }
            f(v0 / kChunk, v0, w);
        }
    }
    // f(first index, logits) of a chunk's vectors
    template <typename F>
    __device__ __forceinline__ void each_of(int v0, const Vec (&w)[kLoads], F f) const {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int k = v0 + j * kThreads + int(threadIdx.x);
            if (k >= last) continue;
            float x[V];
            unpack(w[j], head + k * V, x);
            f(head + k * V, x);
        }
    }
    // the elements outside all vectors, with the first part
    template <typename F>
    __device__ __forceinline__ void each_edge(F f) const {
        const int rest = first == 0 ? vocab - vectors * V : 0;
        for (int k = threadIdx.x; k < rest; k += kThreads) {
            const int i = k < head ? k : k + vectors * V;
            f(i, at(i));
        }
    }
    // A little under all logits of the row's first n bins, and a little above those behind the first n. The little: a part of the
    // border, rounded to 32 bits, and what t is rounded by (2^-33 around kOrigin, else 2^-52 of the numbers it is made of), which
    // alone counts at a border near 0: logits of +-1e-20 have the t of 0.
    __device__ __forceinline__ double border(int n, double side) const {
        const double x = wide ? top - n / scale : (kOrigin - double(base + n)) / scale;
        return x + side * (fabs(x) * 0x1p-22 + (wide ? (fabs(top) + n / scale) * 0x1p-48 : 0x1p-30 / scale));
    }
    __device__ __forceinline__ float lowest(int n) const { return scale > 0.0 ? scalar(float(fmax(border(n, -1.0), -3.5e38))) : -INFINITY; }
    __device__ __forceinline__ float highest(int n) const { return scale > 0.0 ? scalar(float(border(n, 1.0))) : INFINITY; }
    // All logits of the row from `low` to `high`. Where tops says that few chunks of
    // threads hold any, these are listed, and the vectors in them dealt over all
    // threads, so that they come in one or two rounds of loads (a thread that walked
    // its own chunks took one after the other: 18 us for a bin of a row of 152,064).
    // f(vectors on their way together, which of the row each is, or `vectors`)
    template <int AT_ONCE, typename F>
    __device__ __forceinline__ void each_reaching(Shared<E>& sh, float low, F f) const {
        __syncthreads();
        if (threadIdx.x == 0) sh.queued = 0;
        __syncthreads();
        const int entries = (vectors + kChunk - 1) / kChunk * kThreads;
#pragma unroll 4
        for (int e = threadIdx.x; e < entries; e += kThreads) {
            if (from_upper(sh.tops[e]) < low) continue;
            const int k = atomicAdd(&sh.queued, 1);
            if (k < 4 * kList) sh.queue[k] = uint16_t(e);
        }
        __syncthreads();
        const int queued = scalar(sh.queued);
        const bool all = queued > 4 * kList;
        const int items = all ? vectors : queued * kLoads;
        const Vec* const v = body();
#pragma unroll 1
        for (int k0 = threadIdx.x; k0 < items; k0 += AT_ONCE * kThreads) {
            Vec w[AT_ONCE];
            int k[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const int item = k0 + j * kThreads;
                k[j] = vectors;
                if (item < items) {
                    const int e = all ? 0 : sh.queue[item / kLoads];
                    k[j] = all ? item : e / kThreads * kChunk + item % kLoads * kThreads + e % kThreads;
                }
                if (k[j] < vectors) w[j] = v[k[j]];
            }
            f(w, k);
        }
    }
    template <typename F>
    __device__ __forceinline__ void each_within(Shared<E>& sh, float low, float high, F f) const {
        each_reaching<2>(sh, low, [&](const Vec(&w)[2], const int(&k)[2]) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (k[j] >= vectors) continue;
                float x[V];
                unpack(w[j], head + k[j] * V, x);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (x[e] >= low && x[e] <= high) f(head + k[j] * V + e, x[e]);
                    __builtin_amdgcn_sched_barrier(0);  // (side by side they take twice the registers)
                }
            }
        });
        each_edge([&](int i, float x) {
            if (x >= low && x <= high) f(i, x);
        });
    }
};

// A prefix of the ranks: all tokens of the bins before `bin`, and the first
// `tokens` of that bin, which end with `ties` tokens of key `key`.
struct Prefix {
    int bin, tokens, ties;
    uint32_t key;
    uint64_t weight;     // of those of the bin, units of 2^-33 of its largest
    uint64_t mass;       // of the bins before, units of 2^-44
    int before;          // tokens of the bins before
    template <int E>
    __device__ uint64_t all(const Shared<E>& sh) const { return mass + (tokens ? sh.mass_of(bin, weight) : 0); }
};

// What a place on the axis of ranks is given by: the number of tokens up to it,
// weight before its token, weight up to its token, a lowest logit.
enum class By { kCount, kReach, kAbove, kCut };

template <typename T, int E>
struct Bin {
    Shared<E>& sh;
    const Row<T, E>& row;
    int listed;  // bin whose tokens sh.sorted and sh.list hold

    // its place in the bin, 0 to 1; outside: another bin's
    __device__ __forceinline__ double place(float x, int b) const { return row.t_of(x) - double(row.base + b); }
    __device__ __forceinline__ uint64_t weight_of(uint32_t key, int b) const { return kOne - miss_at(place(logit_of(key), b)); }

    // Tokens of bin b, in rank order, and their weights summed up.
    __device__ __forceinline__ void collect(int b, int n) {
        if (listed == b) return;
        __syncthreads();
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        row.each_within(sh, row.lowest(b + 1), row.highest(b), [&](int i, float x) {
            const double f = place(x, b);
            if (f >= 0.0 && f < 1.0) {
                const int k = atomicAdd(&sh.listed, 1);
                if (k < kList) sh.list[k] = (uint64_t(key_of(x)) << 32) | uint32_t(i);
            }
        });
        __syncthreads();
        const int k = threadIdx.x;
        if (k < n) {
            const uint64_t mine = sh.list[k];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += sh.list[j] < mine;
            sh.sorted[rank] = mine;
        }
        __syncthreads();
        const uint64_t w = k < n ? weight_of(uint32_t(sh.sorted[k] >> 32), b) : 0;
        uint64_t total;
        const uint64_t before = sum_before(sh, w, &total);
        if (k < n) sh.list[k] = before + w;
        __syncthreads();
        listed = b;
    }
    // How many of n entries, in order, satisfy what the first ones do.
    template <typename F>
    __device__ static int leading(int n, F f) {
        int lo = 0, hi = n;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (f(mid)) lo = mid + 1;
            else hi = mid;
        }
        return scalar(lo);
    }

    // The bin's first tokens up to a place, by digits of the keys; p.ties - 1 tokens with the last one's key are before it. (Few
    // rows of a language model have so many in a bin. 126,464 equal logits, each look an atomic of one digit and then one
    // after the other for the index, in fp32: a row 520 us, 300 rows 1,160, where normal ones take 48 and 97.)
    __device__ __forceinline__ void descend(Prefix& p, By by, int count, double weight, uint32_t cut, int most) {
        listed = -1;
        const int d = threadIdx.x, b = p.bin;
        uint32_t key = 0;
        int before = 0, equal = 0;
        uint64_t weight_before = 0;
#pragma unroll 1
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (d < 256) sh.digits[d] = 0;
            if (d == 0) sh.found = sh.found_last = -1;
            __syncthreads();
            row.each_within(sh, row.lowest(b + 1), row.highest(b), [&](int, float x) {
                const double f = place(x, b);
                if (!(f >= 0.0 && f < 1.0)) return;
                const uint32_t k = key_of(x);
                if ((uint64_t(k) >> (shift + 8)) != (uint64_t(key) >> (shift + 8))) return;
                add_to(&sh.digits[(k >> shift) & 255], added_at(f));
            });
            __syncthreads();
            const uint64_t bin = d < 256 ? sh.digits[d] : 0;
            const int more = tokens_in(bin);
            uint64_t up_to[2], total[2];
            sums_before(sh, uint64_t(more), weight_in(bin), up_to, total);
            const int n = before + int(up_to[0]);
            const uint64_t w = weight_before + up_to[1], after = w + weight_in(bin);
            const bool here = by == By::kCount   ? n < count && n + more >= count
                              : by == By::kReach ? double(w) < weight && double(after) >= weight
                              : by == By::kAbove ? double(w) <= weight && double(after) > weight
                                                 : d == int((cut >> shift) & 255);
            if (more > 0) atomicMax(&sh.found_last, d);
            if (here) sh.found = d;
            __syncthreads();
            const int at = sh.found >= 0 ? sh.found : sh.found_last;  // (behind all: the last one)
            if (d == at) {
                sh.found_tokens = n;
                sh.found_mass = w;
                sh.found_bin = bin;
            }
            __syncthreads();
            key |= uint32_t(scalar(at)) << shift;
            before = scalar(sh.found_tokens);
            weight_before = scalar(sh.found_mass);
            equal = tokens_in(scalar(sh.found_bin));
        }
        const uint64_t each = scalar(weight_of(key, b));
        // tokens with this key up to the place; kReach: the last that has less than `weight` before it; kAbove: the first with more up to it
        const double into = (weight - double(weight_before)) / double(each);
        int ties = equal;
        if (by != By::kCut) {
            ties = by == By::kCount ? count - before : by == By::kReach ? int(ceil(into)) : int(floor(into)) + 1;
            ties = scalar(max(1, min(ties, min(equal, most - before))));
        }
        p.tokens = before + ties;
        p.ties = ties;
        p.key = key;
        p.weight = weight_before + uint64_t(ties) * each;
    }
    // Index of the last of p's tokens.
    __device__ __forceinline__ int index_of(const Prefix& p) {
        uint64_t before = 0;
#pragma unroll 1
        for (int i0 = 0; i0 < row.vocab; i0 += 8 * kThreads) {
            const int i = i0 + 8 * int(threadIdx.x);
            uint64_t mine = 0, total;
#pragma unroll 1
            for (int e = 0; e < 8; ++e)
                if (i + e < row.vocab) {
                    const float x = row.at(i + e);
                    mine += x == x && key_of(x) == p.key;
                }
            uint64_t left = uint64_t(p.ties - 1) - before - sum_before(sh, mine, &total);
            if (left < mine) {
#pragma unroll 1
                for (int e = 0; e < 8; ++e)
                    if (i + e < row.vocab) {
                        const float x = row.at(i + e);
                        if (x == x && key_of(x) == p.key && left-- == 0) sh.index = i + e;
                    }
            }
            before += total;
            if (before >= uint64_t(p.ties)) break;
        }
        __syncthreads();
        return scalar(sh.index);
    }

    // p's first tokens of its bin (which holds n): up to `count` of them, or those with less than `weight` before them, or up
    // to the first with more than `weight` up to it (at most `most`), or those with a key up to `cut`. Returns the last one's
    // index where it is at hand, else -1.
    __device__ __forceinline__ int first(Prefix& p, int n, By by, int count, double weight, uint32_t cut, int most) {
        if (n > kList) {
            descend(p, by, count, weight, cut, most);
            return -1;
        }
        collect(p.bin, n);
        const int m = by == By::kCount   ? count
                      : by == By::kReach ? max(1, leading(n, [&](int i) { return i == 0 || double(sh.list[i - 1]) < weight; }))
                      : by == By::kAbove ? min(leading(n, [&](int i) { return double(sh.list[i]) <= weight; }), most - 1) + 1
                                         : leading(n, [&](int i) { return uint32_t(sh.sorted[i] >> 32) <= cut; });
        p.tokens = m;
        p.weight = 0;
        if (m == 0) return -1;
        const uint64_t last = scalar(sh.sorted[m - 1]);
        p.key = uint32_t(last >> 32);
        p.ties = m - leading(m, [&](int i) { return uint32_t(sh.sorted[i] >> 32) < p.key; });
        p.weight = scalar(sh.list[m - 1]);
        return int(uint32_t(last));
    }
};

// Parameters of a row, as the header defines them.
struct Params {
    float temperature, top_p, min_p, u;
    int top_k;
    bool none;  // the row's entry is outside: nothing is taken
    __device__ bool whole() const { return temperature == 0.0f && top_k == 0 && top_p >= 1.0f && min_p <= 0.0f; }
};

__device__ __forceinline__ Params params_of(const SampleArgs& a, int64_t r) {
    Params p{};
    const int64_t of = a.params_of ? a.params_of[r] : r;
    p.none = (a.params_of || a.temperatures || a.top_ks || a.top_ps || a.min_ps) && (of < 0 || of >= a.num_params);
    if (p.none) return p;
    p.temperature = a.temperatures ? a.temperatures[of] : a.temperature;
    if (!(p.temperature > 0.0f)) p.temperature = 0.0f;
    p.u = a.u[r];
    p.top_k = a.top_ks ? a.top_ks[of] : a.top_k;
    if (p.top_k < 1 || p.top_k >= a.vocab) p.top_k = 0;
    p.top_p = a.top_ps ? a.top_ps[of] : a.top_p;
    if (!(p.top_p < 1.0f)) p.top_p = 1.0f;
    p.min_p = a.min_ps ? a.min_ps[of] : a.min_p;
    if (!(p.min_p > 0.0f)) p.min_p = 0.0f;
    return p;
}

__device__ __forceinline__ void answer(const SampleArgs& a, int64_t r, int token, double c) {
    if (threadIdx.x == 0) {
        a.tokens[r] = token;
        if (a.conf) a.conf[r] = float(c);
    }
}

// The bins of a row or part, whose largest logit becomes `top`.
enum Filled : int32_t { kFar, kFilled, kNothing };  // kFar: its x / T is too large, or infinite, for bins that do not hang on it
template <typename T, int E>
__device__ __forceinline__ Filled fill(Counts& sh, Row<T, E>& row, float& top, uint16_t* tops) {
    constexpr int V = Row<T, E>::V;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    top = -INFINITY;
    if (!(row.scale > 1e-30)) return kFar;  // (all that is finite may weigh the same)
    bool low = false;  // logits below all bins
    int parity = 0;
    // a chunk's largest logit is in: whether its logits are to be added
    auto raise = [&](float mine) {
        mine = wave_max(mine);
        if (lane == 0) sh.wave_top[parity][wave] = mine;
        __syncthreads();
        float m = sh.wave_top[parity][0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sh.wave_top[parity][w]);
        parity ^= 1;
        if (!(m > top)) return top > -INFINITY;
        const double t = row.t_of(m);
        if (t >= kHighest) {  // so low that bins may not be kept for it
            low = true;
            return false;
        }
        const int to = t >= kLowest ? int(t) : 0;
        if (top > -INFINITY) {
            for (int b = to + tid; b < row.base && b < to + kBins; b += kThreads) sh.bins[b & (kBins - 1)] = 0;
            __syncthreads();
        }
        top = scalar(m);
        row.base = scalar(to);
        return to > 0;
    };
    // the lowest logit that has a bin, with the last one to spare (those below weigh nothing)
    auto cut = [&] {
        const float x = float(fmax((kOrigin - double(row.base + kBins - 1)) / row.scale, -3.4e38));
        return scalar(x + fabsf(x) * 0x1p-21f);
    };
    uint64_t* const bins = sh.bins;
    auto add = [&](float x, float lowest) {
        const double t = __builtin_fma(-double(x), row.scale, kOrigin);
        const int at = x >= lowest ? __double2hiint(t) & (kBins - 1) : kBins;
        static_assert(offsetof(Counts, beyond) == kBins * sizeof(uint64_t), "beyond lies behind the bins");
        add_to(bins + at, added_at(__builtin_amdgcn_fract(t)));
    };
    for (int b = tid; b < kBins; b += kThreads) sh.bins[b] = 0;
    row.each_chunk([&](int chunk, int v0, const auto& w) {
        float m = -INFINITY;
        row.each_of(v0, w, [&](int, const float(&x)[V]) {
#pragma unroll
            for (int e = 0; e < V; ++e) m = fmaxf(m, x[e]);
        });
        tops[chunk * kThreads + tid] = rounded_up(m);
        if (!raise(m)) return;
        const float lowest = cut();
        row.each_of(v0, w, [&](int, const float(&x)[V]) {
#pragma unroll
            for (int e = 0; e < V; ++e) add(x[e], lowest);
        });
    });
    if (row.vocab > row.vectors * V) {
        float m = -INFINITY;
        row.each_edge([&](int, float x) { m = fmaxf(m, x); });
        if (raise(m)) {
            const float lowest = cut();
            row.each_edge([&](int, float x) { add(x, lowest); });
        }
    }
    __syncthreads();
    if (top == -INFINITY) return low ? kFar : kNothing;
    return row.base > 0 && row.base + kBins <= int(kHighest) ? kFilled : kFar;
}

// The same by two looks, for any row. False: the row has no weight.
template <typename T, int E>
__device__ __forceinline__ bool fill_wide(Shared<E>& sh, Row<T, E>& row, float& top) {
    constexpr int V = Row<T, E>::V;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    float m = -INFINITY;
    row.each_chunk([&](int chunk, int v0, const auto& w) {
        float own = -INFINITY;
        row.each_of(v0, w, [&](int, const float(&x)[V]) {
#pragma unroll
            for (int e = 0; e < V; ++e) own = fmaxf(own, x[e]);
        });
        sh.tops[chunk * kThreads + tid] = rounded_up(own);
        m = fmaxf(m, own);
    });
    row.each_edge([&](int, float x) { m = fmaxf(m, x); });
    m = wave_max(m);
    __syncthreads();
    if (lane == 0) sh.wave_top[0][wave] = m;
    for (int b = tid; b < kBins; b += kThreads) sh.bins[b] = 0;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, sh.wave_top[0][w]);
    if (m == -INFINITY) return false;
    if (m == INFINITY) {
        row.infinite = true;
        m = 0.0f;
        for (int k = tid; k < Shared<E>::kTops; k += kThreads) sh.tops[k] = 0x7F80;  // (+inf: every chunk is looked at)
        __syncthreads();
    }
    top = scalar(m);
    row.wide = true;
    row.top = scalar(double(m));
    row.base = 0;
    row.each_within(sh, row.lowest(kBins), INFINITY, [&](int, float x) {
        const double t = row.t_of(x);
        if (t < double(kBins)) add_to(&sh.bins[int(t)], added_at(__builtin_amdgcn_fract(t)));
    });
    __syncthreads();
    return true;
}

// A row's answer from its bins: one place on the axis of ranks after the other.
template <typename T, int E>
__device__ __forceinline__ void choose(Shared<E>& sh, const Row<T, E>& row, const SampleArgs& a, const Params& p, int64_t r, float top) {
    const int tid = threadIdx.x;
    const bool greedy = p.temperature == 0.0f;
    auto slot = [&](int b) -> uint64_t { return sh.bins[(row.base + b) & (kBins - 1)]; };
    // blocks of 64 bins, of which each lane of every wave holds one, and what lies up to its end
    static_assert(kBins == 64 * 64, "a block a lane");
    const int lane = tid & 63, wave = tid / 64;
    __syncthreads();
#pragma unroll 1
    for (int block = wave; block < 64; block += kWaves) {
        const int b = 64 * block + lane;
        const uint64_t bin = slot(b), m = sh.mass_of(b, weight_in(bin));
        const int n = wave_up_to(tokens_in(bin));
        const uint64_t w = wave_up_to(m);
        if (lane == 63) {
            sh.block_tokens[block] = n;
            sh.block_mass[block] = w;
        }
    }
    __syncthreads();
    const int block_tokens = sh.block_tokens[lane];
    const uint64_t block_mass = sh.block_mass[lane];
    const int tokens_end = wave_up_to(block_tokens);
    const uint64_t mass_end = wave_up_to(block_mass);
    const int all_tokens = lane_of(tokens_end, 63);
    const uint64_t all_mass = lane_of(mass_end, 63);
    Bin<T, E> bin{sh, row, -1};
    const uint64_t top_weight = scalar(kOne - miss_at(bin.place(top, 0)));
    Prefix kept{kBins, 0, 0, 0, 0, all_mass, all_tokens};
    const Prefix only_first{0, 1, 1, key_of(top), top_weight, 0, 0};
    double unit = 0.0, weight = 0.0, second = 0.0;  // 2^44 / M; of the token; of the second token, if it is kept
    int token = -1;
    // min_p: the lowest logit that is kept, an estimate and then by the definition, and its bin
    uint32_t cut_key = 0;
    int cut_bin = kBins;
    if (p.min_p > 0.0f && p.min_p <= 1.0f) {
        const double T_ = greedy ? 1.0 : double(p.temperature), low = log(double(p.min_p));
        auto keeps = [&](float x) { return (double(x) - double(top)) / T_ >= low; };
        float cut = float(fmax(double(top) + T_ * low, -0x1.fffffep127));  // (the lowest number has weight, too, under a large T)
#pragma unroll 1
        for (int k = 0; k < 4 && !keeps(cut); ++k) cut = nextafterf(cut, INFINITY);
#pragma unroll 1
        for (int k = 0; k < 4; ++k) {
            const float lower = nextafterf(cut, -INFINITY);
            if (!(lower > -INFINITY) || !keeps(lower)) break;
            cut = lower;
        }
        cut = fminf(cut, top);
        const double t = row.t_of(cut) - double(row.base);
        cut_key = uint32_t(scalar(int(key_of(cut))));
        cut_bin = t < double(kBins) ? scalar(int(t)) : kBins + 1;
    }
    enum Stage { kTopK, kTopP, kMinP, kDraw, kSecond, kStages };
#pragma unroll 1
    for (int stage = kTopK; stage < kStages; ++stage) {
        // the place: the bin whose end is the first at or above `reach`, counted in tokens, weight or bins
        By by = By::kCount;
        uint64_t reach = 0;
        double target = 0.0;
        if (stage == kTopK) {
            if (p.top_k == 0 || p.top_k >= all_tokens) continue;
            reach = uint64_t(p.top_k);
        } else if (stage == kTopP) {
            if (!(p.top_p < 1.0f)) continue;
            target = scalar(ceil(double(p.top_p) * double(kept.all(sh))));
            if (!(target > 0.0)) {
                kept = only_first;
                continue;
            }
            by = By::kReach;
            reach = uint64_t(target);
        } else if (stage == kMinP) {
            if (!(p.min_p > 0.0f)) continue;
            if (p.min_p > 1.0f) {
                kept = only_first;
                continue;
            }
            if (cut_bin > kept.bin) continue;
            by = By::kCut;
            reach = uint64_t(cut_bin) + 1;
        } else if (stage == kDraw) {
            const uint64_t M = scalar(kept.all(sh));
            unit = scalar(0x1p44 / double(M));
            if (!greedy && p.u >= 1.0f) {  // the last that is kept, by its number: M may be reached before it, by less than a unit of 2^-44
                reach = uint64_t(kept.before + kept.tokens);
            } else {
                target = scalar(!greedy && p.u > 0.0f ? double(p.u) * double(M) : 0.0);
                by = By::kAbove;
                reach = scalar(min(uint64_t(target) + 1, M));  // (the sums of long flat rows are beyond 2^53: a target may round up to M)
            }
        } else {
            if (a.confidence != SANGAM_CONFIDENCE_MARGIN || kept.before + kept.tokens < 2) continue;
            reach = 2;
        }
        const uint64_t block_end = by == By::kCount ? uint64_t(tokens_end) : by == By::kCut ? uint64_t(64 * lane + 64) : mass_end;
        const uint64_t block_size = by == By::kCount ? uint64_t(block_tokens) : by == By::kCut ? 64 : block_mass;
        const uint64_t in = __ballot(block_end - block_size < reach && block_end >= reach);
        if (in == 0) continue;  // (not met)
        const int at = __builtin_ctzll(in), mine = 64 * at + lane;
        const uint64_t own = slot(mine), m = sh.mass_of(mine, weight_in(own));
        const int n_end = lane_of(tokens_end - block_tokens, at) + wave_up_to(tokens_in(own));
        const uint64_t m_end = lane_of(mass_end - block_mass, at) + wave_up_to(m);
        const uint64_t end = by == By::kCount ? uint64_t(n_end) : by == By::kCut ? uint64_t(mine) + 1 : m_end;
        const int k = __builtin_ctzll(__ballot(end >= reach) | (uint64_t(1) << 63));
        const int n = lane_of(tokens_in(own), k);
        Prefix q{64 * at + k, 0, 0, 0, 0, lane_of(m_end - m, k), lane_of(n_end, k) - n};
        if (q.bin > kept.bin) continue;  // (not met within what is kept)
        const double into = by == By::kReach || by == By::kAbove ? scalar(fmax(0.0, sh.inside(q.bin, target - double(q.mass)))) : 0.0;
        int index = -1;
        // (a draw at the end of what is kept of this bin is given by the number of its tokens, or it would fall on the one behind)
        const bool at_end = stage == kDraw && q.bin == kept.bin && into >= double(kept.weight);
        if (n > 0)
            index = bin.first(q, n, at_end ? By::kCount : by, at_end ? kept.tokens : int(reach) - q.before, into, cut_key, q.bin == kept.bin ? kept.tokens : n);
        if (stage <= kMinP) {
            if (q.bin < kept.bin || q.tokens < kept.tokens) kept = q;
        } else if (stage == kDraw) {
            token = index >= 0 ? index : bin.index_of(q);
            weight = scalar(sh.bin_weight(q.bin) * double(bin.weight_of(q.key, q.bin)) * 0x1p-33);
        } else {
            second = scalar(sh.bin_weight(q.bin) * double(bin.weight_of(q.key, q.bin)) * 0x1p-33);
        }
    }
    double c = weight * unit;
    if (a.confidence == SANGAM_CONFIDENCE_MARGIN) {
        c = (double(top_weight) * 0x1p-33 - second) * unit;
    } else if (a.confidence == SANGAM_CONFIDENCE_ENTROPY) {
        // (which thread gets which logits hangs on the order of LDS atomics. Sums in doubles would do so, too, and take 600 rows
        // of 50,257 in fp32 under a nucleus in 119 us instead of 123, 300 unfiltered ones of 126,464 in fp16 in 146 instead of 159)
        ExactSum sum{};
        auto part = [&](double t) { return sh.bin_weight(int(t)) * double(kOne - miss_at(t - int(t))) * 0x1p-33 * t; };
        row.each_within(sh, row.lowest(min(kept.bin + 1, kBins)), INFINITY, [&](int, float x) {
            const double t = bin.place(x, 0);
            if (t < double(kept.bin) || (kept.tokens > 0 && t < double(kept.bin + 1) && key_of(x) < kept.key)) sum.add(part(t));  // (under 34)
        });
        uint64_t before[2], all[2];
        sums_before(sh, sum.high, sum.low, before, all);
        double s = ExactSum{all[0], all[1]}.value();
        if (kept.tokens > 0 && kept.ties > 0) s += kept.ties * part(bin.place(logit_of(kept.key), 0));
        c = -(s * unit * (0.69314718055994530942 / 64) - log(unit));
    }
    answer(a, r, token, c);
}

// ---------------------------------------------------------------- rows of bf16

// Adds a part of a row to the counts, which are all there behind the next barrier.
template <int E>
__device__ __forceinline__ void count(Counts& sh, const Row<__bf16, E>& row, uint16_t* tops) {
    uint32_t* const counts = sh.counts;
    // (a value: its bits without the sign, held to [kTiny, kHuge], and the side: sign 0 or -1)
    auto add = [&](uint32_t bits, int32_t sign) {
        const uint32_t v = min(max(bits, uint32_t(kTiny)), uint32_t(kHuge));
        atomicAdd(counts + (int(v) + ((sign & (kSide - kTiny)) | (~sign & -kTiny))), 1u);
    };
    row.each_chunk([&](int chunk, int v0, const auto& w) {
        // the largest as whole numbers: where some are positive that of int32, else the smallest of uint32
        int32_t most = INT32_MIN;
        uint32_t least = UINT32_MAX;
#pragma unroll
        for (int j = 0; j < Row<__bf16, E>::kLoads; ++j) {
            if (v0 + j * kThreads + int(threadIdx.x) >= row.last) continue;
            typedef uint32_t U4 __attribute__((ext_vector_type(4)));
            const U4 u = __builtin_bit_cast(U4, w[j]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t low = u[e] << 16;
                add(u[e] & 0x7FFFu, int32_t(low) >> 31);
                add((u[e] >> 16) & 0x7FFFu, int32_t(u[e]) >> 31);
                // (the lower half behind the upper one changes no order of upper halves)
                most = max(max(most, int32_t(low)), int32_t(u[e]));
                least = min(min(least, low), u[e]);
            }
        }
        tops[chunk * kThreads + threadIdx.x] = uint16_t((most >= 0 ? uint32_t(most) : least) >> 16);
    });
    const int rest = row.first == 0 ? row.vocab - row.vectors * row.V : 0;
    auto bits_of = [&](int i) { return uint32_t(__builtin_bit_cast(uint16_t, row.p[i])); };
    if (int(threadIdx.x) < rest) {
        const uint32_t u = bits_of(int(threadIdx.x) < row.head ? int(threadIdx.x) : int(threadIdx.x) + row.vectors * row.V);
        add(u & 0x7FFFu, -int32_t(u >> 15));
    }
}

// f(index) of all logits equal to x (not 0): two at a time, by what the bits differ in.
template <int E, typename F>
__device__ __forceinline__ void each_equal(Shared<E>& sh, const Row<__bf16, E>& row, float x, F f) {
    typedef uint16_t Halves __attribute__((ext_vector_type(8)));
    typedef uint16_t Two __attribute__((ext_vector_type(2)));
    const uint16_t bits = uint16_t(__float_as_uint(x) >> 16);
    auto found = [&](int i) {
        if (i != row.forbid) f(i);
    };
    constexpr int kAtOnce = 8;
    row.template each_reaching<kAtOnce>(sh, x, [&](const auto& w, const int(&k)[kAtOnce]) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (k[j] >= row.vectors) continue;
            const Halves off = __builtin_bit_cast(Halves, w[j]) ^ bits;
            const Two least = __builtin_elementwise_min(__builtin_elementwise_min(off.s01, off.s23), __builtin_elementwise_min(off.s45, off.s67));
            if (least.x != 0 && least.y != 0) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (off[e] == 0) found(row.head + k[j] * 8 + e);
        }
    });
    row.each_edge([&](int i, float y) {
        if (y == x) found(i);
    });
}

// Takes the forbidden token out of the counts again.
template <int E>
__device__ __forceinline__ void uncount(Shared<E>& sh, const Row<__bf16, E>& row) {
    if (threadIdx.x != 0 || row.forbid < 0) return;
    const uint32_t u = __builtin_bit_cast(uint16_t, row.p[row.forbid]);
    const int v = min(max(int(u & 0x7FFFu), kTiny), kHuge) - kTiny;
    sh.counts[v + ((u & 0x8000u) ? kSide : 0)] -= 1;
}

// Values in rank order: place q's logit, and how many tokens have it.
__device__ __forceinline__ float value_at(int q) {
    return __uint_as_float(q < kValues ? uint32_t(kTiny + kValues - q) << 16 : (uint32_t(kTiny + 1 + q - kValues) << 16) | 0x80000000u);
}
__device__ __forceinline__ int count_at(const Counts& sh, int q) { return int(sh.counts[q < kValues ? kValues - q : kSide + 1 + q - kValues]); }

// A prefix of the ranks: all tokens of the values before q, and the first
// `tokens` of that value.
struct ValuePrefix {
    int q, tokens, before;
    double mass;  // of the values before, the largest weight being 1
};

// A row's answer from its counts; false: they do not tell. Every wave looks for
// the places by itself: a lane holds what lies up to the end of a block of 128
// values, and looks at two values of the block that a place lies in. Weights are
// added up in 64 bits, in an order that is always the same.
template <int E>
__device__ __forceinline__ bool choose_by_value(Shared<E>& sh, Row<__bf16, E>& row, const SampleArgs& a, const Params& p, int64_t r) {
    constexpr int kBlock = kRanked / 64, kSteps = 64 / kWaves;
    static_assert(kBlock == 128, "two values a lane");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    // the thread's values: two of each block kWaves i + wave, and the largest value
    int own[kSteps][2], q0 = kRanked;
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) own[i][h] = count_at(sh, (i * kWaves + wave) * kBlock + 64 * h + lane);
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i)
#pragma unroll
        for (int h = 1; h >= 0; --h) {
            const uint64_t some = __ballot(own[i][h] > 0);
            if (some) q0 = (i * kWaves + wave) * kBlock + 64 * h + __builtin_ctzll(some);
        }
    if (lane == 0) sh.block_tokens[wave] = q0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) q0 = min(q0, sh.block_tokens[w]);
    q0 = scalar(q0);
    const int tiny = scalar(int(sh.counts[0] + sh.counts[kSide]));
    if (q0 == kRanked || (tiny > 0 && q0 >= kValues) || sh.counts[kSide - 1] > 0) return false;
    const float top = value_at(q0);
    // (no weight below -2^8, or none is there)
    if (sh.counts[2 * kSide - 1] > 0 && !((double(top) + 0x1p8) * row.scale >= double(kBins))) return false;
    const double scale = row.scale;
    auto t_of = [&](float x) { return (double(top) - double(x)) * scale; };
    // a token's weight, to 2^-33 of it as everywhere
    auto weight_at = [&](double t) -> double {
        const bool some = t >= 0.0 && t < double(kBins);  // (values above the largest logit are asked for too)
        const double held = some ? t : 0.0, f = __builtin_amdgcn_fract(held);
        const double w = sh.bin_weight(int(held)) * ((0x1p33 - double(miss_at(f))) * 0x1p-33);
        return some ? w : 0.0;
    };
    auto mass_of = [&](float x, int n) { return double(n) * weight_at(t_of(x)); };
    double spread = 0.0;  // weights times t
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        double mass = 0.0;
        int tokens = 0;
        if (__ballot((own[i][0] | own[i][1]) > 0) != 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const double t = t_of(value_at((i * kWaves + wave) * kBlock + 64 * h + lane));
                const double m = double(own[i][h]) * weight_at(t);
                mass += m;
                spread += m > 0.0 ? m * t : 0.0;
            }
            mass = wave_up_to(mass);
            tokens = wave_up_to(own[i][0] + own[i][1]);
        }
        if (lane == 63) {
            sh.block_mass[i * kWaves + wave] = __builtin_bit_cast(uint64_t, mass);
            sh.block_tokens[i * kWaves + wave] = tokens;
        }
    }
    __syncthreads();
    // up to the end of the lane's block, and of the one before (the tiny ones lie before the lower half)
    const double tiny_mass = tiny ? scalar(mass_of(0.0f, tiny)) : 0.0;
    const int block_tokens = sh.block_tokens[lane];
    const double block_mass = __builtin_bit_cast(double, sh.block_mass[lane]);
    const int tokens_end = wave_up_to(block_tokens) + (lane >= 32 ? tiny : 0);
    const double mass_end = wave_up_to(block_mass) + (lane >= 32 ? tiny_mass : 0.0);
    const int tokens_start = tokens_end - block_tokens;
    const double mass_before = __shfl_up(mass_end, 1);  // (by all lanes: the second one's comes from the first)
    const double mass_start = lane == 0 ? 0.0 : mass_before + (lane == 32 ? tiny_mass : 0.0);
    const int all_tokens = lane_of(tokens_end, 63);
    const double all_mass = lane_of(mass_end, 63);
    // (what the tiny ones weigh may be off by 2^-24 of it)
    if (tiny_mass > all_mass / 512) return false;
    ValuePrefix kept{kRanked, 0, all_tokens, all_mass};
    double M = 0.0, weight = 0.0, second = 0.0;
    int drawn = 0, place = 0, drawn_tokens = 0;
    int cut_q = kRanked;  // min_p: the first value that is not kept
    if (p.min_p > 0.0f && p.min_p <= 1.0f) {
        const double T_ = p.temperature == 0.0f ? 1.0 : double(p.temperature), low = log(double(p.min_p));
        // (those that are kept come first: blocks by their last value, then values)
        auto keeps = [&](int q) { return __builtin_popcountll(__ballot((double(value_at(q)) - double(top)) / T_ >= low)); };
        const int blocks = keeps(kBlock * lane + kBlock - 1);
        if (blocks < 64) cut_q = kBlock * blocks + keeps(kBlock * blocks + lane) + keeps(kBlock * blocks + 64 + lane);
        if (cut_q == kValues && tiny > 0) return false;
    }
    enum Stage { kTopK, kTopP, kMinP, kDraw, kSecond, kStages };
#pragma unroll 1
    for (int stage = kTopK; stage < kStages; ++stage) {
        // the place: the first token up to which there are `reach` tokens or values, at least `reach` of weight, or more
        By by = By::kCount;
        double reach = 0.0;
        if (stage == kTopK) {
            if (p.top_k == 0 || p.top_k >= all_tokens) continue;
            reach = double(p.top_k);
        } else if (stage == kTopP || stage == kDraw) {
            if (stage == kTopP && !(p.top_p < 1.0f)) continue;
            M = scalar(kept.mass + (kept.tokens ? mass_of(value_at(kept.q), kept.tokens) : 0.0));
            if (stage == kTopP) {
                reach = scalar(double(p.top_p) * M);
                if (!(reach > 0.0)) {
                    kept = ValuePrefix{q0, 1, 0, 0.0};
                    continue;
                }
                by = By::kReach;
            } else {
                if (p.temperature == 0.0f) {
                    drawn = q0;
                    place = 1;
                    drawn_tokens = scalar(count_at(sh, q0));
                    weight = 1.0;
                    continue;
                }
                if (p.u >= 1.0f) {
                    // the last that is kept and has any weight, by its number: sums may not tell it from those before. Values with
                    // a weight come first: whole blocks of them, then some of a block
                    auto weighs = [&](int q) { return t_of(value_at(q)) < double(kBins); };
                    const int blocks = __builtin_popcountll(__ballot(weighs(kBlock * lane + kBlock - 1)));
                    int tokens = all_tokens;
                    if (blocks < 64) {
                        const int q = kBlock * blocks + lane;
                        const int more = wave_up_to((weighs(q) ? count_at(sh, q) : 0) + (weighs(q + 64) ? count_at(sh, q + 64) : 0));
                        tokens = lane_of(tokens_start, blocks) + lane_of(more, 63);
                    }
                    reach = double(min(tokens, kept.before + kept.tokens));
                } else {
                    reach = scalar(p.u > 0.0f ? double(p.u) * M : 0.0);
                    by = By::kAbove;
                }
            }
        } else if (stage == kMinP) {
            if (!(p.min_p > 0.0f)) continue;
            if (p.min_p > 1.0f) {
                kept = ValuePrefix{q0, 1, 0, 0.0};
                continue;
            }
            if (cut_q > kept.q) continue;
            by = By::kCut;
            reach = double(cut_q);
        } else {
            if (a.confidence != SANGAM_CONFIDENCE_MARGIN || kept.before + kept.tokens < 2) continue;
            reach = 2.0;
        }
    again:
        auto met = [&](double end) { return by == By::kAbove ? end > reach : end >= reach; };
        // the block: the first that has tokens, or weight, and ends at the place or behind it (or, as sums are rounded, the last with
        // any; rounded sums of nothing may grow as well, so that what has no weight is no place by weight)
        const bool by_mass = by == By::kReach || by == By::kAbove;
        const bool some = by == By::kCut || (by_mass ? block_mass > 0.0 : block_tokens > 0);
        const double block_end = by == By::kCount ? double(tokens_end) : by == By::kCut ? double(kBlock * lane + kBlock) : mass_end;
        const uint64_t in = __ballot(some && met(block_end)), any = __ballot(some);
        if (in == 0 && tiny > 0) return false;
        const int at = in ? __builtin_ctzll(in) : 63 - __builtin_clzll(any);
        const double block_start = by == By::kCount ? double(tokens_start) : by == By::kCut ? double(kBlock * lane) : mass_start;
        if (tiny > 0 && at >= 32 && __ballot(lane == at && met(block_start)) != 0) return false;  // among the tiny ones
        // then the value
        const int q = kBlock * at + lane, n0 = count_at(sh, q), n1 = count_at(sh, q + 64);
        const double m0 = mass_of(value_at(q), n0), m1 = mass_of(value_at(q + 64), n1);
        const int n_end0 = lane_of(tokens_start, at) + wave_up_to(n0), n_end1 = lane_of(n_end0, 63) + wave_up_to(n1);
        const double m_end0 = lane_of(mass_start, at) + wave_up_to(m0), m_end1 = lane_of(m_end0, 63) + wave_up_to(m1);
        const double end0 = by == By::kCount ? double(n_end0) : by == By::kCut ? double(q + 1) : m_end0;
        const double end1 = by == By::kCount ? double(n_end1) : by == By::kCut ? double(q + 65) : m_end1;
        const bool none = by == By::kCut;
        const uint64_t in0 = __ballot((none || (by_mass ? m0 > 0.0 : n0 > 0)) && met(end0)), in1 = __ballot((none || (by_mass ? m1 > 0.0 : n1 > 0)) && met(end1));
        const uint64_t with0 = __ballot(m0 > 0.0), with1 = __ballot(m1 > 0.0);
        const int k = in0 ? __builtin_ctzll(in0) : in1 ? 64 + __builtin_ctzll(in1) : with1 ? 127 - __builtin_clzll(with1) : 63 - __builtin_clzll(with0 | 1);
        const int here = k < 64 ? lane_of(n0, k) : lane_of(n1, k - 64);
        ValuePrefix x{kBlock * at + k, here, k < 64 ? lane_of(n_end0 - n0, k) : lane_of(n_end1 - n1, k - 64), 0.0};
        // (what lies before: the end of the one before, the very number that was compared)
        x.mass = k == 0 ? lane_of(mass_start, at) : k <= 64 ? lane_of(m_end0, k - 1) : lane_of(m_end1, k - 65);
        if (x.q > kept.q) {  // not met within what is kept
            if (stage != kDraw) continue;
            if (by == By::kCount) return false;  // (counts are exact: the second time it is)
            by = By::kCount;  // rounded sums: the last that is kept
            reach = double(kept.before + kept.tokens);
            goto again;
        }
        const int most = x.q == kept.q ? kept.tokens : here;
        const double each = scalar(weight_at(t_of(value_at(x.q))));
        if (by == By::kCount) x.tokens = int(reach) - x.before;
        if (by == By::kReach) x.tokens = scalar(max(1, min(most, int(ceil(fmin((reach - x.mass) / each, 0x1p30))))));
        if (by == By::kAbove) x.tokens = scalar(max(1, min(most, int(floor(fmin((reach - x.mass) / each, 0x1p30))) + 1)));
        if (stage <= kMinP) {
            if (x.q < kept.q || x.tokens < kept.tokens) kept = x;
        } else if (stage == kDraw) {
            drawn = x.q;
            place = x.tokens;
            drawn_tokens = here;
            weight = each;
        } else {
            second = each;
        }
    }
    const double unit = scalar(1.0 / M);
    // the token: the place-th by index among those with its logit
    const float x = value_at(drawn);
    int token;
    if (drawn_tokens <= kList) {
        __syncthreads();
        if (tid == 0) sh.listed = 0;
        each_equal(sh, row, x, [&](int i) {
            const int k = atomicAdd(&sh.listed, 1);
            if (k < kList) sh.list[k] = uint32_t(i);
        });
        __syncthreads();
        if (tid < drawn_tokens) {
            const uint64_t mine = sh.list[tid];
            int rank = 1;
            for (int j = 0; j < drawn_tokens; ++j) rank += sh.list[j] < mine;
            if (rank == place) sh.index = int(mine);
        }
        __syncthreads();
        token = sh.index;
    } else {
        Bin<__bf16, E> bin{sh, row, -1};
        token = bin.index_of(Prefix{0, 0, place, key_of(x), 0, 0, 0});
    }
    double c = weight * unit;
    if (a.confidence == SANGAM_CONFIDENCE_MARGIN) {
        c = (1.0 - second) * unit;
    } else if (a.confidence == SANGAM_CONFIDENCE_ENTROPY) {
        double none = 0.0;
        if (kept.q < kRanked) {
            spread = 0.0;
#pragma unroll 1
            for (int q = tid; q <= kept.q; q += kThreads) {
                const double t = t_of(value_at(q)), m = double(q < kept.q ? count_at(sh, q) : kept.tokens) * weight_at(t);
                if (m > 0.0) spread += m * t;
            }
        }
        sum_all(sh, spread, none);
        if (kept.q >= kValues && tiny > 0) spread += tiny_mass * t_of(0.0f);
        c = -(spread * unit * (0.69314718055994530942 / 64) - log(unit));
    }
    answer(a, r, token, c);
    return true;
}

// ---------------------------------------------------------------- the first token, of everything

// Where nothing filters and the first token is taken, no ranks are needed: one
// look sums weights in 32 bits, eight at a time, and those sums in 64. A weight is
// 2^(c x - shift) with shift the lane's largest c x so far; c in two parts, so that
// weights are off by 2^-23 (1 + |c x - shift|) at most and by chance.
struct Whole {
    double s, st;   // weights, and weights times their exponent
    float shift;    // of both
    float best, next;
    int32_t token;  // the first with the largest logit
    int32_t fine;   // there are weights, and all are numbers
};
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eRest = float(1.4426950408889634074 - double(kLog2e));
constexpr float kLowestBest = -1e38f;

// Sums of two ranges as one.
__device__ __forceinline__ void join(double& s, double& st, float& shift, double s2, double st2, float shift2) {
    const float top = fmaxf(shift, shift2);
    const double d = double(shift) - double(top), d2 = double(shift2) - double(top), f = exp2(d), f2 = exp2(d2);
    st = f * (st + s * d) + f2 * (st2 + s2 * d2);
    s = f * s + f2 * s2;
    shift = top;
}

// The product as 32 bits hold it, wherever it is used (and not fused with what it is subtracted from).
__device__ __forceinline__ float shift_of(float best) {
    float shift = best * kLog2e;
    asm("" : "+v"(shift));
    return shift;
}
__device__ __forceinline__ float exponent_of(float x, float shift) { return __builtin_fmaf(x, kLog2eRest, __builtin_fmaf(x, kLog2e, -shift)); }

template <int KIND, typename T, int E>
__device__ __forceinline__ Whole look_once(Counts& sh, const Row<T, E>& row) {
    constexpr int V = Row<T, E>::V, kBatch = 8 / V;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    double s = 0.0, st = 0.0;
    float best = kLowestBest, next = -INFINITY, shift = shift_of(kLowestBest);
    int at = INT32_MAX;
    auto add = [&](auto& x, int n) {  // n logits, of which best takes note already
        const float to = shift_of(best);
        const float r = __builtin_amdgcn_exp2f(shift - to);
        float part = 0.0f, part_t = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e >= n) break;
            const float t = exponent_of(x[e], to), w = __builtin_amdgcn_exp2f(t);
            part += w;
            if (KIND == SANGAM_CONFIDENCE_ENTROPY) part_t += w > 0.0f ? w * t : 0.0f;
        }
        if (KIND == SANGAM_CONFIDENCE_ENTROPY) st = double(r) * (st + s * double(shift - to)) + double(part_t);
        s = double(r) * s + double(part);
        shift = to;
    };
    auto note = [&](float m, int i) {
        if (m > best) at = i;
        best = fmaxf(best, m);
    };
    row.each_chunk([&](int, int v0, const auto& w) {
#pragma unroll
        for (int j = 0; j < Row<T, E>::kLoads; j += kBatch) {
            float x[8];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int k = v0 + (j + i) * kThreads + tid;
                float y[V];
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] = -INFINITY;
                if (k < row.last) row.unpack(w[j + i], row.head + k * V, y);
                float m = y[0];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (e > 0) m = fmaxf(m, y[e]);
                    x[i * V + e] = y[e];
                }
                if (KIND == SANGAM_CONFIDENCE_MARGIN) {
                    float most = best;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        next = fmaxf(next, fminf(most, y[e]));
                        most = fmaxf(most, y[e]);
                    }
                }
                note(m, row.head + k * V);
            }
            add(x, 8);
            __builtin_amdgcn_sched_barrier(0);  // (side by side batches take all registers)
        }
    });
    row.each_edge([&](int i, float x) {
        if (KIND == SANGAM_CONFIDENCE_MARGIN) next = fmaxf(next, fminf(best, x));
        if (x == best && i < at) at = i;
        note(x, i);
        const float one[8] = {x};
        add(one, 1);
    });
    // all lanes', then all waves'
    float top = wave_max(best);
    if (lane == 0) sh.wave_top[0][wave] = top;
    __syncthreads();
    if (tid == 0) sh.first_token = INT32_MAX;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh.wave_top[0][w]);
    const int holders = __syncthreads_count(best == top);
    const float mine = wave_max(best == top && holders == 1 ? next : best);
    if (best == top && at < row.vocab)
        for (int e = 0; e < V && at + e < row.vocab; ++e)
            if (row.at(at + e) == top) {
                atomicMin(&sh.first_token, at + e);
                break;
            }
    const float to = shift_of(top);
    const double d = double(shift) - double(to), f = exp2(d);
    st = f * (st + s * d);
    s = f * s;
#pragma unroll
    for (int k = 32; k > 0; k /= 2) {
        s += __shfl_xor(s, k);
        st += __shfl_xor(st, k);
    }
    if (lane == 0) {
        sh.wave_top[1][wave] = mine;
        sh.wave_sums[wave] = s;
        sh.wave_sums[kWaves + wave] = st;
    }
    __syncthreads();
    Whole all{0.0, 0.0, to, top, -INFINITY, sh.first_token, 0};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        all.s += sh.wave_sums[w];
        all.st += sh.wave_sums[kWaves + w];
        all.next = fmaxf(all.next, sh.wave_top[1][w]);
    }
    all.fine = all.s > 0.0 && all.s < 1e30 && top > kLowestBest && all.token < row.vocab;  // (no number fails)
    return all;
}

template <typename T, int E>
__device__ __forceinline__ Whole look_once(Counts& sh, const Row<T, E>& row, int kind) {
    return kind == SANGAM_CONFIDENCE_ENTROPY  ? look_once<SANGAM_CONFIDENCE_ENTROPY>(sh, row)
           : kind == SANGAM_CONFIDENCE_MARGIN ? look_once<SANGAM_CONFIDENCE_MARGIN>(sh, row)
                                              : look_once<SANGAM_CONFIDENCE_PROBABILITY>(sh, row);
}

__device__ __forceinline__ void answer(const SampleArgs& a, int64_t r, const Whole& all) {
    double c = exp2(double(exponent_of(all.best, all.shift))) / all.s;
    if (a.confidence == SANGAM_CONFIDENCE_MARGIN) c -= exp2(double(exponent_of(all.next, all.shift))) / all.s;
    if (a.confidence == SANGAM_CONFIDENCE_ENTROPY) c = 0.69314718055994530942 * (all.st / all.s) - log(all.s);
    answer(a, r, all.token, c);
}

template <typename T, int E>
__device__ __forceinline__ Row<T, E> row_of(const SampleArgs& a, int64_t r, const Params& p) {
    Row<T, E> row;
    row.p = static_cast<const T*>(a.logits) + r * a.row_stride;
    row.vocab = a.vocab;
    row.forbid = a.forbid;
    row.infinite = row.wide = false;
    row.head = min(int((16 - (reinterpret_cast<uintptr_t>(row.p) & 15)) & 15) / int(sizeof(T)), a.vocab);
    row.vectors = (a.vocab - row.head) / row.V;
    row.first = 0;
    row.last = row.vectors;
    row.top = 0.0;
    row.base = 0;
    row.scale = scalar(64.0 * 1.4426950408889634074 / (p.temperature == 0.0f ? 1.0 : double(p.temperature)));
    return row;
}

// A row's answer from its logits alone, whatever they are.
template <typename T, int E>
__device__ __forceinline__ void from_logits(Shared<E>& sh, Row<T, E>& row, const SampleArgs& a, const Params& p, int64_t r) {
    float top;
    if (fill(sh, row, top, sh.tops) != kFilled && !fill_wide(sh, row, top)) {
        answer(a, r, -1, 0.0);
        return;
    }
    choose(sh, row, a, p, r, top);
}

template <int E>
__device__ __forceinline__ void start(Shared<E>& sh) {
    if (threadIdx.x < 64) sh.powers[threadIdx.x] = exp2(threadIdx.x * (-1.0 / 64));
}

constexpr int kPending = -2;  // the token of a row that the launch before did not tell

// A work-group takes a row of bf16. (What sample_kernel takes more registers for
// is left to it: three work-groups fit a CU.)
__global__ __launch_bounds__(kThreads, 6) void sample_values_kernel(SampleArgs a) {
    constexpr int E = kWhole<__bf16>;
    __shared__ Shared<E> sh;
    const int64_t r = blockIdx.x;
    const Params p = params_of(a, r);
    if (p.none) {
        answer(a, r, -1, 0.0);
        return;
    }
    Row<__bf16, E> row = row_of<__bf16, E>(a, r, p);
    start(sh);
    for (int k = threadIdx.x; k < 2 * kSide; k += kThreads) sh.counts[k] = 0;
    __syncthreads();
    count(sh, row, sh.tops);
    __syncthreads();
    uncount(sh, row);
    __syncthreads();
    if (!choose_by_value(sh, row, a, p, r)) answer(a, r, kPending, 0.0);
}

// A work-group takes a row of which the first token is wanted, of everything.
template <typename T, int KIND>
__global__ __launch_bounds__(kThreads) void sample_whole_kernel(SampleArgs a) {
    __shared__ Counts sh;
    const int64_t r = blockIdx.x;
    const Params p = params_of(a, r);
    if (p.none) {
        answer(a, r, -1, 0.0);
        return;
    }
    if (p.whole()) {
        const Whole all = look_once<KIND>(sh, row_of<T, kWhole<T>>(a, r, p));
        if (all.fine) {
            answer(a, r, all);
            return;
        }
    }
    answer(a, r, kPending, 0.0);
}

// A work-group takes a row, or its row if it is pending.
template <typename T, bool PENDING>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
    constexpr int E = kWhole<T>;
    __shared__ Shared<E> sh;
    const int64_t r = blockIdx.x;
    if (PENDING && a.tokens[r] != kPending) return;
    const Params p = params_of(a, r);
    if (p.none) {
        answer(a, r, -1, 0.0);
        return;
    }
    Row<T, E> row = row_of<T, E>(a, r, p);
    start(sh);
    __syncthreads();  // (and all waves have looked before the row gets its token)
    from_logits(sh, row, a, p, r);
}

// The kernels of a type.
template <typename T>
const void* whole_kernel(int kind) {
    return kind == SANGAM_CONFIDENCE_ENTROPY  ? reinterpret_cast<const void*>(&sample_whole_kernel<T, SANGAM_CONFIDENCE_ENTROPY>)
           : kind == SANGAM_CONFIDENCE_MARGIN ? reinterpret_cast<const void*>(&sample_whole_kernel<T, SANGAM_CONFIDENCE_MARGIN>)
                                              : reinterpret_cast<const void*>(&sample_whole_kernel<T, SANGAM_CONFIDENCE_PROBABILITY>);
}
template <typename T>
const void* row_kernel(bool pending) {
    if (__is_same(T, __bf16) || pending) return reinterpret_cast<const void*>(&sample_kernel<T, true>);
    return reinterpret_cast<const void*>(&sample_kernel<T, __is_same(T, __bf16)>);
}

// Few rows are cut into parts, of some chunks each: a work-group counts a part, and
// another puts the parts of a row together and goes on from there.
struct Split {
    int parts, chunks_each, chunks;
    int64_t record, row_bytes;  // of a part, of a row's parts and tops
    uint8_t* workspace;
};

struct PartHead {
    float top;
    int32_t base, filled;
};
constexpr int kRecordValues = (2 * kSide * int(sizeof(uint16_t)) + 255) / 256 * 256;
constexpr int kRecordBins = kBins * int(sizeof(uint64_t)) + 256;
constexpr int kMostChunks = 65535 / (kThreads * kPart);  // of a part: counts fit 16 bits

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_part_kernel(SampleArgs a, Split s) {
    __shared__ Counts sh;
    const int64_t r = blockIdx.x / s.parts;
    const int part = blockIdx.x % s.parts;
    const Params p = params_of(a, r);
    if (p.none) return;
    Row<T, kPart> row = row_of<T, kPart>(a, r, p);
    row.first = min(part * s.chunks_each * row.kChunk, row.vectors);
    row.last = min(row.first + s.chunks_each * row.kChunk, row.vectors);
    uint8_t* const at = s.workspace + r * s.row_bytes;
    uint16_t* const tops = reinterpret_cast<uint16_t*>(at + s.parts * s.record);
    uint8_t* const record = at + part * s.record;
    if constexpr (__is_same(T, __bf16)) {
        for (int k = threadIdx.x; k < 2 * kSide; k += kThreads) sh.counts[k] = 0;
        __syncthreads();
        count(sh, row, tops);
        __syncthreads();
        for (int k = threadIdx.x; k < kSide; k += kThreads)
            reinterpret_cast<uint32_t*>(record)[k] = sh.counts[2 * k] | (sh.counts[2 * k + 1] << 16);
    } else if (p.whole()) {
        const Whole all = look_once(sh, row, a.confidence);
        if (threadIdx.x == 0) *reinterpret_cast<Whole*>(record) = all;
    } else {
        float top;
        const Filled filled = fill(sh, row, top, tops);
        for (int k = threadIdx.x; k < kBins; k += kThreads) reinterpret_cast<uint64_t*>(record)[k] = sh.bins[k];
        if (threadIdx.x == 0) *reinterpret_cast<PartHead*>(record + kBins * sizeof(uint64_t)) = PartHead{top, row.base, filled};
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_join_kernel(SampleArgs a, Split s) {
    __shared__ Shared<kPart> sh;
    const int64_t r = blockIdx.x;
    const Params p = params_of(a, r);
    if (p.none) {
        answer(a, r, -1, 0.0);
        return;
    }
    Row<T, kPart> row = row_of<T, kPart>(a, r, p);
    start(sh);
    const uint8_t* const at = s.workspace + r * s.row_bytes;
    typedef uint32_t U4 __attribute__((ext_vector_type(4)));
    const U4* const tops = reinterpret_cast<const U4*>(at + s.parts * s.record);
    constexpr int kTopPieces = Shared<kPart>::kTops / 8 / kThreads;
#pragma unroll
    for (int j = 0; j < kTopPieces; ++j)
        if (int(threadIdx.x) + j * kThreads < s.chunks * kThreads / 8)
            reinterpret_cast<U4*>(sh.tops)[int(threadIdx.x) + j * kThreads] = tops[int(threadIdx.x) + j * kThreads];
    if constexpr (__is_same(T, __bf16)) {
        // eight counts at a time, of all the parts
        constexpr int kPieces = kRecordValues / 16, kMine = (kPieces + kThreads - 1) / kThreads;
        constexpr int kAtOnce = 5;
        uint32_t sums[kMine][8] = {};
#pragma unroll 1
        for (int part0 = 0; part0 < s.parts; part0 += kAtOnce) {
            U4 w[kAtOnce][kMine];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                for (int j = 0; j < kMine; ++j)
                    if (part0 + i < s.parts && int(threadIdx.x) + j * kThreads < kPieces)
                        w[i][j] = reinterpret_cast<const U4*>(at + (part0 + i) * s.record)[int(threadIdx.x) + j * kThreads];
                    else w[i][j] = U4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                for (int j = 0; j < kMine; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sums[j][2 * e] += w[i][j][e] & 0xFFFFu;
                        sums[j][2 * e + 1] += w[i][j][e] >> 16;
                    }
        }
#pragma unroll
        for (int j = 0; j < kMine; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = (int(threadIdx.x) + j * kThreads) * 8 + e;
                if (k < 2 * kSide) sh.counts[k] = sums[j][e];
            }
        __syncthreads();
        uncount(sh, row);
        __syncthreads();
        if (choose_by_value(sh, row, a, p, r)) return;
    } else if (p.whole()) {
        Whole all{0.0, 0.0, shift_of(kLowestBest), -INFINITY, -INFINITY, INT32_MAX, 1};
        for (int part = 0; part < s.parts; ++part) {
            const Whole w = *reinterpret_cast<const Whole*>(at + part * s.record);
            // (a part without weight has no say; one with what is no number is not summed up)
            if (!w.fine && w.s == 0.0 && w.best == kLowestBest) continue;
            all.fine = all.fine && w.fine;
            join(all.s, all.st, all.shift, w.s, w.st, w.shift);
            all.next = fmaxf(fmaxf(all.next, w.next), fminf(all.best, w.best));
            if (w.best > all.best) all.token = w.token;  // (parts come in order)
            if (w.best == all.best) all.token = min(all.token, w.token);
            all.best = fmaxf(all.best, w.best);
        }
        if (all.fine && all.s > 0.0) {
            answer(a, r, all);
            return;
        }
    } else {
        float top = -INFINITY;
        bool far = false, any = false;
        for (int part = 0; part < s.parts; ++part) {
            const PartHead h = *reinterpret_cast<const PartHead*>(at + part * s.record + kBins * sizeof(uint64_t));
            far = far || h.filled == kFar;
            if (h.filled == kFilled && h.top > top) {
                any = true;
                top = h.top;
                row.base = h.base;
            }
        }
        if (any && !far) {
            uint64_t sums[kEach] = {};
#pragma unroll 2
            for (int part = 0; part < s.parts; ++part) {
                const uint8_t* const record = at + part * s.record;
                const PartHead h = *reinterpret_cast<const PartHead*>(record + kBins * sizeof(uint64_t));
                uint64_t w[kEach];
#pragma unroll
                for (int j = 0; j < kEach; ++j) w[j] = reinterpret_cast<const uint64_t*>(record)[threadIdx.x + j * kThreads];
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    // (the bin whose slot k is; the part's slot may hold the bin a circle on)
                    const int k = int(threadIdx.x) + j * kThreads, b = row.base + ((k - row.base) & (kBins - 1));
                    if (h.filled == kFilled && b >= h.base) sums[j] += w[j];
                }
            }
#pragma unroll
            for (int j = 0; j < kEach; ++j) sh.bins[threadIdx.x + j * kThreads] = sums[j];
            __syncthreads();
            choose(sh, row, a, p, r, top);
            return;
        }
    }
    __syncthreads();
    from_logits(sh, row, a, p, r);
}

// Rows from which a work-group takes a whole one, for all types. Whole / in parts, us, greedy, then under a nucleus:
//                   256 rows                  384 rows                  640 rows
//   bf16,  50,257   19.6 / 23.8, 22.3 / 26.8  25.8 / 31.0, 29.9 / 35.7  33.6 / 48.3, 39.0 / 54.8
//   bf16, 126,464   34.2 / 32.9, 42.7 / 39.9  40.5 / 47.3, 50.9 / 56.1  50.2 / 68.9, 59.9 / 79.2
//   fp32,  50,257   22.8 / 21.7, 39.3 / 41.5  27.3 / 27.7, 47.0 / 53.2  45.0 / 45.7, 75.7 / 80.7
//   fp32, 126,464   44.3 / 35.0,  107 / 98    50.6 / 55.0,  113 / 119   90.4 / 79.1,  178 / 188
//   fp16,  50,257   15.2 / 17.7, 28.2 / 37.3  27.4 / 21.9, 39.2 / 48.1  41.6 / 34.4, 58.9 / 71.5
//   fp16, 126,464   28.2 / 25.4, 70.1 / 72.5  50.5 / 37.4, 80.7 / 93.1  75.7 / 53.1,  124 / 131
// Whole rows win, but where few of them make a round more. Greedy fp16 rows would gain by parts up to 767 rows:
// sample_whole_kernel takes 130 registers and more for them, so one work-group fits a CU and 257 rows are two rounds; of
// fp32, with 92 to 109, two fit.
constexpr int64_t kWholeRows = 256;
// Work-groups that the parts make if they can: three a CU.
constexpr int64_t kGroups = 3 * 256;
// Parts of a row at most: putting one more together takes longer than its share of the row.
constexpr int kMostParts = 10;

Split split_of(int64_t rows, int32_t vocab, int32_t dtype) {
    Split s{};
    constexpr int chunk = kThreads * kPart;
    s.chunks = (vocab + chunk - 1) / chunk;
    if (rows < 1 || rows >= kWholeRows) {
        s.parts = 1;
        return s;
    }
    const int64_t wanted = std::max<int64_t>((kGroups + rows - 1) / rows, (s.chunks + kMostChunks - 1) / kMostChunks);
    const int parts = int(std::min<int64_t>({wanted, s.chunks, std::max<int64_t>(kMostParts, (s.chunks + kMostChunks - 1) / kMostChunks)}));
    s.chunks_each = (s.chunks + parts - 1) / parts;
    s.parts = (s.chunks + s.chunks_each - 1) / s.chunks_each;
    s.record = dtype == SANGAM_DTYPE_BF16 ? kRecordValues : kRecordBins;
    s.row_bytes = s.parts * s.record + int64_t(s.chunks) * kThreads * int64_t(sizeof(uint16_t));
    return s;
}

sangam_status fail(sangam_status code, const std::string& msg) {
    set_error(msg);
    return code;
}

sangam_status sample(const sangam_sample_desc* d, int32_t* tokens, float* confidence, void* workspace, size_t workspace_bytes, void* stream) {
    clear_error();
    if (!d) return fail(SANGAM_ERR_INVALID_ARG, "desc must not be NULL");
    if (d->dtype != SANGAM_DTYPE_BF16 && d->dtype != SANGAM_DTYPE_FP16 && d->dtype != SANGAM_DTYPE_FP32)
        return fail(SANGAM_ERR_UNSUPPORTED, "dtype must be SANGAM_DTYPE_BF16, _FP16 or _FP32");
    if (d->rows < 0 || d->rows > INT32_MAX || d->vocab < 1 || d->vocab > kMaxVocab)
        return fail(SANGAM_ERR_INVALID_ARG, "rows must be 0 to 2^31 - 1 and vocab 1 to 2^18");
    if (d->confidence < SANGAM_CONFIDENCE_PROBABILITY || d->confidence > SANGAM_CONFIDENCE_ENTROPY)
        return fail(SANGAM_ERR_INVALID_ARG, "confidence must be SANGAM_CONFIDENCE_PROBABILITY, _MARGIN or _ENTROPY");
    if (d->forbid < -1 || d->forbid >= d->vocab) return fail(SANGAM_ERR_INVALID_ARG, "forbid must be -1 or a token");
    // (comparisons that a NaN fails)
    if (!d->temperatures && !(d->temperature >= 0.0f)) return fail(SANGAM_ERR_INVALID_ARG, "temperature must not be negative");
    if (!d->top_ks && d->top_k < 0) return fail(SANGAM_ERR_INVALID_ARG, "top_k must not be negative");
    if (!d->top_ps && !(d->top_p >= 0.0f && d->top_p <= 1.0f)) return fail(SANGAM_ERR_INVALID_ARG, "top_p must be 0 to 1");
    if (!d->min_ps && !(d->min_p >= 0.0f && d->min_p <= 1.0f)) return fail(SANGAM_ERR_INVALID_ARG, "min_p must be 0 to 1");
    const bool arrays = d->temperatures || d->top_ks || d->top_ps || d->min_ps;
    if (d->num_params < 0 || (arrays && !d->params_of && d->num_params < d->rows))
        return fail(SANGAM_ERR_INVALID_ARG, "arrays of parameters must have an entry for every row, or params_of");
    if (d->rows == 0) return SANGAM_OK;
    if (!d->logits || !d->u || !tokens) return fail(SANGAM_ERR_INVALID_ARG, "logits, u and tokens must not be NULL");
    if (d->row_stride < 0 || d->row_stride > (int64_t(1) << 40)) return fail(SANGAM_ERR_INVALID_ARG, "row_stride must be 0 to 2^40");
    const size_t size = d->dtype == SANGAM_DTYPE_FP32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(d->logits) % size) return fail(SANGAM_ERR_ALIGN, "logits must be aligned to their elements");
    for (const void* p : {static_cast<const void*>(d->u), static_cast<const void*>(d->params_of), static_cast<const void*>(d->temperatures),
                          static_cast<const void*>(d->top_ks), static_cast<const void*>(d->top_ps), static_cast<const void*>(d->min_ps),
                          static_cast<const void*>(tokens), static_cast<const void*>(confidence)})
        if (reinterpret_cast<uintptr_t>(p) % 4) return fail(SANGAM_ERR_ALIGN, "the arrays must be 4-byte aligned");
    const size_t need = sangam_sample_workspace_bytes(d->rows, d->vocab, d->dtype);
    if (need > 0 && (!workspace || workspace_bytes < need)) return fail(SANGAM_ERR_BUFFER, "workspace is too small");
    if (need > 0 && reinterpret_cast<uintptr_t>(workspace) % 256) return fail(SANGAM_ERR_ALIGN, "workspace must be 256-byte aligned");
    SampleArgs args{d->logits, d->row_stride, d->u, d->params_of, d->num_params, d->temperatures, d->top_ks, d->top_ps, d->min_ps,
                    d->temperature, d->top_k, d->top_p, d->min_p, d->vocab, d->confidence, d->forbid, tokens, confidence};
    hipStream_t const on = static_cast<hipStream_t>(stream);
    Split split = split_of(d->rows, d->vocab, d->dtype);
    split.workspace = static_cast<uint8_t*>(workspace);
    auto launch = [&](const void* fn, int64_t groups, void** kargs) {
        const hipError_t e = hipLaunchKernel(fn, dim3(unsigned(groups)), dim3(kThreads), kargs, 0, on);
        return e == hipSuccess ? SANGAM_OK : fail(SANGAM_ERR_HIP, std::string("sampling launch: ") + hipGetErrorString(e));
    };
    const bool bf16 = d->dtype == SANGAM_DTYPE_BF16, fp32 = d->dtype == SANGAM_DTYPE_FP32;
    if (split.parts > 1) {
        void* kargs[] = {&args, &split};
        const void* part = bf16   ? reinterpret_cast<const void*>(&sample_part_kernel<__bf16>)
                           : fp32 ? reinterpret_cast<const void*>(&sample_part_kernel<float>)
                                  : reinterpret_cast<const void*>(&sample_part_kernel<_Float16>);
        const void* join = bf16   ? reinterpret_cast<const void*>(&sample_join_kernel<__bf16>)
                           : fp32 ? reinterpret_cast<const void*>(&sample_join_kernel<float>)
                                  : reinterpret_cast<const void*>(&sample_join_kernel<_Float16>);
        if (const sangam_status e = launch(part, d->rows * split.parts, kargs)) return e;
        return launch(join, d->rows, kargs);
    }
    const bool maybe_whole = d->temperatures || d->temperature == 0.0f;  // rows whose first token of everything is wanted
    // a grid's threads are counted in 32 bits
    const int64_t step = (int64_t(1) << 32) / kThreads - 1;
    for (int64_t row = 0; row < d->rows; row += step) {
        SampleArgs some = args;
        some.logits = static_cast<const uint8_t*>(d->logits) + row * d->row_stride * int64_t(size);
        some.u += row;
        if (some.params_of) {
            some.params_of += row;
        } else if (arrays) {
            some.num_params -= row;
            for (const float** x : {&some.temperatures, &some.top_ps, &some.min_ps})
                if (*x) *x += row;
            if (some.top_ks) some.top_ks += row;
        }
        some.tokens += row;
        if (some.conf) some.conf += row;
        const int64_t rows = std::min(step, d->rows - row);
        void* kargs[] = {&some};
        const bool pending = bf16 || maybe_whole;
        if (pending)
            if (const sangam_status e = launch(bf16   ? reinterpret_cast<const void*>(&sample_values_kernel)
                                               : fp32 ? whole_kernel<float>(d->confidence)
                                                      : whole_kernel<_Float16>(d->confidence), rows, kargs))
                return e;
        const void* fn = bf16 ? row_kernel<__bf16>(pending) : fp32 ? row_kernel<float>(pending) : row_kernel<_Float16>(pending);
        if (const sangam_status e = launch(fn, rows, kargs)) return e;
    }
    return SANGAM_OK;
}

}  // namespace

extern "C" size_t sangam_sample_workspace_bytes(int64_t rows, int32_t vocab, int32_t dtype) {
    const bool known = dtype == SANGAM_DTYPE_BF16 || dtype == SANGAM_DTYPE_FP16 || dtype == SANGAM_DTYPE_FP32;
    if (!known || rows < 1 || rows > INT32_MAX || vocab < 1 || vocab > kMaxVocab) return 0;
    const Split s = split_of(rows, vocab, dtype);
    return s.parts > 1 ? size_t(rows * s.row_bytes) : 0;
}

extern "C" sangam_status sangam_sample_tokens(const sangam_sample_desc* desc, int32_t* tokens, float* confidence, void* workspace,
                                              size_t workspace_bytes, void* stream) {
    return entry([&] { return sample(desc, tokens, confidence, workspace, workspace_bytes, stream); });
}
