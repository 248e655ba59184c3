// A token and a confidence for every row of logits, for gfx950, with its C ABI
// entry point (include/sangam_sample.h).
//
// All filters and the draw are places on one axis, the ranks: a prefix of them
// is kept, and the draw falls at a share u of the prefix's weight. What is
// needed of a row is therefore how many tokens and how much weight lie above a
// logit. With t = 64 log2(e) (X - x) / T, a token weighs 2^(-t / 64); bin b
// holds those with floor(t) = b, as a count and the sum of what their weights
// miss of the bin's largest, y = 1 - 2^(-frac(t) / 64) in whole steps of 2^-33.
// Whole numbers, so the order of LDS atomics changes nothing, and 4096 bins
// reach down to 2^-64 of the largest weight. A place inside a bin is found among
// the bin's own tokens, which a further look at the row collects: sorted in LDS
// where they fit (some hundred at most in a row of a language model's logits),
// else by digits of their logits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "../../include/sangam_sample.h"
#include "entry.h"

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
constexpr int kList = 1024;              // tokens of a bin that are sorted
constexpr int kDigits = 2048;
constexpr int kMaxVocab = 1 << 18;
constexpr int kGroups = kMaxVocab / 4 / 64;  // of 64 vectors of 16 bytes
constexpr int kLoads = 4;                    // vectors of a thread on their way together

// A bin or digit: tokens, and what their weights miss, in units of 2^-33 of the
// bin's largest weight. 2^18 tokens miss under 2^44.5 of them.
constexpr int kMissBits = 45;
constexpr uint64_t kOne = uint64_t(1) << 33;
__device__ __forceinline__ int tokens_in(uint64_t bin) { return int(bin >> kMissBits); }
__device__ __forceinline__ uint64_t weight_in(uint64_t bin) {  // in units of 2^-33
    return (bin >> kMissBits) * kOne - (bin & ((uint64_t(1) << kMissBits) - 1));
}
__device__ __forceinline__ double bin_weight(int b) { return exp2(b * (-1.0 / 64)); }
// Units of 2^-33 of a bin's largest weight as units of 2^-44 of the row's.
__device__ __forceinline__ uint64_t mass_of(int b, uint64_t v) { return uint64_t(__builtin_rint(bin_weight(b) * double(v) * 2048.0)); }
// And back.
__device__ __forceinline__ double inside(int b, double mass) { return mass / (bin_weight(b) * 2048.0); }

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

struct Shared {
    uint64_t bins[kBins];
    union {
        struct {
            uint64_t list[kList];    // key and index; then the weight up to each
            uint64_t sorted[kList];
        };
        uint64_t digits[kDigits];
    };
    float tops[kGroups];  // the largest logit of a group of vectors
    uint64_t part[2 * kWaves];
    double sums[kWaves];
    uint64_t found_mass, found_bin;
    int found, found_tokens, found_last, listed;
    int32_t index;
};

// Keys of 32 bits in rank order: the larger the logit, the smaller the key.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);  // -0 equals 0
    return (b >> 31) ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float((key >> 31) ? key : ~key & 0x7FFFFFFFu); }

template <typename T>
struct Row {
    static constexpr int V = 16 / int(sizeof(T));
    const T* p;
    int vocab, forbid;
    int head, vectors, groups;  // elements before the first aligned vector; vectors; groups of 64 of them
    bool infinite;              // some logit is +inf: those count as 0, all others as -inf
    double top, scale;          // t = (top - x) scale

    __device__ float adjusted(float x, int i) const {
        if (i == forbid) x = -INFINITY;
        if (infinite) x = x == INFINITY ? 0.0f : -INFINITY;
        return x;
    }
    __device__ float at(int i) const { return adjusted(float(p[i]), i); }
    __device__ double t_of(float x) const { return (top - double(x)) * scale; }
    // vectors of the groups that want() asks for: f(group, first index, logits)
    template <typename Want, typename F>
    __device__ __forceinline__ void each_vector(Want want, F f) const {
        typedef T Vec __attribute__((ext_vector_type(V)));
        const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
        const Vec* const v = reinterpret_cast<const Vec*>(p + head);
        for (int g0 = wave; g0 < groups; g0 += kWaves * kLoads) {
            Vec w[kLoads];
            bool have[kLoads];
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int g = g0 + j * kWaves;
                have[j] = g < groups && want(g);
                if (have[j] && 64 * g + lane < vectors) w[j] = v[64 * g + lane];
            }
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int g = g0 + j * kWaves;
                if (!have[j]) continue;
                float x[V];
                const int i0 = head + (64 * g + lane) * V;
                if (64 * g + lane < vectors) {
#pragma unroll
                    for (int e = 0; e < V; ++e) x[e] = float(w[j][e]);
                    if (unsigned(forbid - i0) < unsigned(V)) {
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            if (i0 + e == forbid) x[e] = -INFINITY;
                    }
                    if (infinite) {
#pragma unroll
                        for (int e = 0; e < V; ++e) x[e] = x[e] == INFINITY ? 0.0f : -INFINITY;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) x[e] = -INFINITY;
                }
                f(g, i0, x);
            }
        }
    }
    // the elements outside all vectors
    template <typename F>
    __device__ __forceinline__ void each_edge(F f) const {
        const int rest = vocab - vectors * V;
        for (int k = threadIdx.x; k < rest; k += kThreads) {
            const int i = k < head ? k : k + vectors * V;
            f(i, at(i));
        }
    }
    // all logits with t under `limit`, and some of the others
    template <typename F>
    __device__ __forceinline__ void each_under(const float* tops, double limit, F f) const {
        each_vector([&](int g) { return !(t_of(tops[g]) >= limit); },
                    [&](int, int i0, const float(&x)[V]) {
#pragma unroll
                        for (int e = 0; e < V; ++e) f(i0 + e, x[e]);
                    });
        each_edge(f);
    }
};

// What the weight at a fraction f of a bin misses, in units of 2^-33: the low word
// of 2^52 + 2^33 (1 - 2^(-f / 64)). (Cubic without constant, fitted over [0, 1);
// off by 5.3e-12 = 0.05 units.)
__device__ __forceinline__ uint32_t miss_at(double f) {
    constexpr double q1 = 0x1.62e42fb615b67p-7 * 0x1p33, q2 = -0x1.ebfa827a93283p-15 * 0x1p33, q3 = 0x1.c454fdc63ddabp-23 * 0x1p33;
    return uint32_t(__double2loint(__builtin_fma(f, __builtin_fma(f, __builtin_fma(f, q3, q2), q1), 0x1p52)));
}

__device__ __forceinline__ uint64_t wave_up_to(uint64_t x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// Sum over the threads before this one, and over all.
__device__ uint64_t sum_before(Shared& sh, uint64_t x, uint64_t* total) {
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
    *total = all;
    return before + up_to - x;
}

__device__ double sum_all(Shared& sh, double x) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.sums[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += sh.sums[w];
    return x;
}

// A prefix of the ranks: all tokens of the bins before `bin`, and the first
// `tokens` of that bin, which end with `ties` tokens of key `key`.
struct Prefix {
    int bin, tokens, ties;
    uint32_t key;
    uint64_t weight;     // of those of the bin, units of 2^-33 of its largest
    uint64_t mass;       // of the bins before, units of 2^-44
    int before;          // tokens of the bins before
    __device__ uint64_t all() const { return mass + (tokens ? mass_of(bin, weight) : 0); }
};

// A token inside a bin: the place-th of those with its key, behind `before` tokens of the bin.
struct Token {
    uint32_t key;
    int place, before, index;
    uint64_t weight_before;  // of the bin's tokens before those of its key
    int equal;               // tokens with its key
};

enum class By { kCount, kReach, kAbove };

template <typename T>
struct Bin {
    Shared& sh;
    const Row<T>& row;
    int& listed;  // bin whose tokens sh.sorted and sh.list hold

    __device__ uint64_t weight_of(uint32_t key, int b) const { return kOne - miss_at(row.t_of(logit_of(key)) - b); }

    // Tokens of bin b, in rank order, and their weights summed up.
    __device__ void collect(int b, int n) {
        if (listed == b) return;
        __syncthreads();
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        row.each_under(sh.tops, double(b + 1), [&](int i, float x) {
            const double t = row.t_of(x);
            if (t >= double(b) && t < double(b + 1)) {
                const int k = atomicAdd(&sh.listed, 1);
                if (k < kList) sh.list[k] = (uint64_t(key_of(x)) << 32) | uint32_t(i);
            }
        });
        __syncthreads();
        for (int k = threadIdx.x; k < n; k += kThreads) {
            const uint64_t mine = sh.list[k];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += sh.list[j] < mine;
            sh.sorted[rank] = mine;
        }
        __syncthreads();
        static_assert(kList == 2 * kThreads, "two tokens a thread");
        const int k = 2 * threadIdx.x;
        const uint64_t w0 = k < n ? weight_of(uint32_t(sh.sorted[k] >> 32), b) : 0;
        const uint64_t w1 = k + 1 < n ? weight_of(uint32_t(sh.sorted[k + 1] >> 32), b) : 0;
        uint64_t total;
        const uint64_t before = sum_before(sh, w0 + w1, &total);
        if (k < n) sh.list[k] = before + w0;
        if (k + 1 < n) sh.list[k + 1] = before + w0 + w1;
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
        return lo;
    }

    // The key at which a count or weight is met, by digits of the keys.
    __device__ Token descend(int b, By by, int count, double weight) {
        listed = -1;
        Token k{0, 0, 0, -1, 0, 0};
        constexpr int bits[3] = {11, 11, 10}, shifts[3] = {21, 10, 0};
        for (int step = 0; step < 3; ++step) {
            const int shift = shifts[step], width = bits[step];
            __syncthreads();
            for (int d = threadIdx.x; d < kDigits; d += kThreads) sh.digits[d] = 0;
            if (threadIdx.x == 0) sh.found = sh.found_last = -1;
            __syncthreads();
            row.each_under(sh.tops, double(b + 1), [&](int, float x) {
                const double t = row.t_of(x);
                if (!(t >= double(b) && t < double(b + 1))) return;
                const uint32_t key = key_of(x);
                if ((uint64_t(key) >> (shift + width)) != (uint64_t(k.key) >> (shift + width))) return;
                atomicAdd(reinterpret_cast<unsigned long long*>(&sh.digits[(key >> shift) & ((1u << width) - 1)]),
                          (uint64_t(1) << kMissBits) | miss_at(t - b));
            });
            __syncthreads();
            uint64_t bin[kDigits / kThreads], tokens = 0, total, v = 0;
#pragma unroll
            for (int j = 0; j < kDigits / kThreads; ++j) {
                bin[j] = sh.digits[threadIdx.x * (kDigits / kThreads) + j];
                tokens += tokens_in(bin[j]);
                v += weight_in(bin[j]);
            }
            int n = k.before + int(sum_before(sh, tokens, &total));
            uint64_t w = k.weight_before + sum_before(sh, v, &total);
#pragma unroll
            for (int j = 0; j < kDigits / kThreads; ++j) {
                const int d = threadIdx.x * (kDigits / kThreads) + j, more = tokens_in(bin[j]);
                const uint64_t after = w + weight_in(bin[j]);
                const bool here = by == By::kCount   ? n < count && n + more >= count
                                  : by == By::kReach ? double(w) < weight && double(after) >= weight
                                                     : double(w) <= weight && double(after) > weight;
                if (more > 0) atomicMax(&sh.found_last, d);
                if (here) {
                    sh.found = d;
                    sh.found_tokens = n;
                    sh.found_mass = w;
                    sh.found_bin = bin[j];
                }
                n += more;
                w = after;
            }
            __syncthreads();
            const int last = sh.found_last;
            if (sh.found < 0 && threadIdx.x == last / (kDigits / kThreads)) {  // behind all: the last one
                const int j = last % (kDigits / kThreads);
                uint64_t own = 0;
                int more = 0;
#pragma unroll
                for (int e = 0; e < kDigits / kThreads; ++e)
                    if (e >= j) {
                        own += weight_in(bin[e]);
                        more += tokens_in(bin[e]);
                    }
                sh.found_tokens = n - more;
                sh.found_mass = w - own;
                sh.found_bin = sh.digits[last];
            }
            __syncthreads();
            const int d = sh.found < 0 ? last : sh.found;
            k.key |= uint32_t(d) << shift;
            k.before = sh.found_tokens;
            k.weight_before = sh.found_mass;
            k.equal = tokens_in(sh.found_bin);
        }
        const double each = double(weight_of(k.key, b));
        if (by == By::kCount) {
            k.place = count - k.before - 1;
        } else {
            // kReach: the last token that has less than `weight` before it; kAbove: the first with more up to it
            const double into = (weight - double(k.weight_before)) / each;
            k.place = by == By::kReach ? int(ceil(into)) - 1 : int(floor(into));
        }
        k.place = min(max(k.place, 0), k.equal - 1);
        return k;
    }
    // Index of a token among those with its key.
    __device__ int index_of(const Token& k) {
        uint64_t before = 0;
        for (int i0 = 0; i0 < row.vocab; i0 += 8 * kThreads) {
            const int i = i0 + 8 * int(threadIdx.x);
            uint64_t mine = 0, total;
            for (int e = 0; e < 8; ++e)
                if (i + e < row.vocab) {
                    const float x = row.at(i + e);
                    mine += x == x && key_of(x) == k.key;
                }
            const uint64_t place = uint64_t(k.place) - before - sum_before(sh, mine, &total);
            if (place < mine) {
                uint64_t left = place;
                for (int e = 0; e < 8; ++e)
                    if (i + e < row.vocab) {
                        const float x = row.at(i + e);
                        if (x == x && key_of(x) == k.key && left-- == 0) sh.index = i + e;
                    }
            }
            before += total;
            if (before > uint64_t(k.place)) break;
        }
        __syncthreads();
        return sh.index;
    }

    // The first `count` tokens of bin b, or those with less than `weight` before them.
    __device__ void first(Prefix& p, int b, int n, By by, int count, double weight) {
        if (n <= kList) {
            collect(b, n);
            const int m = by == By::kCount ? count : max(1, leading(n, [&](int i) { return i == 0 || double(sh.list[i - 1]) < weight; }));
            ends(p, m);
        } else {
            const Token k = descend(b, by, count, weight);
            p.tokens = k.before + k.place + 1;
            p.ties = k.place + 1;
            p.key = k.key;
            p.weight = k.weight_before + uint64_t(k.place + 1) * weight_of(k.key, b);
        }
    }
    // p's end from the list, m > 0 tokens in.
    __device__ void ends(Prefix& p, int m) {
        p.tokens = m;
        p.key = uint32_t(sh.sorted[m - 1] >> 32);
        p.ties = m - leading(m, [&](int i) { return uint32_t(sh.sorted[i] >> 32) < p.key; });
        p.weight = sh.list[m - 1];
    }
    // Those of bin b whose logit is at least `cut`.
    __device__ void at_least(Prefix& p, int b, int n, float cut) {
        const uint32_t key = key_of(cut);
        if (n <= kList) {
            collect(b, n);
            const int m = leading(n, [&](int i) { return uint32_t(sh.sorted[i] >> 32) <= key; });
            if (m > 0) ends(p, m);
            else p.tokens = 0, p.weight = 0;
            return;
        }
        uint64_t mine = 0, total;
        row.each_under(sh.tops, double(b + 1), [&](int, float x) {
            const double t = row.t_of(x);
            if (t >= double(b) && t < double(b + 1) && key_of(x) <= key) mine += (uint64_t(1) << kMissBits) | miss_at(t - b);
        });
        sum_before(sh, mine, &total);
        p.tokens = tokens_in(total);
        p.weight = weight_in(total);
        p.key = key + 1;  // (with no ties: all up to the cut)
        p.ties = 0;
    }
    // The first token of bin b (n tokens, of which `most` are kept) with more than `weight` up to it: index and weight.
    __device__ void draw(int b, int n, int most, double weight, int* index, uint64_t* w) {
        uint32_t key;
        if (n <= kList) {
            collect(b, n);
            const int i = min(leading(n, [&](int k) { return double(sh.list[k]) <= weight; }), most - 1);
            key = uint32_t(sh.sorted[i] >> 32);
            *index = int(uint32_t(sh.sorted[i]));
        } else {
            Token k = descend(b, By::kAbove, 0, weight);
            if (k.before + k.place >= most) k = descend(b, By::kCount, most, 0.0);
            key = k.key;
            *index = index_of(k);
        }
        *w = weight_of(key, b);
    }
};

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
    __shared__ Shared sh;
    constexpr int V = Row<T>::V;
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    const int64_t of = a.params_of ? a.params_of[r] : r;
    const bool arrays = a.temperatures || a.top_ks || a.top_ps || a.min_ps;
    if ((arrays || a.params_of) && (of < 0 || of >= a.num_params)) {
        if (tid == 0) {
            a.tokens[r] = -1;
            if (a.conf) a.conf[r] = 0.0f;
        }
        return;
    }
    float temperature = a.temperatures ? a.temperatures[of] : a.temperature;
    if (!(temperature > 0.0f)) temperature = 0.0f;
    int top_k = a.top_ks ? a.top_ks[of] : a.top_k;
    float top_p = a.top_ps ? a.top_ps[of] : a.top_p;
    if (!(top_p < 1.0f)) top_p = 1.0f;
    float min_p = a.min_ps ? a.min_ps[of] : a.min_p;
    if (!(min_p > 0.0f)) min_p = 0.0f;
    const bool greedy = temperature == 0.0f;
    const double T_ = greedy ? 1.0 : double(temperature);

    Row<T> row;
    row.p = static_cast<const T*>(a.logits) + r * a.row_stride;
    row.vocab = a.vocab;
    row.forbid = a.forbid;
    row.infinite = false;
    row.head = min(int((16 - (reinterpret_cast<uintptr_t>(row.p) & 15)) & 15) / int(sizeof(T)), a.vocab);
    row.vectors = (a.vocab - row.head) / V;
    row.groups = (row.vectors + 63) / 64;

    // the largest logit, its first index, and the second largest
    float best = -INFINITY, second = -INFINITY;
    int at = INT32_MAX;
    auto look = [&](float x) {
        x = fmaxf(x, -INFINITY);  // (no number)
        second = fmaxf(second, fminf(best, x));
        best = fmaxf(best, x);
    };
    row.each_vector([](int) { return true; },
                    [&](int g, int i0, const float(&x)[V]) {
                        float m = x[0];
#pragma unroll
                        for (int e = 1; e < V; ++e) m = fmaxf(m, x[e]);
                        if (m > best) at = i0;
#pragma unroll
                        for (int e = 0; e < V; ++e) look(x[e]);
#pragma unroll
                        for (int d = 32; d > 0; d /= 2) m = fmaxf(m, __shfl_xor(m, d));
                        if (lane == 0) sh.tops[g] = m;
                    });
    row.each_edge([&](int i, float x) {
        if (x > best || (x == best && i < at)) at = i;
        look(x);
    });
    float top = best;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    if (lane == 0) sh.sums[wave] = top;
    if (tid == 0) sh.index = INT32_MAX;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, float(sh.sums[w]));
    if (!(top > -INFINITY)) {  // nothing to take
        if (tid == 0) {
            a.tokens[r] = -1;
            if (a.conf) a.conf[r] = 0.0f;
        }
        return;
    }
    if (best == top)
        for (int e = 0; e < V && at + e < a.vocab; ++e)
            if (row.at(at + e) == top) {
                atomicMin(&sh.index, at + e);
                break;
            }
    // the second of all: the first of the others, or this one's second where it holds the first
    int holders = __syncthreads_count(best == top);
    float next = best == top && holders == 1 ? second : best;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) next = fmaxf(next, __shfl_xor(next, d));
    __syncthreads();
    if (lane == 0) sh.sums[wave] = next;
    for (int b = tid; b < kBins; b += kThreads) sh.bins[b] = 0;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) next = fmaxf(next, float(sh.sums[w]));
    const int first_index = sh.index;
    if (top == INFINITY) {
        row.infinite = true;
        top = 0.0f;
        next = next == INFINITY ? 0.0f : -INFINITY;
        for (int g = tid; g < row.groups; g += kThreads) sh.tops[g] = sh.tops[g] == INFINITY ? 0.0f : -INFINITY;
        __syncthreads();
    }
    row.top = double(top);
    row.scale = 64.0 * 1.4426950408889634074 / T_;

    // bins
    row.each_under(sh.tops, double(kBins), [&](int, float x) {
        const double t = row.t_of(x);
        if (t < double(kBins)) {
            const int b = int(t);
            atomicAdd(reinterpret_cast<unsigned long long*>(&sh.bins[b]), (uint64_t(1) << kMissBits) | miss_at(t - b));
        }
    });
    __syncthreads();
    uint64_t mass[kEach], tokens = 0, mine = 0, all_tokens, all_mass;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint64_t bin = sh.bins[tid * kEach + j];
        mass[j] = bin ? mass_of(tid * kEach + j, weight_in(bin)) : 0;
        tokens += tokens_in(bin);
        mine += mass[j];
    }
    const int tokens_before = int(sum_before(sh, tokens, &all_tokens));
    const uint64_t mass_before = sum_before(sh, mine, &all_mass);
    // the bin for which here(bin, tokens before, tokens, mass before, mass) holds; at most one; -1: none
    auto find = [&](auto here) {
        __syncthreads();
        if (tid == 0) sh.found = -1;
        __syncthreads();
        int n = tokens_before;
        uint64_t w = mass_before;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int b = tid * kEach + j, more = tokens_in(sh.bins[b]);
            if (here(b, n, more, w, mass[j])) {
                sh.found = b;
                sh.found_tokens = n;
                sh.found_mass = w;
            }
            n += more;
            w += mass[j];
        }
        __syncthreads();
        return sh.found;
    };
    int listed = -1;
    Bin<T> bin{sh, row, listed};
    Prefix kept{kBins, 0, 0, 0, 0, all_mass, int(all_tokens)};
    auto only_first = [&] {
        kept = Prefix{0, 1, 1, key_of(top), kOne, 0, 0};
    };
    if (top_k > 0 && top_k < int(all_tokens)) {
        const int b = find([&](int, int n, int more, uint64_t, uint64_t) { return n < top_k && n + more >= top_k; });
        kept.bin = b;
        kept.before = sh.found_tokens;
        kept.mass = sh.found_mass;
        bin.first(kept, b, tokens_in(sh.bins[b]), By::kCount, top_k - kept.before, 0.0);
    }
    if (top_p < 1.0f) {
        const double share = ceil(double(top_p) * double(kept.all()));
        if (!(share > 0.0)) {
            only_first();
        } else {
            const uint64_t reach = uint64_t(share);
            const int b = find([&](int, int, int, uint64_t w, uint64_t m) { return w < reach && w + m >= reach; });
            if (b >= 0 && b <= kept.bin) {
                Prefix p{b, 0, 0, 0, 0, sh.found_mass, sh.found_tokens};
                bin.first(p, b, tokens_in(sh.bins[b]), By::kReach, 0, inside(b, double(reach - p.mass)));
                if (b < kept.bin || p.tokens < kept.tokens) kept = p;
            }
        }
    }
    if (min_p > 0.0f) {
        const double low = log(double(min_p));
        if (!(low <= 0.0)) {
            only_first();
        } else {
            // the lowest logit that is kept: an estimate, then by the definition
            auto keeps = [&](float x) { return (double(x) - double(top)) / T_ >= low; };
            float cut = float(fmax(double(top) + T_ * low, -3.4e38));
            for (int k = 0; k < 4 && !keeps(cut); ++k) cut = nextafterf(cut, INFINITY);
            for (int k = 0; k < 4 && keeps(nextafterf(cut, -INFINITY)) && nextafterf(cut, -INFINITY) > -INFINITY; ++k) cut = nextafterf(cut, -INFINITY);
            cut = fminf(cut, top);
            const double t = row.t_of(cut);
            if (t < double(kBins) && int(t) <= kept.bin) {
                const int b = int(t);
                find([&](int k, int, int, uint64_t, uint64_t) { return k == b; });
                Prefix p{b, 0, 0, 0, 0, sh.found_mass, sh.found_tokens};
                if (tokens_in(sh.bins[b]) > 0) bin.at_least(p, b, tokens_in(sh.bins[b]), cut);
                if (b < kept.bin || p.tokens < kept.tokens) kept = p;
            }
        }
    }
    const uint64_t M = kept.all();
    const double unit = 0x1p44 / double(M);  // weights as shares of M
    int token = first_index;
    double weight = 1.0;
    if (!greedy) {
        const float u = a.u[r];
        const double target = fmin(u > 0.0f ? double(u) * double(M) : 0.0, double(M - 1));
        const uint64_t above = uint64_t(target);
        const int b = find([&](int, int, int, uint64_t w, uint64_t m) { return w <= above && w + m > above; });
        if (b >= 0) {
            const int n = tokens_in(sh.bins[b]);
            uint64_t v;
            const double into = fmax(0.0, inside(b, target - double(sh.found_mass)));
            bin.draw(b, n, b == kept.bin ? kept.tokens : n, into, &token, &v);
            weight = bin_weight(b) * double(v) * 0x1p-33;
        }
    }
    double c = weight * unit;
    if (a.confidence == SANGAM_CONFIDENCE_MARGIN) {
        double other = 0.0;
        const double t = row.t_of(next);
        if (kept.before + kept.tokens > 1 && t < double(kBins)) other = bin_weight(int(t)) * double(kOne - miss_at(t - int(t))) * 0x1p-33;
        c = (1.0 - other) * unit;
    } else if (a.confidence == SANGAM_CONFIDENCE_ENTROPY) {
        double s = 0.0;
        auto part = [&](double t) { return bin_weight(int(t)) * double(kOne - miss_at(t - int(t))) * 0x1p-33 * t; };
        row.each_under(sh.tops, double(min(kept.bin + 1, kBins)), [&](int, float x) {
            const double t = row.t_of(x);
            if (t < double(kept.bin) || (kept.tokens > 0 && t < double(kept.bin + 1) && key_of(x) < kept.key)) s += part(t);
        });
        s = sum_all(sh, s);
        if (kept.tokens > 0 && kept.ties > 0) s += kept.ties * part(row.t_of(logit_of(kept.key)));
        c = -(s * unit * (0.69314718055994530942 / 64) + log(double(M) * 0x1p-44));
    }
    if (tid == 0) {
        a.tokens[r] = token;
        if (a.conf) a.conf[r] = float(c);
    }
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
    const void* fn = d->dtype == SANGAM_DTYPE_FP32   ? reinterpret_cast<const void*>(&sample_kernel<float>)
                     : d->dtype == SANGAM_DTYPE_FP16 ? reinterpret_cast<const void*>(&sample_kernel<_Float16>)
                                                     : reinterpret_cast<const void*>(&sample_kernel<__bf16>);
    // a grid's threads are counted in 32 bits
    const int64_t step = (int64_t(1) << 32) / kThreads - 1;
    for (int64_t row = 0; row < d->rows; row += step) {
        SampleArgs some = args;
        some.logits = static_cast<const uint8_t*>(d->logits) + row * d->row_stride * int64_t(size);
        some.u += row;
        if (some.params_of) some.params_of += row;
        some.tokens += row;
        if (some.conf) some.conf += row;
        void* kargs[] = {&some};
        const hipError_t e = hipLaunchKernel(fn, dim3(unsigned(std::min(step, d->rows - row))), dim3(kThreads), kargs, 0, static_cast<hipStream_t>(stream));
        if (e != hipSuccess) return fail(SANGAM_ERR_HIP, std::string("sampling launch: ") + hipGetErrorString(e));
    }
    return SANGAM_OK;
}

}  // namespace

extern "C" size_t sangam_sample_workspace_bytes(int64_t, int32_t, int32_t) { return 0; }

extern "C" sangam_status sangam_sample_tokens(const sangam_sample_desc* desc, int32_t* tokens, float* confidence, void* workspace,
                                              size_t workspace_bytes, void* stream) {
    return entry([&] { return sample(desc, tokens, confidence, workspace, workspace_bytes, stream); });
}
