// Which masked rows of a block take their token, for gfx950, with its C ABI
// entry point (include/sangam_sample.h).
//
// The `count` most confident candidates are those above a border key, and of
// those equal to it the lowest rows. The border is found bit by bit: with the
// confidences as whole numbers of their order, the largest key that at least
// `count` of them reach. A block is a wave's, its keys in registers (up to 4 a
// lane), a bit of the border one ballot a register; larger blocks are a
// work-group's, by digits of 8 bits counted in LDS, up to 4096 rows with their
// keys there, too. A launch moves 16 bytes a row and is bound by its own
// latency: one block of 32 rows takes 2.8 us, 4096 of them 5.3, 64 of 256 rows
// 5.4, 120 of 1024 8.0, 120 of 2048 11.4; 4097 rows 40.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "../../include/sangam_sample.h"
#include "entry.h"
#include "wave_sum.h"

namespace sangam {
void set_error(const std::string& msg);
void clear_error();
}  // namespace sangam

using namespace sangam;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kKeys = 4;     // of a lane: blocks of up to 256 rows are a wave's (1024 take 15.1 us by a wave, 7.5 by a work-group)
// A grid's threads are counted in 32 bits. (Blocks that have a work-group to themselves hold over 128 rows each on average: under 2^24 of them.)
constexpr int kMostBlocks = kWaves * ((1 << 24) - 1);
constexpr int kHeld = 4096;  // keys of a work-group: blocks of up to so many rows are looked at once

struct UnmaskArgs {
    const int32_t* tokens;
    const float* confidence;
    int32_t* ids;
    const int64_t* slots;
    const int32_t* row_indptr;
    const int32_t* counts;
    const float* thresholds;
    int64_t rows, num_ids;
    int32_t num_blocks, mask_id, count;
    float threshold;
    int32_t *out, *left;
    int32_t each;  // blocks of a work-group, up to one a wave
};

// A row's id before the step, and where it lies (nullptr: nowhere to be written).
__device__ __forceinline__ int id_of(const UnmaskArgs& a, int64_t r, int32_t** place) {
    *place = nullptr;
    if (!a.slots) return a.ids[r];
    const int64_t s = a.slots[r];
    if (s < 0 || s >= a.num_ids) return -1;
    *place = a.ids + s;
    return a.ids[s];
}

// 1 + a whole number in the order of the confidences (no number: the least); 0 for a row that is no candidate.
__device__ __forceinline__ uint32_t key_of(float c) {
    if (!(c == c)) return 1;
    c += 0.0f;  // -0 equals 0
    const uint32_t b = __float_as_uint(c);
    return ((b >> 31) ? ~b : b | 0x80000000u) - 0x7FFFFFu + 2;  // -inf is 0x7FFFFF
}

struct Row {
    int id;
    uint32_t key;
    bool sure;  // reaches the threshold
};

__device__ __forceinline__ Row row_at(const UnmaskArgs& a, int64_t r, float threshold) {
    Row x;
    int32_t* place;
    x.id = id_of(a, r, &place);
    const int token = a.tokens[r];
    const float c = a.confidence[r];
    if (a.slots && !place) x.id = ~a.mask_id;  // (mask_id may be -1)
    const bool candidate = x.id == a.mask_id && token >= 0 && token != a.mask_id;
    x.key = candidate ? key_of(c) : 0;
    x.sure = candidate && c >= threshold;
    return x;
}

__device__ __forceinline__ void put(const UnmaskArgs& a, int64_t r, bool takes) {
    int32_t* place;
    int id = id_of(a, r, &place);
    if (takes) {
        id = a.tokens[r];
        if (place) *place = id;
    }
    a.out[r] = id;
}

__device__ __forceinline__ int ones(uint64_t m) { return __builtin_popcountll(m); }

// A block of n <= 64 K rows, by one wave.
template <int K>
__device__ __forceinline__ void by_wave(const UnmaskArgs& a, int block, int64_t r0, int n, int count, float threshold) {
    const int lane = threadIdx.x & 63;
    uint32_t key[K], sure = 0;
    int candidates = 0, masked = 0;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        key[j] = 0;
        bool hidden = false;
        if (64 * j + lane < n) {
            const Row x = row_at(a, r0 + 64 * j + lane, threshold);
            key[j] = x.key;
            sure |= uint32_t(x.sure) << j;
            hidden = x.id == a.mask_id;
        }
        candidates += ones(__ballot(key[j] > 0));
        masked += ones(__ballot(hidden));
    }
    // the border: the largest key that `count` candidates reach; 1 where all are taken
    uint32_t border = 1;
    int ties = n;  // equal to the border, to be taken
    if (count <= 0) {
        border = 0xFFFFFFFFu;
        ties = 0;
    } else if (count < candidates) {
        border = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t next = border | (1u << bit);
            int reach = 0;
#pragma unroll
            for (int j = 0; j < K; ++j) reach += ones(__ballot(key[j] >= next));
            if (reach >= count) border = next;
        }
        int above = 0;
#pragma unroll
        for (int j = 0; j < K; ++j) above += ones(__ballot(key[j] > border));
        ties = count - above;
    }
    int taken = 0, equal = 0;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const uint64_t same = __ballot(key[j] > 0 && key[j] == border);
        const int mine = equal + ones(same & ((uint64_t(1) << lane) - 1));
        equal += ones(same);
        const bool takes = key[j] > 0 && (((sure >> j) & 1) || key[j] > border || (key[j] == border && mine < ties));
        taken += ones(__ballot(takes));
        if (64 * j + lane < n) put(a, r0 + 64 * j + lane, takes);
    }
    if (a.left && lane == 0) a.left[block] = masked - taken;
}

struct Groups {
    int bins[256];
    int part[kWaves];
    uint32_t key[kHeld];
};

// Sum over the work-group.
__device__ __forceinline__ int sum_all(Groups& sh, int x) {
    x = wave_up_to(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh.part[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += sh.part[w];
    return x;
}

// The `count`-th largest key, and how many of those equal to it are among the `count` largest; each(f) calls f with every
// key, 0 < count <= number of keys above 0. Every wave finds a digit by itself, a lane holding four bins from the top.
template <typename F>
__device__ __forceinline__ uint32_t border_of(Groups& sh, int count, int& ties, F each) {
    const int tid = threadIdx.x, lane = tid & 63;
    uint32_t known = 0;
    int wanted = count;  // among the keys that begin as the border does
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        sh.bins[tid] = 0;
        __syncthreads();
        each([&](uint32_t key) {
            if (key > 0 && (uint64_t(key) >> (shift + 8)) == (uint64_t(known) >> (shift + 8))) atomicAdd(&sh.bins[(key >> shift) & 255], 1);
        });
        __syncthreads();
        int n[4], up_to = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) up_to += n[k] = sh.bins[255 - 4 * lane - k];
        const int mine = up_to;
        up_to = wave_up_to(up_to);
        const uint64_t in = __ballot(up_to >= wanted);
        const int at = in ? __builtin_ctzll(in) : 63;
        int above = up_to - mine, digit = 255 - 4 * lane;
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (digit == 255 - 4 * lane - k && above + n[k] < wanted) {
                above += n[k];
                digit -= 1;
            }
        known |= uint32_t(__builtin_amdgcn_readlane(digit, at)) << shift;
        wanted -= __builtin_amdgcn_readlane(above, at);
    }
    ties = wanted;
    return known;
}

// A block of up to kHeld rows, by a whole work-group: a wave's rows follow one another. (Keys in registers take 104 of them and
// spill the ballots of 16 a lane: 4096 blocks of 32 rows then take 11.2 us beside them.)
__device__ __forceinline__ void by_group_held(Groups& sh, const UnmaskArgs& a, int block, int64_t r0, int n, int count, float threshold) {
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const int first = (n + kThreads - 1) / kThreads * 64 * wave + lane, end = min(first - lane + (n + kThreads - 1) / kThreads * 64, n);
    uint32_t sure = 0;
    int candidates = 0, masked = 0;
#pragma unroll 4
    for (int i = first; i < end; i += 64) {
        const Row x = row_at(a, r0 + i, threshold);
        sh.key[i] = x.key;
        sure = sure << 1 | uint32_t(x.sure);
        candidates += x.key > 0;
        masked += x.id == a.mask_id;
    }
    sure = __brev(sure) >> ((32 - (first < end ? (end - first + 63) / 64 : 0)) & 31);  // the first one's bit lowest again
    candidates = sum_all(sh, candidates);
    uint32_t border = count <= 0 ? 0xFFFFFFFFu : 1;
    int ties = count <= 0 ? 0 : n;
    if (count > 0 && count < candidates)
        border = border_of(sh, count, ties, [&](auto f) {
#pragma unroll 4
            for (int i = first; i < end; i += 64) f(sh.key[i]);
        });
    // those equal to the border before this wave's
    int own = 0;
    for (int i = first; i < end; i += 64) own += border > 0 && sh.key[i] == border;
    own = wave_up_to(own);
    __syncthreads();
    if (lane == 63) sh.part[wave] = own;
    __syncthreads();
    int equal = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (w < wave) equal += sh.part[w];
    for (int i0 = first - lane; i0 < end; i0 += 64) {
        const int i = i0 + lane;
        const uint32_t key = i < end ? sh.key[i] : 0;
        const uint64_t same = __ballot(key > 0 && key == border);
        const int mine = equal + ones(same & ((uint64_t(1) << lane) - 1));
        equal += ones(same);
        const bool takes = key > 0 && ((sure & 1) || key > border || (key == border && mine < ties));
        sure >>= 1;
        masked -= takes;
        if (i < end) put(a, r0 + i, takes);
    }
    masked = sum_all(sh, masked);
    if (a.left && threadIdx.x == 0) a.left[block] = masked;
}

// A block of any size, by a whole work-group, which looks at it six times.
__device__ __forceinline__ void by_group(Groups& sh, const UnmaskArgs& a, int block, int64_t r0, int64_t n, int count, float threshold) {
    const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
    int candidates = 0;
    for (int64_t i = tid; i < n; i += kThreads) candidates += row_at(a, r0 + i, threshold).key > 0;
    candidates = sum_all(sh, candidates);
    uint32_t border = count <= 0 ? 0xFFFFFFFFu : 1;
    int64_t ties = count <= 0 ? 0 : n;
    if (count > 0 && count < candidates) {
        int among = 0;
        border = border_of(sh, count, among, [&](auto f) {
            for (int64_t i = tid; i < n; i += kThreads) f(row_at(a, r0 + i, threshold).key);
        });
        ties = among;
    }
    // rows in order, so that the lowest of equal ones are taken
    int64_t equal = 0;
    int masked = 0;
    for (int64_t i0 = 0; i0 < n; i0 += kThreads) {
        const int64_t i = i0 + tid;
        Row x{~a.mask_id, 0, false};
        if (i < n) x = row_at(a, r0 + i, threshold);
        const uint64_t same = __ballot(x.key > 0 && x.key == border);
        __syncthreads();
        if (lane == 0) sh.part[wave] = ones(same);
        __syncthreads();
        int64_t mine = equal + ones(same & ((uint64_t(1) << lane) - 1));
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) mine += sh.part[w];
            equal += sh.part[w];
        }
        const bool takes = x.key > 0 && (x.sure || x.key > border || (x.key == border && mine < ties));
        if (i < n) {
            put(a, r0 + i, takes);
            masked += x.id == a.mask_id && !takes;
        }
    }
    masked = sum_all(sh, masked);
    if (a.left && tid == 0) a.left[block] = masked;
}

// Work-group g: blocks each g and on, a wave each, then those of them that are
// larger; the rows outside all blocks are dealt over the work-groups.
__global__ __launch_bounds__(kThreads) void unmask_kernel(UnmaskArgs a) {
    __shared__ Groups sh;
    const int wave = threadIdx.x / 64;
    auto block_at = [&](int b, int64_t& r0, int64_t& n) {
        r0 = min(max(int64_t(a.row_indptr[b]), int64_t(0)), a.rows);
        n = max(min(int64_t(a.row_indptr[b + 1]), a.rows) - r0, int64_t(0));
    };
    auto count_of = [&](int b) { return a.counts ? a.counts[b] : a.count; };
    auto threshold_of = [&](int b) { return a.thresholds ? a.thresholds[b] : a.threshold; };
    bool large = false;
    for (int w = 0; w < a.each; ++w) {
        const int b = blockIdx.x * a.each + w;
        if (b >= a.num_blocks) break;
        int64_t r0, n;
        block_at(b, r0, n);
        if (n > 64 * kKeys) large = true;
        else if (w != wave) continue;
        else if (n <= 64) by_wave<1>(a, b, r0, int(n), count_of(b), threshold_of(b));
        else by_wave<kKeys>(a, b, r0, int(n), count_of(b), threshold_of(b));
    }
    if (large)
        for (int w = 0; w < a.each; ++w) {
            const int b = blockIdx.x * a.each + w;
            if (b >= a.num_blocks) break;
            int64_t r0, n;
            block_at(b, r0, n);
            if (n > 64 * kKeys && n <= kHeld) by_group_held(sh, a, b, r0, int(n), count_of(b), threshold_of(b));
            if (n > kHeld) by_group(sh, a, b, r0, n, count_of(b), threshold_of(b));
        }
    const int64_t before = min(max(int64_t(a.row_indptr[0]), int64_t(0)), a.rows);
    const int64_t behind = max(min(max(int64_t(a.row_indptr[a.num_blocks]), int64_t(0)), a.rows), before);
    const int64_t outside = before + (a.rows - behind);
    for (int64_t k = int64_t(blockIdx.x) * kThreads + threadIdx.x; k < outside; k += int64_t(gridDim.x) * kThreads) {
        const int64_t r = k < before ? k : k - before + behind;
        int32_t* place;
        a.out[r] = id_of(a, r, &place);
    }
}

sangam_status fail(sangam_status code, const std::string& msg) {
    set_error(msg);
    return code;
}

sangam_status unmask(const sangam_unmask_desc* d, int32_t* out, int32_t* left, void* stream) {
    clear_error();
    if (!d || d->rows < 0 || d->rows > INT32_MAX || d->num_blocks < 0 || d->num_blocks > kMostBlocks || d->num_ids < 0)
        return fail(SANGAM_ERR_INVALID_ARG, "desc must not be NULL, rows 0 to 2^31 - 1, num_blocks 0 to 4 (2^24 - 1), num_ids not negative");
    if (d->count < 0) return fail(SANGAM_ERR_INVALID_ARG, "count must not be negative");
    if (!d->thresholds && std::isnan(d->threshold)) return fail(SANGAM_ERR_INVALID_ARG, "threshold must be a number");
    if (!d->row_indptr) return fail(SANGAM_ERR_INVALID_ARG, "row_indptr must not be NULL");
    if (d->rows > 0 && (!d->tokens || !d->confidence || !out || (!d->ids && (!d->slots || d->num_ids > 0))))
        return fail(SANGAM_ERR_INVALID_ARG, "tokens, confidence, ids and out must not be NULL");
    if (!d->slots && d->num_ids < d->rows) return fail(SANGAM_ERR_INVALID_ARG, "ids must hold an id for every row");
    for (const void* p : {static_cast<const void*>(d->tokens), static_cast<const void*>(d->confidence), static_cast<const void*>(d->ids),
                          static_cast<const void*>(d->row_indptr), static_cast<const void*>(d->counts), static_cast<const void*>(d->thresholds),
                          static_cast<const void*>(out), static_cast<const void*>(left)})
        if (reinterpret_cast<uintptr_t>(p) % 4) return fail(SANGAM_ERR_ALIGN, "the arrays must be 4-byte aligned");
    if (reinterpret_cast<uintptr_t>(d->slots) % 8) return fail(SANGAM_ERR_ALIGN, "slots must be 8-byte aligned");
    if (d->rows == 0 && (d->num_blocks == 0 || !left)) return SANGAM_OK;
    // blocks of over 128 rows on average have a work-group to themselves, so that large ones do not wait for one another
    const int32_t each = d->rows > int64_t(d->num_blocks) * (kThreads / 2) ? 1 : kWaves;
    UnmaskArgs args{d->tokens, d->confidence, d->ids, d->slots, d->row_indptr, d->counts, d->thresholds, d->rows, d->num_ids,
                    d->num_blocks, d->mask_id, d->count, d->threshold, out, left, each};
    void* kargs[] = {&args};
    const int64_t groups = std::max<int64_t>((int64_t(d->num_blocks) + args.each - 1) / args.each, std::min<int64_t>((d->rows + kThreads - 1) / kThreads, 64));
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&unmask_kernel), dim3(unsigned(std::max<int64_t>(groups, 1))), dim3(kThreads), kargs, 0,
                                         static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SANGAM_OK : fail(SANGAM_ERR_HIP, std::string("unmask launch: ") + hipGetErrorString(e));
}

}  // namespace

extern "C" sangam_status sangam_sample_unmask(const sangam_unmask_desc* desc, int32_t* out, int32_t* left, void* stream) {
    return entry([&] { return unmask(desc, out, left, stream); });
}
