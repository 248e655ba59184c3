// Block tables that follow their requests' lengths, and the page list, positions
// and slots of a batch, for gfx950, with their C ABI entry points
// (include/sangam_tables.h).
//
// Both move a few bytes per page and row (the batch of a busy worker: some tens
// of KB, 0.01 us of a copy), so what they cost is the launch and a chain of
// dependent loads: sizes, their prefix sum, the entries. One launch each, the
// prefix sums in LDS. A batch of 32 decodes or of 48 beside long prefills is
// built in 4.8 to 5.3 us of the kernel, 13.5 from Python; 1024 items of 32 rows in
// 6.4, 1025 by two launches in 9.4, 4096 (385,000 pages) in 15.4.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "../../include/sangam_tables.h"
#include "entry.h"
#include "offsets.h"
#include "wave_sum.h"

namespace sangam {
void set_error(const std::string& msg);
void clear_error();
}  // namespace sangam

using namespace sangam;

namespace {

constexpr int kPage = 16;
constexpr int kResizeThreads = 1024;
constexpr int kBuildThreads = 256;
constexpr int kItemsInLds = 1024;
constexpr int kMost = 1 << 30;  // requests and items: they are counted on in steps of work-groups, in 32 bits

__device__ __forceinline__ int pages_of(int len) { return len <= 0 ? 0 : (len - 1) / kPage + 1; }

// Sum over the threads before this one; *total over all. `part`: an entry per wave.
template <int THREADS>
__device__ int64_t sum_before(int64_t x, int64_t* part, int64_t* total) {
    const int wave = threadIdx.x / 64;
    const int64_t up_to = int64_t(wave_up_to(uint64_t(x)));
    __syncthreads();
    if ((threadIdx.x & 63) == 63) part[wave] = up_to;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const int64_t p = part[w];
        if (w < wave) before += p;
        all += p;
    }
    *total = all;
    return before + up_to - x;
}

struct ResizeArgs {
    int32_t* pages;
    int64_t row_stride;
    int32_t* held;
    const int32_t* lengths;
    int32_t* free_pages;
    int32_t* num_free;
    int32_t* short_of;
    int32_t requests, max_pages, free_cap;
};

// One work-group: what a request takes depends on all before it. The pages that
// move are dealt over the threads one by one, each finds its request by its number:
// 12,800 pages of 100 requests among 1024 are taken in 11.2 us and given back in
// 13.2 (by a wave a request 16.8 and 27.5).
__global__ __launch_bounds__(kResizeThreads) void tables_resize_kernel(ResizeArgs a) {
    __shared__ int64_t part[kResizeThreads / 64];
    __shared__ int64_t at[kResizeThreads];  // moves before a request's
    __shared__ int32_t first[kResizeThreads];
    const int tid = threadIdx.x;
    const int64_t had = min(max(a.num_free[0], 0), a.free_cap);
    int held, need;
    auto look = [&](int r) {
        held = r < a.requests ? min(max(a.held[r], 0), a.max_pages) : 0;
        need = r < a.requests ? pages_of(a.lengths[r]) : 0;
    };
    const bool one = a.requests <= kResizeThreads;  // (then a look is enough)
    look(tid);
    // the `moves` of requests [r0, r0 + kResizeThreads), numbered from `before`: take(entry of the table, number) gives a
    // page, which put(entry, number, page) moves; some are on their way together
    auto each_move = [&](int r0, int64_t before, int64_t moves, auto take, auto put) {
        constexpr int kTogether = 4;
        for (int64_t k0 = tid; k0 < moves; k0 += kTogether * kResizeThreads) {
            int32_t *entry[kTogether], page[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const int64_t k = k0 + j * kResizeThreads;
                entry[j] = nullptr;
                if (k >= moves) continue;
                int i = 0;  // the last request whose moves begin at or before this one
#pragma unroll
                for (int step = kResizeThreads / 2; step > 0; step /= 2)
                    if (at[i + step] <= before + k) i += step;
                entry[j] = a.pages + int64_t(r0 + i) * a.row_stride + first[i] + (before + k - at[i]);
                page[j] = take(entry[j], before + k);
            }
#pragma unroll
            for (int j = 0; j < kTogether; ++j)
                if (entry[j]) put(entry[j], before + k0 + j * kResizeThreads, page[j]);
        }
    };
    // the pages that come back: how many, then where they go
    int64_t given = 0, total;
    for (int r0 = 0; r0 < a.requests; r0 += kResizeThreads) {
        if (!one) look(r0 + tid);
        sum_before<kResizeThreads>(max(held - need, 0), part, &total);
        given += total;
    }
    const int64_t many = had + given;
    if (given > 0) {
        int64_t before = 0;
        for (int r0 = 0; r0 < a.requests; r0 += kResizeThreads) {
            if (!one) look(r0 + tid);
            const int gives = max(held - need, 0);
            at[tid] = before + sum_before<kResizeThreads>(gives, part, &total);
            first[tid] = need;
            __syncthreads();
            each_move(r0, before, total, [](const int32_t* entry, int64_t) { return *entry; }, [&](int32_t* entry, int64_t k, int32_t page) {
                const int64_t place = many - 1 - k;
                if (place < a.free_cap) a.free_pages[place] = page;
                *entry = -1;
            });
            before += total;
            if (gives > 0) a.held[r0 + tid] = held = need;
            __syncthreads();
        }
    }
    // the pages that are taken: a request's all or none, none behind one that found too few
    const int64_t top = min(many, int64_t(a.free_cap));
    int64_t before = 0, taken = 0, short_of = 0;
    for (int r0 = 0; r0 < a.requests; r0 += kResizeThreads) {
        if (!one) look(r0 + tid);
        const int wants = need <= a.max_pages ? max(need - held, 0) : 0;
        const int64_t mine = before + sum_before<kResizeThreads>(wants, part, &total);
        const bool fits = mine + wants <= top;
        before += total;
        // (those that fit come first, so their moves are numbered on without a gap)
        constexpr int64_t kShort = int64_t(1) << 48;
        int64_t sums;
        const bool none = (!fits && wants > 0) || need > a.max_pages;
        sum_before<kResizeThreads>((fits ? wants : 0) + (none ? kShort : 0), part, &sums);
        at[tid] = fits ? mine : taken + sums % kShort;
        first[tid] = held;
        __syncthreads();
        each_move(r0, taken, sums % kShort, [&](const int32_t*, int64_t k) { return a.free_pages[top - 1 - k]; },
                  [](int32_t* entry, int64_t, int32_t page) { *entry = page; });
        if (fits && wants > 0) a.held[r0 + tid] = need;
        taken += sums % kShort;
        short_of += sums / kShort;
    }
    if (tid == 0) {
        a.num_free[0] = int32_t(top - taken);
        a.short_of[0] = int32_t(short_of);
    }
}

struct BuildArgs {
    const int32_t* pages;
    int64_t row_stride;
    int32_t requests, max_pages, items;
    const int32_t *request, *kv_len, *q_indptr, *q_offset, *q_pos;
    int32_t *page_indptr, *page_ids;
    int64_t num_pages;
    int32_t* positions;
    int64_t* slots;
    int32_t* row_items;
    int64_t rows;
};

// Offsets of the items' pages into out[0, items]; a whole work-group.
__device__ void page_offsets(const BuildArgs& a, int32_t* out, int64_t* part) {
    int64_t before = 0, total;
    for (int i0 = 0; i0 < a.items; i0 += kBuildThreads) {
        const int i = i0 + threadIdx.x;
        const int n = i < a.items ? min(pages_of(a.kv_len[i]), a.max_pages) : 0;
        const int64_t mine = before + sum_before<kBuildThreads>(n, part, &total);
        if (i < a.items) out[i + 1] = int32_t(min(mine + n, int64_t(INT32_MAX)));
        before += total;
    }
    if (threadIdx.x == 0) out[0] = 0;
}

__global__ __launch_bounds__(kBuildThreads) void tables_offsets_kernel(BuildArgs a) {
    __shared__ int64_t part[kBuildThreads / 64];
    page_offsets(a, a.page_indptr, part);
}

// SMALL: every work-group sums the items' pages by itself, in LDS; else they are
// in page_indptr.
template <bool SMALL>
__global__ __launch_bounds__(kBuildThreads) void tables_build_kernel(BuildArgs a) {
    __shared__ int64_t part[kBuildThreads / 64];
    __shared__ int32_t page_at[SMALL ? kItemsInLds + 1 : 1], row_at[SMALL ? kItemsInLds + 1 : 1];
    const int32_t *indptr = a.page_indptr, *q_indptr = a.q_indptr;
    if (SMALL) {
        page_offsets(a, page_at, part);
        for (int i = threadIdx.x; i <= a.items; i += kBuildThreads) row_at[i] = a.q_indptr[i];
        __syncthreads();
        if (blockIdx.x == 0)
            for (int i = threadIdx.x; i <= a.items; i += kBuildThreads) a.page_indptr[i] = page_at[i];
        indptr = page_at;
        q_indptr = row_at;
    }
    auto row_of = [&](int i) -> const int32_t* {
        const int r = a.request ? a.request[i] : i;
        return r >= 0 && r < a.requests ? a.pages + int64_t(r) * a.row_stride : nullptr;
    };
    const int64_t step = int64_t(gridDim.x) * kBuildThreads, t0 = int64_t(blockIdx.x) * kBuildThreads + threadIdx.x;
    if (a.page_ids)
        for (int64_t k = t0; k < a.num_pages; k += step) {
            const int i = last_offset(indptr, a.items, k);
            int page = -1;
            if (i >= 0 && i < a.items) {
                const int32_t* row = row_of(i);
                const int64_t j = k - indptr[i];
                if (row && j < a.max_pages) page = row[j];
            }
            a.page_ids[k] = page;
        }
    for (int64_t r = t0; r < a.rows; r += step) {
        const int i = last_offset(q_indptr, a.items, r);
        const bool in = i >= 0 && i < a.items;
        int pos = 0;
        int64_t slot = -1;
        if (in) {
            pos = a.q_pos ? a.q_pos[r] : int(uint32_t(a.q_offset[i]) + uint32_t(r - q_indptr[i]));
            const int32_t* row = row_of(i);
            if (row && pos >= 0 && pos < a.kv_len[i] && pos / kPage < a.max_pages) {
                const int page = row[pos / kPage];
                if (page >= 0) slot = int64_t(page) * kPage + pos % kPage;
            }
        }
        if (a.positions) a.positions[r] = pos;
        if (a.slots) a.slots[r] = slot;
        if (a.row_items) a.row_items[r] = in ? i : -1;
    }
}

sangam_status fail(sangam_status code, const std::string& msg) {
    set_error(msg);
    return code;
}

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

sangam_status check_table(const sangam_block_table* t) {
    if (!t || t->requests < 0 || t->requests > kMost || t->max_pages < 0)
        return fail(SANGAM_ERR_INVALID_ARG, "table must not be NULL, nor its requests outside 0 to 2^30, nor max_pages negative");
    if (t->requests > 0 && t->max_pages > 0) {
        if (!t->pages) return fail(SANGAM_ERR_INVALID_ARG, "the table's pages must not be NULL");
        if (t->row_stride < t->max_pages || t->row_stride > (int64_t(1) << 40))
            return fail(SANGAM_ERR_INVALID_ARG, "the table's row_stride must be max_pages to 2^40");
    }
    if (!aligned(t->pages, 4)) return fail(SANGAM_ERR_ALIGN, "the table must be 4-byte aligned");
    return SANGAM_OK;
}

sangam_status launched(hipError_t e, const char* what) {
    return e == hipSuccess ? SANGAM_OK : fail(SANGAM_ERR_HIP, std::string(what) + " launch: " + hipGetErrorString(e));
}

sangam_status resize(const sangam_block_table* table, int32_t* held, const int32_t* lengths, int32_t* free_pages, int32_t free_cap,
                     int32_t* num_free, int32_t* short_of, void* stream) {
    clear_error();
    if (const sangam_status s = check_table(table)) return s;
    if (free_cap < 0) return fail(SANGAM_ERR_INVALID_ARG, "free_cap must not be negative");
    if (!num_free || !short_of || (table->requests > 0 && (!held || !lengths)) || (free_cap > 0 && !free_pages))
        return fail(SANGAM_ERR_INVALID_ARG, "held, lengths, free_pages, num_free and short_of must not be NULL");
    for (const void* p : {static_cast<const void*>(held), static_cast<const void*>(lengths), static_cast<const void*>(free_pages),
                          static_cast<const void*>(num_free), static_cast<const void*>(short_of)})
        if (!aligned(p, 4)) return fail(SANGAM_ERR_ALIGN, "the arrays must be 4-byte aligned");
    ResizeArgs args{table->pages, table->row_stride, held, lengths, free_pages, num_free, short_of,
                    table->requests, table->max_pages, free_cap};
    void* kargs[] = {&args};
    return launched(hipLaunchKernel(reinterpret_cast<const void*>(&tables_resize_kernel), dim3(1), dim3(kResizeThreads), kargs, 0,
                                    static_cast<hipStream_t>(stream)), "table");
}

sangam_status build(const sangam_block_table* table, const sangam_tables_batch* b, int32_t* page_indptr, int32_t* page_ids, int64_t pages,
                    int32_t* positions, int64_t* slots, int32_t* items, int64_t rows, void* stream) {
    clear_error();
    if (const sangam_status s = check_table(table)) return s;
    if (!b || b->num_items < 0 || b->num_items > kMost || pages < 0 || pages > INT32_MAX || rows < 0 || rows > INT32_MAX)
        return fail(SANGAM_ERR_INVALID_ARG, "batch must not be NULL, nor num_items outside 0 to 2^30, nor pages and rows outside 0 to 2^31 - 1");
    if (!page_indptr || !b->q_indptr || (b->num_items > 0 && (!b->kv_len || !b->q_offset)))
        return fail(SANGAM_ERR_INVALID_ARG, "page_indptr and the batch's kv_len, q_indptr and q_offset must not be NULL");
    for (const void* p : {static_cast<const void*>(b->request), static_cast<const void*>(b->kv_len), static_cast<const void*>(b->q_indptr),
                          static_cast<const void*>(b->q_offset), static_cast<const void*>(b->q_pos), static_cast<const void*>(page_indptr),
                          static_cast<const void*>(page_ids), static_cast<const void*>(positions), static_cast<const void*>(items)})
        if (!aligned(p, 4)) return fail(SANGAM_ERR_ALIGN, "the arrays must be 4-byte aligned");
    if (!aligned(slots, 8)) return fail(SANGAM_ERR_ALIGN, "slots must be 8-byte aligned");
    BuildArgs args{table->pages, table->row_stride, table->requests, table->max_pages, b->num_items, b->request, b->kv_len, b->q_indptr,
                   b->q_offset, b->q_pos, page_indptr, page_ids, page_ids ? pages : 0, positions, slots, items,
                   positions || slots || items ? rows : 0};
    void* kargs[] = {&args};
    const int64_t most = std::max<int64_t>({args.num_pages, args.rows, 1});
    const unsigned groups = unsigned(std::min<int64_t>((most + kBuildThreads - 1) / kBuildThreads, 2048));
    const bool small = b->num_items <= kItemsInLds;
    if (!small) {
        const sangam_status s = launched(hipLaunchKernel(reinterpret_cast<const void*>(&tables_offsets_kernel), dim3(1), dim3(kBuildThreads),
                                                         kargs, 0, static_cast<hipStream_t>(stream)), "table");
        if (s) return s;
    }
    const void* fn = small ? reinterpret_cast<const void*>(&tables_build_kernel<true>) : reinterpret_cast<const void*>(&tables_build_kernel<false>);
    return launched(hipLaunchKernel(fn, dim3(groups), dim3(kBuildThreads), kargs, 0, static_cast<hipStream_t>(stream)), "table");
}

}  // namespace

extern "C" sangam_status sangam_tables_resize(const sangam_block_table* table, int32_t* held, const int32_t* lengths, int32_t* free_pages,
                                              int32_t free_cap, int32_t* num_free, int32_t* short_of, void* stream) {
    return entry([&] { return resize(table, held, lengths, free_pages, free_cap, num_free, short_of, stream); });
}

extern "C" sangam_status sangam_tables_build(const sangam_block_table* table, const sangam_tables_batch* batch, int32_t* page_indptr,
                                             int32_t* page_ids, int64_t pages, int32_t* positions, int64_t* slots, int32_t* items,
                                             int64_t rows, void* stream) {
    return entry([&] { return build(table, batch, page_indptr, page_ids, pages, positions, slots, items, rows, stream); });
}
