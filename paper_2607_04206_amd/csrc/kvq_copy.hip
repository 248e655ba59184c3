// Export and import of quantised KV pages for gfx950 and their C ABI entry
// points (include/sangam_kvq.h): pages of codes and scale bytes to packed bf16
// rows, and back.
//
// As kv_copy_kernel: one work-group per (listed page, 256 / (2 D) heads,
// tensor). A thread moves one piece of 8 values, 16 bytes on the packed side
// and 8 (e4m3) or 4 (e2m1) on the pool side; four neighbouring lanes hold a
// block, so that both sides' accesses are whole rows and whole chunks of a
// page, and the import finds the block's largest magnitude with two exchanges
// inside the quad. Bound by HBM: a hand-off of 304 MB (packed) through e4m3 pages
// 163 us, 5.7 TB/s of a streaming read's 5.83, one of 91 MB through e2m1 pages 48
// (4.8 TB/s); large exports, four fifths of whose bytes are written, by its
// write rate (3.8 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "../../include/sangam_kvq.h"
#include "entry.h"
#include "kv_format.h"
#include "mx_format.h"

namespace sangam {
void set_error(const std::string& msg);
void clear_error();
const KvPlanHeader* check_kv_plan(const void* plan);
}  // namespace sangam

using namespace sangam;

namespace {

struct KvqCopyArgs {
    const KvPageRec* recs;
    uint8_t* codes[2];   // K, V
    uint8_t* scales[2];
    uint16_t* packed[2];
    int32_t hkv;
    uint32_t groups;  // head groups of a page
};

constexpr int64_t kMaxBlocks = (int64_t(1) << 32) / 256 - 1;  // a grid's threads are counted in 32 bits

// Packed bytes (K and V) from which the stores are nontemporal. Measured, import
// and export by themselves with plain -> with nontemporal stores: e4m3 65 MB
// 19.8 -> 18.0 and 20.6 -> 15.5 us, 304 MB 87.1 -> 83.9 and 87.4 -> 79.9, 1408 MB
// 397 -> 372 and 417 -> 378; e2m1 65 MB 15.3 -> 15.1 and 17.1 -> 13.1, 1408 MB 344
// -> 338 and 438 -> 366. An export right behind its import, which finds less of
// the pages in the cache: e4m3 65 MB together 41.7 -> 38.8, 91 MB 51.7 -> 53.2, 304
// MB 174 -> 163. Smaller ones are left to whoever reads them next.
constexpr int64_t kStreamBytes = int64_t(32) << 20;

// the largest of a quad's values, in all four lanes
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    x = max(x, uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0xB1, 0xF, 0xF, true)));  // lanes 1 0 3 2
    return max(x, uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0x4E, 0xF, 0xF, true)));  // lanes 2 3 0 1
}

template <bool STREAM, typename T>
__device__ __forceinline__ void put(T* p, T v) {
    if (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}

template <typename Fmt, int D, bool EXPORT, bool STREAM>
__global__ __launch_bounds__(256) void kvq_copy_kernel(KvqCopyArgs a) {
    constexpr int NC = D / 8;             // pieces of a row
    constexpr int HPG = 256 / (16 * NC);  // heads of a work-group
    const uint32_t page = blockIdx.x / a.groups;
    const KvPageRec r = a.recs[page];
    const int t = blockIdx.y;
    const int tid = threadIdx.x;
    const int pos = tid % NC;
    const int s = (tid / NC) % 16;
    const int h = int(blockIdx.x - page * a.groups) * HPG + tid / (16 * NC);
    if (s >= r.nslots || h >= a.hkv) return;  // whole quads: a row's pieces
    const size_t row = ((size_t)r.page * a.hkv + h) * 16 + s;  // of the pool
    const size_t piece = row * NC + pos;
    const size_t block = piece / 4;
    mx_u32x4* const packed = (mx_u32x4*)(a.packed[t] + ((size_t)(r.row0 + s) * a.hkv + h) * D + pos * 8);
    uint32_t* const code = reinterpret_cast<uint32_t*>(a.codes[t]) + piece * Fmt::kWords;
    uint32_t c[Fmt::kWords];
    if (EXPORT) {
#pragma unroll
        for (int w = 0; w < Fmt::kWords; ++w) c[w] = code[w];
        put<STREAM>(packed, mx_read<Fmt>(c, a.scales[t][block]));
    } else {
        const mx_u32x4 x = *packed;
        const mx_u16x2 m = mx_largest(mx_u16x2{0, 0}, x);
        const uint32_t scale = mx_scale<Fmt>(quad_max(m[0] > m[1] ? m[0] : m[1]));
        mx_write<Fmt>(c, x, scale);
#pragma unroll
        for (int w = 0; w < Fmt::kWords; ++w) put<STREAM>(code + w, c[w]);
        if (pos % 4 == 0) a.scales[t][block] = uint8_t(scale);
    }
}

template <typename Fmt, int D>
const void* copy_fn(bool is_export, bool stream) {
    if (is_export)
        return stream ? reinterpret_cast<const void*>(&kvq_copy_kernel<Fmt, D, true, true>)
                      : reinterpret_cast<const void*>(&kvq_copy_kernel<Fmt, D, true, false>);
    return stream ? reinterpret_cast<const void*>(&kvq_copy_kernel<Fmt, D, false, true>)
                  : reinterpret_cast<const void*>(&kvq_copy_kernel<Fmt, D, false, false>);
}
template <typename Fmt>
const void* copy_fn(int d, bool is_export, bool stream) {
    return d == 128 ? copy_fn<Fmt, 128>(is_export, stream) : copy_fn<Fmt, 64>(is_export, stream);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

sangam_status fail(sangam_status code, const std::string& msg) {
    set_error(msg);
    return code;
}

sangam_status run_copy(bool is_export, const void* plan_host, const void* plan_dev, const sangam_kvq_cache* cache,
                       const void* k_packed, const void* v_packed, void* stream) {
    clear_error();
    const KvPlanHeader* h = check_kv_plan(plan_host);
    if (!h) return fail(SANGAM_ERR_PLAN, "plan_host is not a KV transfer plan of this library version");
    if (!cache || !plan_dev || !k_packed || !v_packed || !cache->k || !cache->v || !cache->k_scale || !cache->v_scale)
        return fail(SANGAM_ERR_INVALID_ARG, "plan_dev, the cache, its arrays and the packed buffers must not be NULL");
    if (cache->format != SANGAM_KV_E4M3 && cache->format != SANGAM_KV_E2M1)
        return fail(SANGAM_ERR_UNSUPPORTED, "cache format must be SANGAM_KV_E4M3 or SANGAM_KV_E2M1");
    for (const void* p : {plan_dev, k_packed, v_packed, static_cast<const void*>(cache->k), static_cast<const void*>(cache->v),
                          static_cast<const void*>(cache->k_scale), static_cast<const void*>(cache->v_scale)})
        if (!aligned16(p)) return fail(SANGAM_ERR_ALIGN, "plan_dev, the cache's arrays and the packed buffers must be 16-byte aligned");
    if (cache->pool_pages < h->num_pool_pages)
        return fail(SANGAM_ERR_BUFFER, "the plan addresses " + std::to_string(h->num_pool_pages) + " pool pages, the cache holds " +
                                           std::to_string(cache->pool_pages));
    KvqCopyArgs args;
    const KvPageRec* recs = reinterpret_cast<const KvPageRec*>(static_cast<const uint8_t*>(plan_dev) + h->off_pages);
    args.codes[0] = static_cast<uint8_t*>(cache->k);
    args.codes[1] = static_cast<uint8_t*>(cache->v);
    args.scales[0] = static_cast<uint8_t*>(cache->k_scale);
    args.scales[1] = static_cast<uint8_t*>(cache->v_scale);
    args.packed[0] = static_cast<uint16_t*>(const_cast<void*>(k_packed));  // (an import only reads them)
    args.packed[1] = static_cast<uint16_t*>(const_cast<void*>(v_packed));
    args.hkv = h->hkv;
    const int heads = 256 / (2 * h->d);  // of a work-group
    args.groups = uint32_t((h->hkv + heads - 1) / heads);
    const bool nt = h->total_rows * h->hkv * h->d * 4 > kStreamBytes;
    const void* fn = cache->format == SANGAM_KV_E4M3 ? copy_fn<MxE4m3>(h->d, is_export, nt) : copy_fn<MxE2m1>(h->d, is_export, nt);
    void* kargs[] = {&args};
    const int64_t step = std::max<int64_t>(kMaxBlocks / args.groups, 1);  // pages of a launch
    for (int64_t first = 0; first < h->total_pages; first += step) {
        args.recs = recs + first;
        const int64_t pages = std::min<int64_t>(step, h->total_pages - first);
        const hipError_t e = hipLaunchKernel(fn, dim3(unsigned(pages * args.groups), 2), dim3(256), kargs, 0,
                                             static_cast<hipStream_t>(stream));
        if (e != hipSuccess)
            return fail(SANGAM_ERR_HIP, std::string(is_export ? "quantised kv export" : "quantised kv import") + " launch: " + hipGetErrorString(e));
    }
    return SANGAM_OK;
}

}  // namespace

extern "C" sangam_status sangam_kvq_export(const void* plan_host, const void* plan_dev, const sangam_kvq_cache* cache,
                                           void* k_packed, void* v_packed, void* stream) {
    return entry([&] { return run_copy(true, plan_host, plan_dev, cache, k_packed, v_packed, stream); });
}

extern "C" sangam_status sangam_kvq_import(const void* plan_host, const void* plan_dev, const void* k_packed,
                                           const void* v_packed, const sangam_kvq_cache* cache, void* stream) {
    return entry([&] { return run_copy(false, plan_host, plan_dev, cache, k_packed, v_packed, stream); });
}
