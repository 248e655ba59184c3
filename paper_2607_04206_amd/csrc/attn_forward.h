// The host side of the attention call, shared by its entry points over a bf16
// cache (attn_fwd.hip) and over a quantised one (attn_quant.hip): checks of the
// arguments, then the launches that the plan asks for.
#pragma once

#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <string>

#include "../../include/sangam_attn.h"
#include "attn_tile.h"
#include "mixed_order.h"
#include "nonce.h"
#include "plan_format.h"

namespace sangam {
void set_error(const std::string& msg);
void clear_error();
const PlanHeader* check_plan(const void* plan);

// Start / stop events attached to one launch (timed entry point), or none.
struct LaunchEvents {
    hipEvent_t start = nullptr;
    hipEvent_t stop = nullptr;
};

// A launch with events carries them in its dispatch (hipExtLaunchKernel), so
// their timestamps bracket the kernel itself, as a kernel trace does.
inline hipError_t launch_args(const void* fn, dim3 grid, unsigned threads, void** kargs, hipStream_t stream, LaunchEvents ev) {
    if (!ev.start && !ev.stop) return hipLaunchKernel(fn, grid, dim3(threads), kargs, 0, stream);
    return hipExtLaunchKernel(fn, grid, dim3(threads), kargs, 0, stream, ev.start, ev.stop, 0);
}
template <typename Args>
hipError_t launch(const void* fn, dim3 grid, unsigned threads, Args args, hipStream_t stream, LaunchEvents ev) {
    void* kargs[] = {&args};
    return launch_args(fn, grid, threads, kargs, stream, ev);
}

// The split merge of a call whose tiles do not merge (attn_fwd.hip).
hipError_t launch_merge(const PlanHeader& h, const uint8_t* plan_dev, const float* ws, uint16_t* out, float* lse,
                        hipStream_t stream, LaunchEvents ev);

inline sangam_status hip_fail(hipError_t e, const char* what) {
    set_error(std::string(what) + ": " + hipGetErrorString(e));
    return SANGAM_ERR_HIP;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The tensors of a call, as its entry point got them.
struct ForwardTensors {
    const void *plan_host, *plan_dev, *q, *k_new, *v_new;
    void *k_cache, *v_cache;
    int64_t pool_pages;
    const int32_t* page_ids_dev;
    int64_t num_page_ids;
    void* out;
    float* lse;
    void* workspace;
    size_t workspace_bytes;
    void* stream;
    void* const* events;
};

// One call on `Kernels`, which launches the kernels of its cache:
//   Kernels::Args                  their arguments: AttnArgs and what else they take
//   args(base)                     those, from an AttnArgs
//   mixed(h, args, decodes, order, blocks, stream, ev)
//   prefill(h, args, stream, ev, &supported), decode(h, args, stream, ev, &supported)
// `scratch(h, &workspace, &bytes)` may put another workspace in the place of the caller's.
template <typename Kernels, typename Scratch>
sangam_status run_forward(const Kernels& kernels, const ForwardTensors& c, const Scratch& scratch) {
    clear_error();
    const PlanHeader* h = check_plan(c.plan_host);
    if (!h) {
        set_error("plan_host is not a plan of this library version");
        return SANGAM_ERR_PLAN;
    }
    if (!c.plan_dev || !c.q || !c.k_new || !c.v_new || !c.k_cache || !c.v_cache || !c.page_ids_dev || !c.out) {
        set_error("plan_dev, q, k_new, v_new, k_cache, v_cache, page_ids_dev and out must not be NULL");
        return SANGAM_ERR_INVALID_ARG;
    }
    if (!aligned16(c.plan_dev) || !aligned16(c.q) || !aligned16(c.k_new) || !aligned16(c.v_new) ||
        !aligned16(c.k_cache) || !aligned16(c.v_cache) || !aligned16(c.out) ||
        (reinterpret_cast<uintptr_t>(c.page_ids_dev) & 3u) || (c.lse && (reinterpret_cast<uintptr_t>(c.lse) & 3u))) {
        set_error("tensors must be 16-byte aligned (page_ids and lse 4-byte aligned)");
        return SANGAM_ERR_ALIGN;
    }
    if (c.pool_pages < h->num_pool_pages) {
        set_error("the plan addresses " + std::to_string(h->num_pool_pages) + " pool pages, the cache holds " +
                  std::to_string(c.pool_pages));
        return SANGAM_ERR_BUFFER;
    }
    if (c.num_page_ids < h->total_pages) {
        set_error("the plan reads " + std::to_string(h->total_pages) + " page ids, page_ids_dev holds " +
                  std::to_string(c.num_page_ids));
        return SANGAM_ERR_BUFFER;
    }
    void* workspace = c.workspace;
    size_t workspace_bytes = c.workspace_bytes;
    if (h->workspace_bytes > 0) {
        if (sangam_status st = scratch(*h, &workspace, &workspace_bytes); st != SANGAM_OK) return st;
        if (!workspace || workspace_bytes < size_t(h->workspace_bytes)) {
            set_error("workspace needs " + std::to_string(h->workspace_bytes) + " bytes");
            return SANGAM_ERR_BUFFER;
        }
        if (!aligned16(workspace)) {
            set_error("workspace must be 16-byte aligned");
            return SANGAM_ERR_ALIGN;
        }
    }
    hipStream_t stream = static_cast<hipStream_t>(c.stream);
    const uint8_t* pd = static_cast<const uint8_t*>(c.plan_dev);
    // events[2k], events[2k+1] bracket launch k (prefill-shaped, decode-shaped,
    // merge); a launch with no work records its pair back to back
    auto evs = [&](int k) {
        LaunchEvents ev;
        if (c.events) {
            ev.start = static_cast<hipEvent_t>(c.events[2 * k]);
            ev.stop = static_cast<hipEvent_t>(c.events[2 * k + 1]);
        }
        return ev;
    };
    auto mark_empty = [&](int k) -> hipError_t {
        const LaunchEvents ev = evs(k);
        for (hipEvent_t e : {ev.start, ev.stop})
            if (e)
                if (hipError_t r = hipEventRecord(e, stream); r != hipSuccess) return r;
        return hipSuccess;
    };
    typename Kernels::Args args = kernels.args(AttnArgs{nullptr,
                                                        reinterpret_cast<const ItemRec*>(pd + h->off_items),
                                                        c.page_ids_dev,
                                                        static_cast<const uint16_t*>(c.q),
                                                        static_cast<const uint16_t*>(c.k_new),
                                                        static_cast<const uint16_t*>(c.v_new),
                                                        static_cast<uint16_t*>(c.k_cache),
                                                        static_cast<uint16_t*>(c.v_cache),
                                                        static_cast<uint16_t*>(c.out),
                                                        c.lse,
                                                        static_cast<float*>(workspace),
                                                        reinterpret_cast<const int32_t*>(pd + h->off_positions),
                                                        reinterpret_cast<const uint32_t*>(pd + h->off_page_info),
                                                        h->hq,
                                                        h->hkv,
                                                        h->scale_log2,
                                                        h->mark_bytes > 0 ? next_nonce() : 0});
    // 1. attention: prefill-shaped tiles (compute-bound) first, then
    // decode-shaped tiles; both also write the fresh rows into their pages
    const bool mixed = one_launch(*h);
    if (mixed) {
        args.tiles = reinterpret_cast<const TileRec*>(pd + h->off_prefill_tiles);
        // a block for 128 rows, wide tiles in halves; a round of one per CU
        const int64_t prefill_blocks = int64_t(h->n_prefill_tiles) << int(h->prefill_rows == kWidePrefillRows);
        MixedOrder order;
        const int64_t blocks = mixed_order(&order, prefill_blocks, h->n_decode_tiles, h->cus > 0 ? h->cus : 256);
        if (hipError_t e = kernels.mixed(*h, args, reinterpret_cast<const TileRec*>(pd + h->off_decode_tiles), order,
                                         unsigned(blocks), stream, evs(0));
            e != hipSuccess)
            return hip_fail(e, "mixed attention launch");
    } else if (h->n_prefill_tiles > 0) {
        args.tiles = reinterpret_cast<const TileRec*>(pd + h->off_prefill_tiles);
        bool ok = false;
        const hipError_t e = kernels.prefill(*h, args, stream, evs(0), &ok);
        if (!ok) {
            set_error("no prefill kernel for this tile shape");
            return SANGAM_ERR_UNSUPPORTED;
        }
        if (e != hipSuccess) return hip_fail(e, "prefill attention launch");
    } else if (hipError_t e = mark_empty(0); e != hipSuccess) {
        return hip_fail(e, "event record");
    }
    if (!mixed && h->n_decode_tiles > 0) {
        args.tiles = reinterpret_cast<const TileRec*>(pd + h->off_decode_tiles);
        bool ok = false;
        const hipError_t e = kernels.decode(*h, args, stream, evs(1), &ok);
        if (!ok) {
            set_error("no decode kernel for this head grouping");
            return SANGAM_ERR_UNSUPPORTED;
        }
        if (e != hipSuccess) return hip_fail(e, "decode attention launch");
    } else if (hipError_t e = mark_empty(1); e != hipSuccess) {
        return hip_fail(e, "event record");
    }

    // 2. merge split contexts, unless the tiles do
    if (merge_launch(*h)) {
        const hipError_t e = launch_merge(*h, pd, static_cast<const float*>(workspace), static_cast<uint16_t*>(c.out),
                                          c.lse, stream, evs(2));
        if (e != hipSuccess) return hip_fail(e, "merge launch");
    } else if (hipError_t e = mark_empty(2); e != hipSuccess) {
        return hip_fail(e, "event record");
    }
    return SANGAM_OK;
}

// The caller's workspace.
inline sangam_status own_workspace(const PlanHeader&, void**, size_t*) { return SANGAM_OK; }

}  // namespace sangam
