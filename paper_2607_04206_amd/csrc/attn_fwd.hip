// gfx950 kernels of the mixed block-decode / prefill attention call and the
// C-ABI forward entry point that launches them.
//
// What is computed (Sangam paper, Sec. 2.1 and Sec. 2.2): dLLM attention is
// bidirectional, so each query row of an item attends to all L positions of
// its sequence; a block decode recomputes only its 32 block rows and reuses
// the request's approximately cached KV for every other position, a prefill
// brings (and writes back) its whole sequence. Batches mix both kinds
// (Sec. 4.1, Alg. 1); the KV cache is paged with 16-token pages (Sec. 5,
// Sec. 6.1).
//
// Kernels:
//   attn_tiles_kernel one work-group per plan tile: a context range of one
//                     item and KV head against up to 8 x 32 query rows; one
//                     tile per item, KV head and row block also copies the
//                     fresh K/V rows into their cache pages.
//                     Per wave: S^T = K Q^T with v_mfma_f32_32x32x16_bf16
//                     (each lane holds the scores of one query, so row max /
//                     row sum need one cross-half exchange), online softmax
//                     in the exp2 domain, P^T rounded to bf16 feeds
//                     O^T += V^T P^T directly from the score registers.
//                     K/V stream global -> LDS with global_load_lds_dwordx4
//                     into XOR-swizzled tiles (double buffered); V^T operands
//                     come from ds_read_b64_tr_b16 transposing reads. Output
//                     rows leave through LDS, whole rows per 16 lanes.
//   attn_mixed_kernel the same tiles, prefill-shaped ones and block decodes of
//                     one query head per KV head in one launch.
//   merge_kernel      combines split-context partial (O, LSE) in split order,
//                     in calls whose tiles do not do so themselves.
#include <hip/hip_runtime.h>

#include <mutex>
#include <string>

#include "../../include/sangam_attn.h"
#include "attn_forward.h"
#include "attn_tile.h"
#include "mixed_order.h"
#include "nonce.h"
#include "plan_format.h"

using namespace sangam;

namespace {

template <int D, int QW, int KW, int QB, int NB, int NSTAGE, bool HEADS_ACROSS>
__global__ __launch_bounds__(64 * QW * KW, waves_per_simd(QB, few_registers(D, QW, HEADS_ACROSS))) void attn_tiles_kernel(AttnArgs a) {
    __shared__ TileShared<2 * NSTAGE * 32 * NB * KW * D * 2> shared;
    const TileRec t = a.tiles[blockIdx.x];
    attn_tile<D, QW, KW, QB, NB, NSTAGE, HEADS_ACROSS, 0, Bf16Cache>(a, t, a.items[t.item], shared);
}

// Prefill-shaped tiles and the block decodes of one query head per KV head
// (which no prefill-shaped tile takes) in one launch, where the planner finds
// that faster than one for each (launch_each_kind): the former are bound by
// the matrix cores and the latter by HBM, so they run beside each other, one
// of each per CU as far as they last. Both are four waves and hold 64 KiB of
// LDS; two waves of a decode only stage. Prefill tiles of 256 rows (WIDE) are
// taken as two of 128 that keep their 128-key stages, so that a prefill's sums
// are those of a launch without decodes, bit for bit: K and V have one buffer
// each and take turns (with two of 64 keys each, 16 decodes beside 1819 and
// 1201 rows, 32/32 heads, take 195 us instead of 199, but the sums differ by
// 2e-3).
// Order: `round` prefill tiles (one per CU), as many decodes, then groups of
// eight blocks (one per XCD) of either kind in the ratio of what is left.
// Measured on the same batch: 231 us in two launches, 198 in this one (the order
// was taken with the 64-key halves: 194 us, all prefill tiles first 206, all
// decodes first 212, no first round 197).
struct MixedArgs {
    AttnArgs a;                   // tiles: the prefill-shaped ones
    const TileRec* decode_tiles;
    MixedOrder order;
};

template <int D, bool WIDE>
__global__ __launch_bounds__(256, 2) void attn_mixed_kernel(MixedArgs m) {
    __shared__ TileShared<2 * 2 * 64 * D * 2> shared;
    const MixedBlock b = mixed_block(m.order, blockIdx.x);
    if (b.index < 0) return;
    if (b.decode) {
        const TileRec t = m.decode_tiles[b.index];
        attn_tile<D, 1, 2, 1, 1, 2, true, 2, Bf16Cache>(m.a, t, m.a.items[t.item], shared);
        return;
    }
    TileRec t = m.a.tiles[WIDE ? b.index >> 1 : b.index];
    const ItemRec it = m.a.items[t.item];
    if (WIDE) t.row0 += kPrefillRows * (b.index & 1);
    if (t.row0 < it.n) attn_tile<D, 4, 1, 1, WIDE ? 4 : 2, WIDE ? 1 : 2, false, 0, Bf16Cache>(m.a, t, it, shared);
}

// --------------------------------------------------------------- split merge
struct MergeArgs {
    const MergeRow* rows;
    const ItemRec* items;
    const float* ws;
    uint16_t* out;
    float* lse;
    int32_t hq;
    int32_t d;
};

// grid: (merge row, 256-element slice of the row's Hq x D/4 float4 outputs);
// one thread per float4 of one head, so that every partial of a row is
// loaded by a different thread in parallel.
__global__ __launch_bounds__(256) void merge_kernel(MergeArgs a) {
    const MergeRow mr = a.rows[blockIdx.x];
    const ItemRec it = a.items[mr.item];
    const int S = it.num_splits;
    const int d4n = a.d / 4;
    const int e = blockIdx.y * 256 + threadIdx.x;
    if (e >= a.hq * d4n) return;
    const int head = e / d4n;
    const int d4 = e - head * d4n;
    float mx = -INFINITY;
    for (int s = 0; s < S; ++s) mx = fmaxf(mx, a.ws[it.ws_lse + (size_t)(s * it.n + mr.row) * a.hq + head]);
    float tot = 0.0f;
    float4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < S; ++s) {
        const size_t prow = (size_t)(s * it.n + mr.row) * a.hq + head;
        const float w = __expf(a.ws[it.ws_lse + prow] - mx);
        const float4 v = *(const float4*)(a.ws + it.ws_o + prow * a.d + 4 * d4);
        tot += w;
        acc.x += w * v.x;
        acc.y += w * v.y;
        acc.z += w * v.z;
        acc.w += w * v.w;
    }
    const float inv = 1.0f / tot;
    const bf16x4 v = {(__bf16)(acc.x * inv), (__bf16)(acc.y * inv), (__bf16)(acc.z * inv), (__bf16)(acc.w * inv)};
    const size_t orow = (size_t)(it.q_start + mr.row) * a.hq + head;
    *(u32x2*)(a.out + orow * a.d + 4 * d4) = __builtin_bit_cast(u32x2, v);
    if (d4 == 0 && a.lse) a.lse[orow] = mx + logf(tot);
}

// ------------------------------------------------------------------ launch
template <int D, int QW, int KW, int QB, int NB, bool HA, int NSTAGE = 2>
hipError_t launch_tiles(const AttnArgs& args, int n_tiles, hipStream_t stream, LaunchEvents ev) {
    return launch(reinterpret_cast<const void*>(&attn_tiles_kernel<D, QW, KW, QB, NB, NSTAGE, HA>),
                  dim3(unsigned(n_tiles)), unsigned(64 * QW * KW), args, stream, ev);
}

template <int D>
hipError_t launch_decode(const AttnArgs& args, int n_tiles, int qw, int kw, int nb, hipStream_t stream,
                         LaunchEvents ev, bool* supported) {
    *supported = true;
    if (qw == 1 && kw == 2 && nb == 1) return launch_tiles<D, 1, 2, 1, 1, true>(args, n_tiles, stream, ev);
    if (qw == 2 && kw == 2 && nb == 2) return launch_tiles<D, 2, 2, 1, 2, true>(args, n_tiles, stream, ev);
    if (kw == 1 && nb == 2) {
        switch (qw) {
            case 3: return launch_tiles<D, 3, 1, 1, 2, true>(args, n_tiles, stream, ev);
            case 4: return launch_tiles<D, 4, 1, 1, 2, true>(args, n_tiles, stream, ev);
            case 5: return launch_tiles<D, 5, 1, 1, 2, true>(args, n_tiles, stream, ev);
            case 6: return launch_tiles<D, 6, 1, 1, 2, true>(args, n_tiles, stream, ev);
            case 7: return launch_tiles<D, 7, 1, 1, 2, true>(args, n_tiles, stream, ev);
            case 8: return launch_tiles<D, 8, 1, 1, 2, true>(args, n_tiles, stream, ev);
            default: break;
        }
    }
    *supported = false;
    return hipSuccess;
}

struct Bf16Kernels {
    typedef AttnArgs Args;

    Args args(const AttnArgs& base) const { return base; }

    hipError_t mixed(const PlanHeader& h, const Args& args, const TileRec* decodes, const MixedOrder& order,
                     unsigned blocks, hipStream_t stream, LaunchEvents ev) const {
        const void* fn = h.d == 64                             ? reinterpret_cast<const void*>(&attn_mixed_kernel<64, false>)
                         : h.prefill_rows == kWidePrefillRows ? reinterpret_cast<const void*>(&attn_mixed_kernel<128, true>)
                                                              : reinterpret_cast<const void*>(&attn_mixed_kernel<128, false>);
        return launch(fn, dim3(blocks), 256u, MixedArgs{args, decodes, order}, stream, ev);
    }

    hipError_t prefill(const PlanHeader& h, const Args& args, hipStream_t stream, LaunchEvents ev, bool* supported) const {
        *supported = true;
        if (h.prefill_rows == kWidePrefillRows && h.d == 128)
            return launch_tiles<128, kWidePrefillQWaves, 1, 1, 4, false>(args, h.n_prefill_tiles, stream, ev);
        if (h.prefill_rows == kPrefillRows)
            return h.d == 128
                       ? launch_tiles<128, kPrefillQWaves, 1, kPrefillQBlocks, 2, false>(args, h.n_prefill_tiles, stream, ev)
                       : launch_tiles<64, kPrefillQWaves, 1, kPrefillQBlocks, 2, false>(args, h.n_prefill_tiles, stream, ev);
        *supported = false;
        return hipSuccess;
    }

    hipError_t decode(const PlanHeader& h, const Args& args, hipStream_t stream, LaunchEvents ev, bool* supported) const {
        return h.d == 128
                   ? launch_decode<128>(args, h.n_decode_tiles, h.decode_qw, h.decode_kw, h.decode_nb, stream, ev, supported)
                   : launch_decode<64>(args, h.n_decode_tiles, h.decode_qw, h.decode_kw, h.decode_nb, stream, ev, supported);
    }
};

}  // namespace

// ---------------------------------------------------------- allocation-free
// Split-KV partial results of sangam_attn_forward_noalloc live in this array
// instead of a caller workspace. Each GPU the library runs on holds its own
// copy for the life of the process. In host code the name is only a stand-in
// for the symbol: kernels receive the device address that hipGetSymbolAddress
// returns for the current device, cached per device below.
namespace {
// beside them the merge marks of any plan with that many bytes of partials
// (at worst 256 bytes of marks to 768 of partials: two splits of one row)
constexpr size_t kScratchMarks = kScratchBytes / 3 + 4096;
static __device__ __align__(256) uint8_t scratch[kScratchBytes + kScratchMarks];

constexpr int kMaxScratchDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_dev[kMaxScratchDevices] = {};

// the scratch array's address on the device that runs `stream`, which must
// be the current device (the symbol is resolved with that device current)
sangam_status scratch_address(hipStream_t stream, void** addr) {
    int cur = -1;
    if (hipError_t e = hipGetDevice(&cur); e != hipSuccess) return hip_fail(e, "hipGetDevice");
    if (stream) {
        hipDevice_t sd = -1;
        if (hipError_t e = hipStreamGetDevice(stream, &sd); e != hipSuccess) return hip_fail(e, "hipStreamGetDevice");
        if (int(sd) != cur) {
            set_error("the stream belongs to device " + std::to_string(int(sd)) + ", the current device is " +
                      std::to_string(cur));
            return SANGAM_ERR_INVALID_ARG;
        }
    }
    if (cur < 0 || cur >= kMaxScratchDevices) {
        set_error("device ordinal " + std::to_string(cur) + " beyond the scratch table");
        return SANGAM_ERR_UNSUPPORTED;
    }
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_dev[cur]) {
        void* p = nullptr;
        if (hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)); e != hipSuccess)
            return hip_fail(e, "hipGetSymbolAddress(scratch)");
        g_scratch_dev[cur] = p;
    }
    *addr = g_scratch_dev[cur];
    return SANGAM_OK;
}
}  // namespace

hipError_t sangam::launch_merge(const PlanHeader& h, const uint8_t* plan_dev, const float* ws, uint16_t* out, float* lse,
                                hipStream_t stream, LaunchEvents ev) {
    const MergeArgs m{reinterpret_cast<const MergeRow*>(plan_dev + h.off_merge),
                      reinterpret_cast<const ItemRec*>(plan_dev + h.off_items),
                      ws,
                      out,
                      lse,
                      h.hq,
                      h.d};
    const unsigned slices = unsigned((h.hq * (h.d / 4) + 255) / 256);
    return launch(reinterpret_cast<const void*>(&merge_kernel), dim3(unsigned(h.n_merge_rows), slices), 256u, m, stream, ev);
}

extern "C" sangam_status sangam_attn_forward(const void* plan_host, const void* plan_dev, const void* q,
                                             const void* k_new, const void* v_new, void* k_cache,
                                             void* v_cache, int64_t pool_pages, const int32_t* page_ids_dev,
                                             int64_t num_page_ids, void* out, float* lse, void* workspace,
                                             size_t workspace_bytes, void* stream) {
    return run_forward(Bf16Kernels(),
                       ForwardTensors{plan_host, plan_dev, q, k_new, v_new, k_cache, v_cache, pool_pages, page_ids_dev,
                                      num_page_ids, out, lse, workspace, workspace_bytes, stream, nullptr},
                       own_workspace);
}

extern "C" size_t sangam_noalloc_scratch_bytes(void) { return kScratchBytes; }

extern "C" sangam_status sangam_attn_forward_noalloc(const void* plan_host, const void* plan_dev, const void* q,
                                                     const void* k_new, const void* v_new, void* k_cache,
                                                     void* v_cache, int64_t pool_pages,
                                                     const int32_t* page_ids_dev, int64_t num_page_ids,
                                                     void* out, float* lse, void* stream) {
    // split partials go to the scratch array
    auto scratch = [stream](const PlanHeader& h, void** workspace, size_t* bytes) {
        if (size_t(h.workspace_bytes - h.mark_bytes) > kScratchBytes || size_t(h.mark_bytes) > kScratchMarks) {
            set_error("the plan's split partials need " + std::to_string(h.workspace_bytes - h.mark_bytes) +
                      " bytes; the allocation-free forward holds " + std::to_string(kScratchBytes));
            return sangam_status(SANGAM_ERR_BUFFER);
        }
        *bytes = kScratchBytes + kScratchMarks;
        return scratch_address(static_cast<hipStream_t>(stream), workspace);
    };
    return run_forward(Bf16Kernels(),
                       ForwardTensors{plan_host, plan_dev, q, k_new, v_new, k_cache, v_cache, pool_pages, page_ids_dev,
                                      num_page_ids, out, lse, nullptr, 0, stream, nullptr},
                       scratch);
}

extern "C" sangam_status sangam_attn_forward_timed(const void* plan_host, const void* plan_dev,
                                                   const void* q, const void* k_new, const void* v_new,
                                                   void* k_cache, void* v_cache, int64_t pool_pages,
                                                   const int32_t* page_ids_dev, int64_t num_page_ids,
                                                   void* out, float* lse, void* workspace,
                                                   size_t workspace_bytes, void* stream, void* const* events) {
    clear_error();
    if (!events) {
        set_error("events must not be NULL");
        return SANGAM_ERR_INVALID_ARG;
    }
    return run_forward(Bf16Kernels(),
                       ForwardTensors{plan_host, plan_dev, q, k_new, v_new, k_cache, v_cache, pool_pages, page_ids_dev,
                                      num_page_ids, out, lse, workspace, workspace_bytes, stream, events},
                       own_workspace);
}
