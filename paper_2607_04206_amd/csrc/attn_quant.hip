// gfx950 kernels of the attention call over a quantised KV cache and their C
// ABI entry point (include/sangam_kvq.h).
//
// The call, its plans and its tiles are those of attn_fwd.hip (attn_tile in
// attn_tile.h); what differs is how a cached page gets into a product. With
// several query heads on a KV head, a code that each wave converted for itself
// would be converted once per head: a lane loads whole blocks (32 codes and
// their scale) of the next stage into registers while the present stage is
// computed, converts them and writes the bf16 values, which are exact, into the
// tile in LDS that all waves read. With one query head each wave streams keys of
// its own through its registers, without barriers. Fresh rows pass unquantised,
// and the tiles that write them back quantise them on the way.
#include <hip/hip_runtime.h>

#include "../../include/sangam_kvq.h"
#include "attn_forward.h"
#include "attn_tile.h"
#include "entry.h"
#include "mixed_order.h"
#include "plan_format.h"
#include "xcd_order.h"

using namespace sangam;

namespace {

// LDS of a tile: its stage buffers, or V tiles and page ids where waves are on
// their own, and, later, the sums of those that share a context
constexpr int tile_bytes(int d, int qw, int kw, int nb, int nstage, bool across) {
    const bool solo = qw == 1 && across;
    const int stages = solo ? kw * 32 * d * 2 + kMaxCachedRange / 16 * 8 : 2 * nstage * 32 * nb * kw * d * 2;
    const int sums = kw > 1 ? qw * kw * (d / 2 + 2) * 64 * 4 : 0;
    return stages > sums ? stages : sums;
}

// Waves per SIMD that the registers leave room for: three at head dim 64, where
// tiles of two and three heads would spill. 24 decodes beside three prefills of
// 32/8 heads of 64, with two -> three: e4m3 77.5 -> 70.6 us, e2m1 74.5 -> 67.1.
constexpr int waves(int d, int qw) { return d == 64 && qw != 2 && qw != 3 ? 3 : 2; }

// deal: 0, or the number of CUs, where all of a launch's tiles, longest first,
// are on the chip at once, several to a CU: every other round of one per CU is
// dealt out backwards, so that the CUs with the longest tiles of one get the
// shortest of the next (32 MHA decodes of up to 1151 keys 51.2 -> 49.1 us).
template <typename Fmt, int D, int QW, int KW, int QB, int NB, int NSTAGE, bool HEADS_ACROSS, int HELP>
__global__ __launch_bounds__(64 * (QW * KW + HELP), waves(D, QW)) void attn_quant_kernel(QuantArgs a, uint32_t deal) {
    __shared__ TileShared<tile_bytes(D, QW, KW, NB, NSTAGE, HEADS_ACROSS)> shared;
    uint32_t b = blockIdx.x;
    if (QW == 1 && deal > 0) {
        const uint32_t round = b / deal;
        if ((round & 1) && (round + 1) * deal <= gridDim.x) b = (2 * round + 1) * deal - 1 - b;
    }
    const TileRec t = a.tiles[b];
    attn_tile<D, QW, KW, QB, NB, NSTAGE, HEADS_ACROSS, HELP, QuantCache<Fmt>>(a, t, a.items[t.item], shared);
}

// Prefill-shaped tiles and MHA block decodes in one launch, as
// attn_mixed_kernel; tiles of 256 rows are taken as two of 128. At head dim 128
// all four waves take a decode's keys (16 decodes beside 1819 and 1201 rows 169
// us, with two of them 174), a block ahead (two do not fit the registers).
struct MixedQuantArgs {
    QuantArgs a;  // tiles: the prefill-shaped ones
    const TileRec* decode_tiles;
    MixedOrder order;
    int32_t wide;
    int32_t round;       // prefill blocks on the chip at a time: one per CU
    int32_t plan_chunk;  // xcd_plan_chunk of the plan's prefill tiles
};

template <typename Fmt, int D>
__global__ __launch_bounds__(256, waves(D, 4)) void attn_quant_mixed_kernel(MixedQuantArgs m) {
    constexpr int KW = D == 128 ? 4 : 2;
    constexpr int PREFILL = tile_bytes(D, 4, 1, 2, 2, false), DECODE = tile_bytes(D, 1, KW, 1, 1, true);
    __shared__ TileShared<(PREFILL > DECODE ? PREFILL : DECODE)> shared;
    const MixedBlock b = mixed_block(m.order, blockIdx.x);
    if (b.index < 0) return;
    if (b.decode) {
        const TileRec t = m.decode_tiles[b.index];
        attn_tile<D, 1, KW, 1, 1, 1, true, 4 - KW, QuantCache<Fmt>>(m.a, t, m.a.items[t.item], shared);
        return;
    }
    // Each XCD has consecutive blocks of every round (16 decodes beside prefills
    // of 1819 and 1201 rows, 32/32 heads, 177 -> 170.5 us; 8 beside 2500 rows 150
    // -> 145; smaller batches within 1 %).
    const XcdTile x = xcd_mixed_tile(b.index, m.order.n_prefill, m.wide, m.round, m.plan_chunk);
    TileRec t = m.a.tiles[x.tile];
    const ItemRec it = m.a.items[t.item];
    t.row0 += kPrefillRows * x.half;
    if (t.row0 < it.n) attn_tile<D, 4, 1, 1, 2, 2, false, 0, QuantCache<Fmt>>(m.a, t, it, shared);
}

template <typename Fmt>
struct QuantKernels {
    typedef QuantArgs Args;
    uint8_t *k_scale, *v_scale;

    Args args(const AttnArgs& base) const {
        Args a;
        static_cast<AttnArgs&>(a) = base;
        a.k_scale = k_scale;
        a.v_scale = v_scale;
        return a;
    }

    template <int D, int QW, int KW, int QB, int NB, bool HA, int NSTAGE = 2, int HELP = 0>
    static hipError_t tiles(const Args& args, int n_tiles, hipStream_t stream, LaunchEvents ev, uint32_t deal = 0) {
        void* kargs[] = {const_cast<Args*>(&args), &deal};
        return launch_args(reinterpret_cast<const void*>(&attn_quant_kernel<Fmt, D, QW, KW, QB, NB, NSTAGE, HA, HELP>),
                           dim3(unsigned(n_tiles)), unsigned(64 * (QW * KW + HELP)), kargs, stream, ev);
    }

    hipError_t mixed(const PlanHeader& h, const Args& args, const TileRec* decodes, const MixedOrder& order,
                     unsigned blocks, hipStream_t stream, LaunchEvents ev) const {
        const void* fn = h.d == 64 ? reinterpret_cast<const void*>(&attn_quant_mixed_kernel<Fmt, 64>)
                                   : reinterpret_cast<const void*>(&attn_quant_mixed_kernel<Fmt, 128>);
        const int cus = h.cus > 0 ? h.cus : 256;
        return launch(fn, dim3(blocks), 256u,
                      MixedQuantArgs{args, decodes, order, h.prefill_rows == kWidePrefillRows, cus, xcd_plan_chunk(h.n_prefill_tiles, h.prefill_rows, cus)},
                      stream, ev);
    }

    hipError_t prefill(const PlanHeader& h, const Args& args, hipStream_t stream, LaunchEvents ev, bool* supported) const {
        *supported = true;
        if (h.prefill_rows == kWidePrefillRows && h.d == 128)
            return tiles<128, kWidePrefillQWaves, 1, 1, 4, false>(args, h.n_prefill_tiles, stream, ev);
        if (h.prefill_rows == kPrefillRows)
            return h.d == 128 ? tiles<128, kPrefillQWaves, 1, kPrefillQBlocks, 2, false>(args, h.n_prefill_tiles, stream, ev)
                              : tiles<64, kPrefillQWaves, 1, kPrefillQBlocks, 2, false>(args, h.n_prefill_tiles, stream, ev);
        *supported = false;
        return hipSuccess;
    }

    template <int D>
    static hipError_t decode_tiles(const PlanHeader& h, const Args& args, hipStream_t stream, LaunchEvents ev, bool* supported) {
        *supported = true;
        const int n = h.n_decode_tiles, kw = h.decode_kw, nb = h.decode_nb;
        const int cus = h.cus > 0 ? h.cus : 256;
        // one query head: four work-groups to a CU at least
        if (h.decode_qw == 1 && kw == 2 && nb == 1) return tiles<D, 1, 2, 1, 1, true>(args, n, stream, ev, n <= 4 * cus ? cus : 0);
        if (h.decode_qw == 2 && kw == 2 && nb == 2) return tiles<D, 2, 2, 1, 2, true, 1>(args, n, stream, ev);
        if (kw == 1 && nb == 2) {
            // Two or three waves more, which only stage, where five or six heads
            // leave that many places of a CU's eight: 64 decodes of 20/4 heads
            // e4m3 67.5 -> 61.0 us, e2m1 67.4 -> 59.7, of 24/4 68.5 -> 67.3 and 68.7
            // -> 63.5. One more cannot keep up with seven heads (48 decodes of
            // 28/4 44.8 -> 49.8 us) or three (73.4 -> 83.3). At head dim 64 a CU
            // holds more work-groups instead.
            constexpr bool H = D == 128;
            switch (h.decode_qw) {
                case 3: return tiles<D, 3, 1, 1, 2, true>(args, n, stream, ev);
                case 4: return tiles<D, 4, 1, 1, 2, true>(args, n, stream, ev);
                case 5: return tiles<D, 5, 1, 1, 2, true, 2, H ? 3 : 0>(args, n, stream, ev);
                case 6: return tiles<D, 6, 1, 1, 2, true, 2, H ? 2 : 0>(args, n, stream, ev);
                case 7: return tiles<D, 7, 1, 1, 2, true>(args, n, stream, ev);
                case 8: return tiles<D, 8, 1, 1, 2, true>(args, n, stream, ev);
                default: break;
            }
        }
        *supported = false;
        return hipSuccess;
    }

    hipError_t decode(const PlanHeader& h, const Args& args, hipStream_t stream, LaunchEvents ev, bool* supported) const {
        return h.d == 128 ? decode_tiles<128>(h, args, stream, ev, supported) : decode_tiles<64>(h, args, stream, ev, supported);
    }
};

template <typename Fmt>
sangam_status run_quant(const sangam_kvq_cache& cache, const ForwardTensors& c) {
    return run_forward(QuantKernels<Fmt>{static_cast<uint8_t*>(cache.k_scale), static_cast<uint8_t*>(cache.v_scale)}, c, own_workspace);
}

}  // namespace

extern "C" sangam_status sangam_kvq_forward(const void* plan_host, const void* plan_dev, const void* q, const void* k_new,
                                            const void* v_new, const sangam_kvq_cache* cache, const int32_t* page_ids_dev,
                                            int64_t num_page_ids, void* out, float* lse, void* workspace,
                                            size_t workspace_bytes, void* stream, void* const* events) {
    return entry([&]() -> sangam_status {
        clear_error();
        if (!cache || !cache->k_scale || !cache->v_scale) {
            set_error("the cache and its scales must not be NULL");
            return SANGAM_ERR_INVALID_ARG;
        }
        if (!aligned16(cache->k_scale) || !aligned16(cache->v_scale)) {
            set_error("the cache's scales must be 16-byte aligned");
            return SANGAM_ERR_ALIGN;
        }
        const ForwardTensors c{plan_host, plan_dev, q, k_new, v_new, cache->k, cache->v, cache->pool_pages, page_ids_dev,
                               num_page_ids, out, lse, workspace, workspace_bytes, stream, events};
        if (cache->format == SANGAM_KV_E4M3) return run_quant<MxE4m3>(*cache, c);
        if (cache->format == SANGAM_KV_E2M1) return run_quant<MxE2m1>(*cache, c);
        set_error("cache format must be SANGAM_KV_E4M3 or SANGAM_KV_E2M1");
        return SANGAM_ERR_UNSUPPORTED;
    });
}
