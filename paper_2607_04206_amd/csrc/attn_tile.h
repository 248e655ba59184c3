// One tile of the attention call (a work-group's share of it), shared by the
// kernels over a bf16 cache (attn_fwd.hip) and over a quantised one
// (attn_quant.hip): the types, the asynchronous copies into LDS, and attn_tile.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "mx_format.h"
#include "plan_format.h"

using namespace sangam;

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

#define LDS __attribute__((address_space(3)))

struct AttnArgs {
    const TileRec* tiles;
    const ItemRec* items;
    const int32_t* page_ids;
    const uint16_t* q;
    const uint16_t* k_new;
    const uint16_t* v_new;
    uint16_t* k_cache;  // read (cached rows) and written (the fresh rows' pages)
    uint16_t* v_cache;
    uint16_t* out;
    float* lse;
    float* ws;
    const int32_t* positions;    // rows of per-token cached decodes (kItemPosList items)
    const uint32_t* page_info;   // per page of such items: listed slots and earlier rows
    int32_t hq;
    int32_t hkv;
    float scale_log2;
    uint64_t nonce;  // marks this call's split partials as written (0: merge_kernel merges)
};

// The same over a quantised cache: k_cache and v_cache hold codes, beside them
// a scale byte per block of 32 dims.
struct QuantArgs : AttnArgs {
    uint8_t* k_scale;
    uint8_t* v_scale;
};

// What a tile's cached rows are: bf16, copied into LDS as they are, or blocks
// of a format of mx_format.h, which pass through registers on their way.
struct Bf16Cache {
    static constexpr bool QUANT = false;
    typedef AttnArgs Args;
    struct Block {};
};
template <typename Fmt>
struct QuantCache {
    static constexpr bool QUANT = true;
    typedef QuantArgs Args;
    typedef MxBlock<Fmt> Block;
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Asynchronous copy of one K or V page (16 key rows of one head) from global
// memory into LDS by one wave: IPP global_load_lds_dwordx4, each moving 1 KiB
// (lane l's 16 bytes land at the instruction's LDS base + 16 l). The
// instruction adds its offset field to the global and to the LDS address, so
// one M0 write serves the page: instruction j lands at dst + 1024 j, and the
// lane offsets of instruction j are given less 1024 j. Issued through inline
// assembly so that the compiler does not track the LDS write: it would
// otherwise wait for every copy in flight before any later LDS read,
// including the copies that prefetch the next stage into another buffer,
// which serialises the prefetch with the compute it should overlap. The
// kernels order the copies themselves: s_waitcnt vmcnt and a barrier before a
// staged buffer is read, a barrier before it is overwritten. M0 is saved and
// restored around the copies, with the wait state the hardware needs between
// an M0 write and its use. Nor does the compiler count wait states into the
// block: a base it has just restored from a spill (v_readlane) is read five
// wait states after at the earliest, so the first copy stands behind that many.
__device__ __forceinline__ uint32_t lds_wave_base(LDS void* p) {
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)p);
}
// from a wave-uniform base plus per-lane 32-bit byte offsets
template <int IPP>
__device__ __forceinline__ void copy_page(const void* base, const uint32_t (&off)[IPP], LDS void* dst) {
    uint32_t saved;
    static_assert(IPP == 2 || IPP == 4, "a page is 2 or 4 KiB");
    if constexpr (IPP == 4)
        asm volatile(
            "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\t"
            "global_load_lds_dwordx4 %2, %6\n\tglobal_load_lds_dwordx4 %3, %6 offset:1024\n\t"
            "global_load_lds_dwordx4 %4, %6 offset:2048\n\tglobal_load_lds_dwordx4 %5, %6 offset:3072\n\t"
            "s_nop 0\n\ts_mov_b32 m0, %0"
            : "=&s"(saved)
            : "s"(lds_wave_base(dst)), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base)
            : "memory");
    else
        asm volatile(
            "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\t"
            "global_load_lds_dwordx4 %2, %4\n\tglobal_load_lds_dwordx4 %3, %4 offset:1024\n\t"
            "s_nop 0\n\ts_mov_b32 m0, %0"
            : "=&s"(saved)
            : "s"(lds_wave_base(dst)), "v"(off[0]), "v"(off[1]), "s"(base)
            : "memory");
}
// the same from per-lane addresses
template <int IPP>
__device__ __forceinline__ void copy_page(const uint64_t (&addr)[IPP], LDS void* dst) {
    uint32_t saved;
    if constexpr (IPP == 4)
        asm volatile(
            "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
            "global_load_lds_dwordx4 %2, off\n\tglobal_load_lds_dwordx4 %3, off offset:1024\n\t"
            "global_load_lds_dwordx4 %4, off offset:2048\n\tglobal_load_lds_dwordx4 %5, off offset:3072\n\t"
            "s_nop 0\n\ts_mov_b32 m0, %0"
            : "=&s"(saved)
            : "s"(lds_wave_base(dst)), "v"(addr[0]), "v"(addr[1]), "v"(addr[2]), "v"(addr[3])
            : "memory");
    else
        asm volatile(
            "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
            "global_load_lds_dwordx4 %2, off\n\tglobal_load_lds_dwordx4 %3, off offset:1024\n\t"
            "s_nop 0\n\ts_mov_b32 m0, %0"
            : "=&s"(saved)
            : "s"(lds_wave_base(dst)), "v"(addr[0]), "v"(addr[1])
            : "memory");
}

// Swizzle of 16-byte chunks inside a staged key row. K rows are read one key
// per lane (ds_read_b128), so 16 consecutive keys (4 KiB at D = 128; at
// D = 64 two keys share the 256 bytes of all banks) spread their chunks. V rows are
// read four keys at a time by ds_read_b64_tr_b16, so groups of four keys
// spread over the LDS banks.
template <int D>
__device__ __forceinline__ int swz_k(int r) {
    return D == 128 ? r & 15 : (r >> 1) & 7;
}
template <int D>
__device__ __forceinline__ int swz_v(int r) {
    return D == 128 ? ((r & 3) << 2) : (((r >> 1) & 1) << 2);
}

// Cross-half (lane l <-> l ^ 32) pair of a value: v_permlane32_swap with both
// operands x returns (x[l], x[l^32]) for the lower half and (x[l^32], x[l])
// for the upper half, so a symmetric combine of the two results is the pair's.
__device__ __forceinline__ float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// x of both halves summed in the lower one, y of both halves in the upper one,
// and such a pair's two sums in every lane.
__device__ __forceinline__ float half_sums(float x, float y) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float2 both_sums(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return float2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}

// The running max moves only when a score exceeds it by more than this (log2
// units), so P <= 2^8 and O is rescaled rarely; the result is unchanged
// because O and l always share the same reference.
constexpr float kRescaleThreshold = 8.0f;

// Split partials cross the XCDs, whose L2s are not coherent: stores write
// through to memory and loads bypass the L2 (agent scope, sc1).
// The 16-byte store's data registers may be written again two wait states after
// it at the earliest, which the compiler does not see in assembly.
__device__ __forceinline__ void store_agent(float* p, float4 v) {
    asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" ::"v"(p), "v"(__builtin_bit_cast(u32x4, v)) : "memory");
}
__device__ __forceinline__ void store_agent(float* p, float v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float load_agent(const float* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
constexpr int kBufferAgent = 16;  // sc1 in a buffer load's cache policy

// Decode tiles of five to eight query heads at head dim 64 fit twice or three
// times on a CU with 128 registers a wave (four waves per SIMD), once or twice
// with the 165 they take otherwise. They get there with fragments read two steps
// ahead instead of four and with no more splits' sums than they merge. Measured
// with 165 -> 128 registers: 100 decodes of 1500 keys, 28/4 heads, 67.5 -> 61.2
// us, 150 of 20/4 95.0 -> 75.1, 250 of 64/8 304 -> 276; launches of up to one
// work-group per CU take the same time.
constexpr bool few_registers(int d, int qw, bool heads_across) { return d == 64 && heads_across && qw >= 5; }

// Waves per SIMD the register budget is sized for: two (256 registers) when a
// wave holds one query block.
constexpr int waves_per_simd(int qb, bool few) { return few ? 4 : qb == 1 ? 2 : 1; }

// LDS of a work-group
template <int BYTES>
struct TileShared {
    __attribute__((aligned(1024))) uint8_t stages[BYTES];  // K and V stage buffers
    int32_t wpages[kWaveRows];  // pages of the fresh rows this tile writes back
    int32_t fpos[kWaveRows];    // the listed positions (kItemPosList items)
    bool merging;               // this tile merges its rows' splits
};

// One work-group per plan tile: a context range [kv_begin, kv_end) of one
// item and KV head against QW query slots x QB blocks of 32 rows per slot.
//   D      head dim (64, 128)
//   QW     waves holding distinct query rows (query heads of a GQA group when
//          HEADS_ACROSS, else consecutive 32*QB-row blocks of one head)
//   KW     waves splitting each stage's keys (merged through LDS at the end)
//   QB     32-row query blocks per wave: every K and V fragment read from
//          LDS feeds QB MFMAs, so QB = 2 halves LDS traffic per flop
//   NB     32-key blocks per wave per stage
//   NSTAGE K/V stage buffers in LDS (NSTAGE - 1 stages in flight). 1: K and V
//          have one buffer each, and K of the next stage arrives while V of
//          this one is used, V while its K is
//          (bf16; over a quantised cache the next stage waits in registers;
//          where every wave is for itself, this many blocks do)
//   HELP   more waves, which only stage and write back
//   Cache  what the cached rows are
template <int D, int QW, int KW, int QB, int NB, int NSTAGE, bool HEADS_ACROSS, int HELP, typename Cache, typename Shared>
__device__ __forceinline__ void attn_tile(const typename Cache::Args& a, const TileRec t, const ItemRec it, Shared& shared) {
    constexpr bool QUANT = Cache::QUANT;
    constexpr bool SOLO = QUANT && QW == 1 && HEADS_ACROSS;  // every wave for itself (below)
    constexpr int NT = 64 * (QW * KW + HELP);  // threads
    constexpr int KT = 32 * NB;          // keys per wave per stage
    constexpr int STEP = KT * KW;        // keys per stage
    constexpr int NC = D / 8;            // 16-byte chunks per key row
    constexpr int ROWB = D * 2;          // bytes per key row
    constexpr int TILE = STEP * ROWB;    // bytes of one staged K (or V) tile
    constexpr int NW = QW * KW + HELP;   // waves
    constexpr int SP = STEP / 16;        // 16-key pages per stage
    constexpr int PW = (SP + NW - 1) / NW;  // pages a wave copies per stage
    constexpr int RPI = 64 / NC;         // key rows per copy instruction
    constexpr int IPP = 16 / RPI;        // copy instructions per page
    constexpr int DS = D / 16;           // k-steps of the QK^T contraction
    constexpr int MB = D / 32;           // 32-dim blocks of O^T
    // MFMAs at raised wave priority: those of QK^T (1), of PV (2) or none (0).
    // Two waves share a SIMD. Measured: 128-key stages QK^T (long prefills
    // 6,510 us with PV, 6,480 with it), 64-key ones PV (Dream mixed batch 261
    // us with QK^T or none, 255 with it), D = 64 none (mixed batch 80.9 us
    // with PV, 76.4 without). Decode batches take the same time either way
    // (1 to 48 decodes, 14.8 to 78 us, within 0.2 %).
    constexpr int PRIO = D == 64 ? 0 : NB == 4 ? 1 : 2;
    constexpr bool FEW = few_registers(D, QW, HEADS_ACROSS) && !QUANT;  // (the blocks on their way take more)
    constexpr int RA = FEW ? 2 : 4;      // steps between a fragment's LDS read and its MFMA
    constexpr int MAXS = FEW ? max_merge_in_tile(QW) : kMaxMergeInTile;  // splits that a tile merges
    constexpr int MERGE_REGS = MB * 16 + 2;
    static_assert(KW == 1 || QB == 1, "context-splitting waves hold one query block");
    static_assert(!HEADS_ACROSS || QB == 1, "a decode block is 32 rows");
    static_assert(KW == 1 || (QW * KW * MERGE_REGS * 64 * 4) <= sizeof(shared.stages),
                  "cross-wave merge must fit in the stage buffers");
    static_assert(MB % KW == 0, "the waves of a query slot share its dims");
    static_assert(NSTAGE >= 1 && NSTAGE <= 4, "1 to 4 stage buffers");
    constexpr bool TURNS = NSTAGE == 1 && !QUANT;  // K and V take turns
    static_assert(!TURNS || (KW == 1 && !HEADS_ACROSS && HELP == 0), "every wave meets the barrier between K and V");
    // pages a tile's write-back can touch: its rows at any offset, or one per listed row
    static_assert((32 * QB * QW + 15) / 16 + 1 <= kWaveRows && kWaveRows <= NT, "one thread per write-back page id");
    // with more than two buffers the wait counts loads, so every wave must
    // issue the same number per stage
    static_assert(NSTAGE <= 2 || SP % NW == 0, "deeper pipelines need whole staging rounds");
    static_assert(64 % SP == 0 && (NSTAGE - 1) * SP < 64, "a stage's page ids sit in one register of 64 lanes");

    static_assert(SOLO || sizeof(shared.stages) >= 2 * NSTAGE * TILE, "the stage buffers");
    uint8_t* const smem = shared.stages;
    int32_t* const fpos = shared.fpos;
    int32_t* const wpages = shared.wpages;

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = uniform(tid >> 6);
    const bool computes = HELP == 0 || wave < QW * KW;
    const int qs = computes ? wave % QW : 0;
    const int ks = computes ? wave / QW : 0;
    const int qn = lane & 31;   // query (column) this lane holds in each block
    const int hh = lane >> 5;   // half-wave

    // heads across the waves: a decode-shaped work-group, or a block decode
    // cut into a prefill-shaped one (whose last tile of a GQA group may hold
    // fewer heads than waves: the extra waves only stage K/V, write back and
    // meet the barriers; they compute and store nothing)
    const bool across = HEADS_ACROSS || (!TURNS && (t.flags & kTileHeadsAcross));
    const int head_want = across ? t.q_head0 + qs : t.q_head0;
    const bool head_ok = computes && head_want < (t.kv_head + 1) * (a.hq / a.hkv);
    const int head = head_ok ? head_want : t.q_head0;
    const int row_base = across ? t.row0 : t.row0 + 32 * QB * qs;
    const bool split_out = it.num_splits > 1;  // fp32 partials go to the workspace
    const bool merge_here = split_out && a.nonce != 0;
    const int kv_begin = t.kv_begin, kv_end = t.kv_end;
    const int nstages = (kv_end - kv_begin + STEP - 1) / STEP;
    // a whole prefill brings every position fresh: no page lookups
    const bool all_fresh = it.o == 0 && it.n == it.L;
    // a per-token cached decode: its rows sit at listed positions
    const bool plist = (it.flags & kItemPosList) != 0;
    const int pg0 = kv_begin >> 4;
    const int npg = ((kv_end + 15) >> 4) - pg0;
    // The tile's page ids (and page_info of kItemPosList items) sit in a
    // register, 64 at a time (lane l holds entry 64 c + l of chunk c): a stage
    // reads its ids with v_readlane, with no LDS or barrier in between.
    int32_t pv = 0;
    uint32_t iv = 0;
    auto load_pages = [&](int first) {
        const int k = it.page_start + pg0 + min(first + lane, npg - 1);
        pv = a.page_ids[k];
        if (plist) iv = a.page_info[k];
    };
    if (!all_fresh) load_pages(0);
    int32_t lpos = 0;  // the listed position of row `lane`, in every wave
    if (plist) lpos = a.positions[it.pos_start + min(lane, it.n - 1)];

    // ---- Q fragments (B operand: k = dims, n = query). Lanes past the last
    // row hold row 0 again: a query is a column of every product, so they
    // change no other row, and nothing of theirs is stored.
    bf16x8 qf[QB][DS];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int row = row_base + 32 * qb + qn;
        const uint16_t* qp = a.q + ((size_t)(it.q_start + (row < it.n ? row : 0)) * a.hq + head) * D;
#pragma unroll
        for (int s = 0; s < DS; ++s) qf[qb][s] = *(const bf16x8*)(qp + (SOLO ? 8 * s + D / 2 * hh : 16 * s + 8 * hh));
    }

    // ---- staging. A stage is SP pages of 16 key rows; wave w copies pages
    // w, w + NW, ... of it, K and V, IPP instructions each. Instruction j
    // covers rows RPI j + lane / NC; the lane's chunk of LDS row r is source
    // chunk (lane % NC) ^ swizzle(r). A work-group by itself is bound by its
    // serial chain of stages, and the scalar instructions of the copies stood
    // in it (about 110 per page; now about 20): one LLaDA decode 17.3 -> 16.6
    // us, a batch of 32 75.3 -> 74.1 us.
    const size_t row_stride = (size_t)a.hkv * D;                       // elements between positions
    const uint32_t row_bytes = uint32_t(row_stride * 2);
    const uint16_t* kfresh = a.k_new + ((size_t)(it.q_start - it.o) * a.hkv + t.kv_head) * D;
    const uint16_t* vfresh = a.v_new + ((size_t)(it.q_start - it.o) * a.hkv + t.kv_head) * D;
    const size_t page_stride = (size_t)a.hkv * 16 * D;
    const uint16_t* kcache = a.k_cache + (size_t)t.kv_head * 16 * D;
    const uint16_t* vcache = a.v_cache + (size_t)t.kv_head * 16 * D;

    // byte offsets of a lane's chunks from the first row of a page, less the
    // instruction's offset field: rows ROWB apart in the cache, row_bytes
    // apart among the fresh rows (row_bytes >= ROWB, so none is negative)
    uint32_t coff_k[IPP], coff_v[IPP], foff_k[IPP], foff_v[IPP];
#pragma unroll
    for (int j = 0; j < IPP; ++j) {
        const int r = RPI * j + lane / NC, pos = lane % NC;
        const uint32_t ck = uint32_t((pos ^ swz_k<D>(r)) << 4), cv = uint32_t((pos ^ swz_v<D>(r)) << 4);
        coff_k[j] = uint32_t(r * ROWB - 1024 * j) + ck;
        coff_v[j] = uint32_t(r * ROWB - 1024 * j) + cv;
        foff_k[j] = uint32_t(r) * row_bytes - 1024 * j + ck;
        foff_v[j] = uint32_t(r) * row_bytes - 1024 * j + cv;
    }

    // stages [mixed0, mixed1) may hold fresh rows beside cached ones (a block's,
    // or from the first to the last listed position), full_stages and on a
    // partial page
    const int last_pos = plist ? a.positions[it.pos_start + it.n - 1] : it.o + it.n - 1;
    const int full_stages = (kv_end - kv_begin) / STEP;
    const int mixed0 = all_fresh ? full_stages : min(full_stages, max(0, it.o - kv_begin) / STEP);
    const int mixed1 = all_fresh ? full_stages : last_pos < kv_begin ? 0 : (last_pos - kv_begin) / STEP + 1;
    const uint16_t* kfresh_w = kfresh + (int64_t)(kv_begin + wave * 16) * (int64_t)row_stride;
    const uint16_t* vfresh_w = vfresh + (int64_t)(kv_begin + wave * 16) * (int64_t)row_stride;
    const size_t stage_stride = STEP * row_stride;  // elements

    // do_k, do_v: whether to copy the stage's K rows and its V rows
    // (Over a quantised cache only whole prefills are copied: what cached and
    // listed rows need takes no registers there.)
    const bool copies_fresh = QUANT || all_fresh, copies_listed = !QUANT && plist;
    auto issue_stage = [&](int st, int buf, auto do_k, auto do_v) __attribute__((always_inline)) {
        uint8_t* kb = smem + buf * 2 * TILE;
        uint8_t* vb = kb + TILE;
        const int pl0 = st * SP & 63;  // lane holding the id of the stage's first page
        if (__builtin_expect(st < mixed0 || (st >= mixed1 && st < full_stages), 1)) {
            // a whole stage of one kind: wave-uniform bases, precomputed lane offsets
            const uint16_t* kf = kfresh_w + (size_t)unsigned(st) * stage_stride;
            const uint16_t* vf = vfresh_w + (size_t)unsigned(st) * stage_stride;
#pragma unroll
            for (int i = 0; i < PW; ++i) {
                const int k = wave + i * NW;  // page of the stage
                if (SP % NW != 0 && k >= SP) break;
                LDS void* kd = (LDS void*)(kb + k * 16 * ROWB);
                LDS void* vd = (LDS void*)(vb + k * 16 * ROWB);
                if (copies_fresh) {
                    if (do_k) copy_page(kf + i * NW * 16 * row_stride, foff_k, kd);
                    if (do_v) copy_page(vf + i * NW * 16 * row_stride, foff_v, vd);
                } else {
                    const size_t off = size_t(uint32_t(__builtin_amdgcn_readlane(pv, pl0 + k))) * page_stride;
                    if (do_k) copy_page(kcache + off, coff_k, kd);
                    if (do_v) copy_page(vcache + off, coff_v, vd);
                }
            }
            return;
        }
        const int skey0 = kv_begin + st * STEP;
        for (int k = wave; k < SP; k += NW) {
            LDS void* kd = (LDS void*)(kb + k * 16 * ROWB);
            LDS void* vd = (LDS void*)(vb + k * 16 * ROWB);
            // a page past the range: the stage's first page again, masked later
            const bool past = skey0 + k * 16 >= kv_end;
            const int key0 = past ? skey0 : skey0 + k * 16;
            const int pl = past ? pl0 : pl0 + k;
            const uint32_t inf = copies_listed ? uint32_t(__builtin_amdgcn_readlane(int(iv), pl)) : 0u;
            const size_t off = copies_fresh ? 0 : (size_t)__builtin_amdgcn_readlane(pv, pl) * page_stride;
            if (key0 + 16 <= kv_end && !copies_fresh &&
                (copies_listed ? (inf & 0xFFFFu) == 0 : key0 + 16 <= it.o || key0 >= it.o + it.n)) {
                if (do_k) copy_page(kcache + off, coff_k, kd);
                if (do_v) copy_page(vcache + off, coff_v, vd);
                continue;
            }
            // fresh rows of a block, listed positions, the range's partial
            // last page (rows past its end repeat its last row)
            const int lim = min(16, kv_end - key0);
            // fresh rows of the page: row `first` onwards, in order
            const int64_t first = copies_listed ? int64_t(it.q_start) + (inf >> kPageInfoRowShift)
                                        : int64_t(it.q_start) + key0 - it.o;
            const uint64_t fk = (uint64_t)(a.k_new + (size_t)t.kv_head * D) + uint64_t(first * int64_t(row_bytes));
            const uint64_t fv = (uint64_t)(a.v_new + (size_t)t.kv_head * D) + uint64_t(first * int64_t(row_bytes));
            uint64_t ak[IPP], av[IPP];
#pragma unroll
            for (int j = 0; j < IPP; ++j) {
                const int r = RPI * j + lane / NC, pos = lane % NC;
                const int rc = min(r, lim - 1);
                const bool fresh = copies_listed ? (inf >> rc) & 1u : unsigned(key0 + rc - it.o) < unsigned(it.n);
                const uint32_t frow = copies_listed ? __builtin_popcount(inf & ((1u << rc) - 1u)) : rc;
                const uint32_t ro = fresh ? frow * row_bytes : uint32_t(rc * ROWB);
                const int64_t lo = int64_t(ro) - 1024 * j;
                ak[j] = (fresh ? fk : (uint64_t)(kcache + off)) + uint64_t(lo + ((pos ^ swz_k<D>(r)) << 4));
                av[j] = (fresh ? fv : (uint64_t)(vcache + off)) + uint64_t(lo + ((pos ^ swz_v<D>(r)) << 4));
            }
            if (do_k) copy_page(ak, kd);
            if (do_v) copy_page(av, vd);
        }
    };

    // ---- staging of quantised pages: fetch() loads a stage's blocks into
    // registers, place() writes their values into the LDS tiles. A page is 16
    // rows of BPR blocks, and a lane has one block of each: of K's and of V's
    // page, or at head dim 64, where a page has half as many, of K's in the
    // lower half-wave and of V's in the upper one. A lane of a page with fresh
    // rows takes those from k_new / v_new in place(), as they are.
    // Where there are HELP waves, they do all of it.
    constexpr int SW = HELP > 0 ? HELP : NW;           // staging waves
    constexpr int PWQ = (SP + SW - 1) / SW;            // pages of one per stage
    const int swave = HELP > 0 ? wave - QW * KW : wave;
    constexpr int BPR = D / kMxBlock;
    constexpr int TPL = BPR / 2;  // tensors of a page that a lane has a block of
    const int ublock = lane % (16 * BPR);
    const int urow = ublock / BPR;
    typename Cache::Block raw[PWQ][TPL];
    uint32_t fresh_info[PWQ];  // page_info of the pages
    auto fetch = [&](int st) __attribute__((always_inline)) {
        if constexpr (QUANT) {
            if (all_fresh) return;
            const bool whole = st < mixed0 || (st >= mixed1 && st < full_stages);
            const int pl0 = st * SP & 63;
#pragma unroll
            for (int i = 0; i < PWQ; ++i) {
                const int k = swave + i * SW;  // page of the stage
                if (SP % SW != 0 && k >= SP) break;
                int pl = pl0 + k, row = urow;
                if (!whole) {  // a page past the range: the stage's first page again, rows past its end: its last row
                    int key0 = kv_begin + st * STEP;
                    if (key0 + 16 * k < kv_end) key0 += 16 * k;
                    else pl = pl0;
                    row = min(urow, kv_end - key0 - 1);
                    fresh_info[i] = plist ? uint32_t(__builtin_amdgcn_readlane(int(iv), pl)) : 0u;
                }
                const size_t at = (size_t(uint32_t(__builtin_amdgcn_readlane(pv, pl))) * a.hkv + t.kv_head) * (16 * BPR) +
                                  row * BPR + ublock % BPR;
#pragma unroll
                for (int j = 0; j < TPL; ++j) {
                    const bool v = TPL == 2 ? j != 0 : hh != 0;
                    raw[i][j].load(reinterpret_cast<const uint8_t*>(v ? a.v_cache : a.k_cache), v ? a.v_scale : a.k_scale, at);
                }
            }
        }
    };
    auto place = [&](int st, int buf) __attribute__((always_inline)) {
        if constexpr (QUANT) {
            const bool whole = st < mixed0 || (st >= mixed1 && st < full_stages);
#pragma unroll
            for (int i = 0; i < PWQ; ++i) {
                const int k = swave + i * SW;
                if (SP % SW != 0 && k >= SP) break;
                uint8_t* const tile = smem + buf * 2 * TILE + (k * 16 + urow) * ROWB;
                int64_t fresh_row = -1;  // row of k_new / v_new, -1: a cached row
                if (!whole) {
                    int key0 = kv_begin + st * STEP;
                    if (key0 + 16 * k < kv_end) key0 += 16 * k;
                    const int r = min(urow, kv_end - key0 - 1);
                    const uint32_t inf = fresh_info[i];
                    if (plist) {
                        if ((inf >> r) & 1u) fresh_row = int64_t(it.q_start) + (inf >> kPageInfoRowShift) + __builtin_popcount(inf & ((1u << r) - 1u));
                    } else if (unsigned(key0 + r - it.o) < unsigned(it.n)) {
                        fresh_row = int64_t(it.q_start) + key0 + r - it.o;
                    }
                }
#pragma unroll
                for (int j = 0; j < TPL; ++j) {
                    const bool v = TPL == 2 ? j != 0 : hh != 0;
                    u32x4 x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = raw[i][j].piece(e);
                    if (!whole && fresh_row >= 0) {
                        const uint16_t* src = (v ? a.v_new : a.k_new) + ((size_t)fresh_row * a.hkv + t.kv_head) * D + (ublock % BPR) * kMxBlock;
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = *(const u32x4*)(src + 8 * e);
                    }
                    const int swz = v ? swz_v<D>(urow) : swz_k<D>(urow);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *(LDS u32x4*)(tile + (v ? TILE : 0) + ((((ublock % BPR) * 4 + e) ^ swz) << 4)) = x[e];
                }
            }
        }
    };

    // place() of a stage without fresh rows, in PIECES of 8 dims of a lane's
    // blocks each, for the steps of the stage before
    constexpr int PIECES = PWQ * TPL * 4;
    auto place_piece = [&](int buf, int n) __attribute__((always_inline)) {
        if constexpr (QUANT) {
            const int i = n / (TPL * 4), j = n / 4 % TPL, e = n % 4;
            const int k = swave + i * SW;
            if (SP % SW != 0 && k >= SP) return;
            const bool v = TPL == 2 ? j != 0 : hh != 0;
            *(LDS u32x4*)(smem + buf * 2 * TILE + (v ? TILE : 0) + (k * 16 + urow) * ROWB +
                          ((((ublock % BPR) * 4 + e) ^ (v ? swz_v<D>(urow) : swz_k<D>(urow))) << 4)) = raw[i][j].piece(e);
        }
    };

    // ---- write-back of the fresh K/V rows into their cache pages. Per item
    // and KV head, the tiles of the group's first query head copy the fresh
    // rows they stage (a prefill tile its own row block, a block decode its
    // rows) from LDS, right after the stage lands: no second read of k_new /
    // v_new. Every fresh position lies in exactly one such tile's row block
    // and context range. No tile reads these cache rows (fresh positions come
    // from k_new / v_new, and the planner rejects pages shared between items),
    // so the copy needs no ordering with the attention. The pages written are
    // kept in LDS (one per page of a block, one per listed row), so the copy
    // loop issues no global load whose wait would also drain the prefetch.
    const int group = a.hq / a.hkv;
    const bool wb_head = across ? t.q_head0 == t.kv_head * group : t.q_head0 % group == 0;
    // positions written: [wb_lo, wb_hi) for a block; for a position list (a
    // decode, so heads-across), its listed positions inside the span from the
    // first to the last listed position
    const int wb_lo = max(kv_begin, it.o + (across ? 0 : t.row0));
    const int wb_hi = min(kv_end, across ? last_pos + 1 : it.o + min(it.n, t.row0 + 32 * QB * QW));
    const bool writer = wb_head && wb_lo < wb_hi;
    const int wpg0 = wb_lo >> 4;
    const int wst0 = writer ? (wb_lo - kv_begin) / STEP : nstages;  // stages [wst0, wst1) hold such rows
    const int wst1 = writer ? (wb_hi - 1 - kv_begin) / STEP + 1 : 0;
    auto write_back = [&](int st, auto do_k, auto do_v) {
        const int key0 = kv_begin + st * STEP;
        const int lo = max(wb_lo, key0), hi = min(wb_hi, key0 + STEP);
        if (lo >= hi) return;
        const uint8_t* kb = smem + (st % NSTAGE) * 2 * TILE;
        const uint8_t* vb = kb + TILE;
        if constexpr (QUANT) {  // the same rows, a block per thread
            uint64_t in = 0;
            if (plist) in = __builtin_amdgcn_ballot_w64(lane < it.n && lpos >= lo && lpos < hi);
            const int first = plist ? __builtin_ctzll(in | 1ull << 63) : 0;
            const int count = plist ? __builtin_popcountll(in) : hi - lo;
            for (int u = tid; u < count * BPR; u += NT) {
                const int row = first + u / BPR, b = u % BPR;
                const int p = plist ? fpos[row] : lo + row;
                const int page = plist ? wpages[row] : wpages[(p >> 4) - wpg0];
                const int r = p - key0;
                const size_t at = (((size_t)page * a.hkv + t.kv_head) * 16 + (p & 15)) * BPR + b;
                typename Cache::Block q;
                u32x4 x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = *(const LDS u32x4*)(kb + r * ROWB + (((4 * b + e) ^ swz_k<D>(r)) << 4));
                q.quantise(x);
                q.store(reinterpret_cast<uint8_t*>(a.k_cache), a.k_scale, at);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = *(const LDS u32x4*)(vb + r * ROWB + (((4 * b + e) ^ swz_v<D>(r)) << 4));
                q.quantise(x);
                q.store(reinterpret_cast<uint8_t*>(a.v_cache), a.v_scale, at);
            }
            return;
        }
        if (plist) {  // the listed positions inside [lo, hi): a run of the list
            const uint64_t in = __builtin_amdgcn_ballot_w64(lane < it.n && lpos >= lo && lpos < hi);
            const int first = __builtin_ctzll(in | 1ull << 63), count = __builtin_popcountll(in);
            for (int cidx = tid; cidx < count * NC; cidx += NT) {
                const int row = first + cidx / NC, p = fpos[row], pos = cidx % NC;
                const int r = p - key0;
                const u32x4 kv = *(const LDS u32x4*)(kb + r * ROWB + ((pos ^ swz_k<D>(r)) << 4));
                const u32x4 vv = *(const LDS u32x4*)(vb + r * ROWB + ((pos ^ swz_v<D>(r)) << 4));
                const size_t dst = (((size_t)wpages[row] * a.hkv + t.kv_head) * 16 + (p & 15)) * D + pos * 8;
                if (do_k) *(u32x4*)(a.k_cache + dst) = kv;
                if (do_v) *(u32x4*)(a.v_cache + dst) = vv;
            }
            return;
        }
        for (int cidx = tid; cidx < (hi - lo) * NC; cidx += NT) {
            const int p = lo + cidx / NC, pos = cidx % NC;
            const int r = p - key0;
            const u32x4 kv = *(const LDS u32x4*)(kb + r * ROWB + ((pos ^ swz_k<D>(r)) << 4));
            const u32x4 vv = *(const LDS u32x4*)(vb + r * ROWB + ((pos ^ swz_v<D>(r)) << 4));
            const size_t dst = (((size_t)wpages[(p >> 4) - wpg0] * a.hkv + t.kv_head) * 16 + (p & 15)) * D + pos * 8;
            if (do_k) *(u32x4*)(a.k_cache + dst) = kv;
            if (do_v) *(u32x4*)(a.v_cache + dst) = vv;
        }
    };

    // ---- stage-invariant LDS read offsets
    // K (A operand): lane reads key qn of each 32-key block, chunk 2k + hh of
    // k-step k: koff ^ (k << 5)
    const uint32_t koff = qn * ROWB + ((hh ^ swz_k<D>(qn)) << 4);
    // V^T (A operand) via transposing reads: 16-lane group g16 covers dims
    // mb*32 + (g16&1)*16 .. +15; lane (r4, j4) points at key row 4hh + r4 (+8),
    // dims 4 j4 .. 4 j4 + 3 of that group: voff ^ (mb << 6)
    const int g16 = lane >> 4;
    const int r4 = (lane >> 2) & 3;
    const int j4 = lane & 3;
    const int vdim = (g16 & 1) * 16 + 4 * j4;
    const uint32_t voff = (4 * hh + r4) * ROWB + (((vdim >> 3) ^ swz_v<D>(4 * hh + r4)) << 4) + (vdim & 7) * 2;
    const uint32_t lds0 = lds_wave_base((LDS void*)smem);

    f32x16 o[QB][MB];
    float m_used[QB];  // reference max (log2 domain) of this lane's query, per block
    float l_run[QB];   // sum of the rounded P over this lane's half of the keys
    float l_full[QB];  // over a quantised cache: of P as it is, which the LSE is then exact in
                       // (SOLO has no register for it: l_run is both, as below)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m_used[qb] = -INFINITY;
        l_run[qb] = l_full[qb] = 0.0f;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[qb][mb][i] = 0.0f;
    }
    const float c = a.scale_log2;

    // One stage of this wave: S^T = K Q^T (rows = keys, columns = queries; NB
    // 32-key blocks, each K fragment feeding the QB query blocks), online
    // softmax (exp2 domain), O^T += V^T P^T. tail: the stage may hold keys past
    // the range (set to -inf).
    //
    // The order of instructions is fixed here, MFMA by MFMA
    // (sched_barrier(0) after each step): the operand fragments form one
    // stream, K's then V's, each read from LDS RA steps before its MFMA; a
    // block's row max is taken beside the next block's QK^T and the
    // exponentials of the next 16 keys beside the PV of these. Left to the
    // compiler, most MFMAs sat right behind the LDS read they wait for (about
    // 130 cycles each), which a second wave on the SIMD hides in part only.
    // Measured per 64-key stage, K/V in L2, one 128-row work-group on the CU:
    // 1.30 -> 1.16 us at D = 128, 1.07 -> 0.85 us at D = 64; two: 1.98 -> 1.96
    // us and 1.32 -> 1.24 us (at D = 128 two work-groups draw the power limit:
    // the same MFMAs on random operands without the rest take 1.33 us).
    // between: called when the wave is done with the stage's K and is to read its V
    // beside: called with n in step n of QK^T, which leaves the VALU idle
    auto attend = [&](int st, auto tail, auto between, auto beside) __attribute__((always_inline)) {
        constexpr bool TAIL = decltype(tail)::value;
        constexpr int NK = NB * DS;      // K fragments (and QK^T steps)
        constexpr int NV = NB * 2 * MB;  // V fragments (and PV steps)
        const uint32_t buf = lds0 + (st % NSTAGE) * 2 * TILE + ks * KT * ROWB;
        const uint32_t ka = buf + koff, va = buf + TILE + voff;
        auto read_frag = [&](int n) -> bf16x8 {
            if (n < NK) return *(const LDS bf16x8*)(uintptr_t)((ka ^ uint32_t((n % DS) << 5)) + (n / DS) * 32 * ROWB);
            const int v = n - NK;  // 16 keys v / MB, 32 dims v % MB
            const uint32_t vp = (va ^ uint32_t((v % MB) << 6)) + (v / MB) * 16 * ROWB;
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS bf16x4*)(uintptr_t)vp);
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS bf16x4*)(uintptr_t)(vp + 8 * ROWB));
            return bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        };
        f32x16 s[QB][NB];
        float mx[QB];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) mx[qb] = -INFINITY;
        // row max over scores [i0, i1) of block b
        auto take_max = [&](int b, int i0, int i1) {
#pragma unroll
            for (int i = i0; i < i1; ++i) {
                const int key = kv_begin + st * STEP + ks * KT + b * 32 + 8 * (i >> 2) + 4 * hh + (i & 3);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) {
                    if (TAIL && key >= kv_end) s[qb][b][i] = -INFINITY;
                    mx[qb] = fmaxf(mx[qb], s[qb][b][i]);
                }
            }
        };

        bf16x8 frag[RA];
#pragma unroll
        for (int n = 0; n < RA; ++n) frag[n] = read_frag(n);
        if (PRIO == 1) __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < NK; ++n) {
            const int b = n / DS, k = n % DS;
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                if (k == 0)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[qb][b][i] = 0.0f;
                s[qb][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % RA], qf[qb][k], s[qb][b], 0, 0, 0);
            }
            if (!TURNS || n + RA < NK) frag[n % RA] = read_frag(n + RA);
            // the previous block's scores are written two steps into this one
            if (b > 0 && k >= 2) take_max(b - 1, (k - 2) * 16 / (DS - 2), (k - 1) * 16 / (DS - 2));
            beside(n);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (PRIO == 1) __builtin_amdgcn_s_setprio(0);
        take_max(NB - 1, 0, 16);

        // The reference max moves (and O, l are rescaled) only when a score
        // exceeds it by more than kRescaleThreshold, which is rare after the
        // first stage.
        bool any_need = false;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            mx[qb] = half_max(mx[qb]) * c;
            any_need |= mx[qb] > m_used[qb] + kRescaleThreshold;
        }
        if (__builtin_amdgcn_ballot_w64(any_need)) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                const bool need = mx[qb] > m_used[qb] + kRescaleThreshold;
                const float alpha = need ? __builtin_amdgcn_exp2f(m_used[qb] - mx[qb]) : 1.0f;
                m_used[qb] = need ? mx[qb] : m_used[qb];
                l_run[qb] *= alpha;
                if constexpr (QUANT) l_full[qb] *= alpha;
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[qb][mb][i] *= alpha;
            }
        }

        if constexpr (TURNS) {
            between();
#pragma unroll
            for (int n = NK; n < NK + RA; ++n) frag[n % RA] = read_frag(n);
            __builtin_amdgcn_sched_barrier(0);
        }

        // P = exp2(s c - m) rounded to bf16 (the PV operand); l += the rounded
        // values. Lane slot j of the P^T of 16 keys kk holds key
        // 16kk + 8(j/4) + 4hh + j%4.
        bf16x8 pf[QB][NB * 2];
        float mneg[QB];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) mneg[qb] = m_used[qb] == -INFINITY ? 0.0f : -m_used[qb];
        auto exps = [&](int kk, int j0, int j1) {
#pragma unroll
            for (int j = j0; j < j1; j += 2)
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) {
                    const f32x16& sb = s[qb][kk >> 1];
                    const int i = 8 * (kk & 1) + j;
                    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sb[i], c, mneg[qb]));
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sb[i + 1], c, mneg[qb]));
                    const bf16x2 pp = {(__bf16)p0, (__bf16)p1};
                    if constexpr (QUANT) l_full[qb] += p0 + p1;
                    l_run[qb] = __builtin_amdgcn_fdot2_f32_bf16(pp, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, l_run[qb], false);
                    pf[qb][kk][j] = pp[0];
                    pf[qb][kk][j + 1] = pp[1];
                }
        };
        exps(0, 0, 8);
        if (PRIO == 2) __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int kk = n / MB, mb = n % MB;
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
                o[qb][mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[(NK + n) % RA], pf[qb][kk], o[qb][mb], 0, 0, 0);
            if (n + RA < NV) frag[(NK + n) % RA] = read_frag(NK + n + RA);
            if (kk + 1 < NB * 2) exps(kk + 1, mb * 8 / MB, (mb + 1) * 8 / MB);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (PRIO == 2) __builtin_amdgcn_s_setprio(0);
    };

    // Stages st+1 .. st+NSTAGE-1 are in flight while stage st is computed.
    // Loads complete in order, so waiting for stage st leaves the later
    // stages outstanding.
    constexpr int LPS = 2 * IPP * PW;  // loads per stage per wave (K and V)
    auto wait_stage = [&](int st) {
        const int later = min(NSTAGE - 2, nstages - 1 - st);  // stages issued after st
        if (NSTAGE >= 4 && later >= 2)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LPS) : "memory");
        else if (NSTAGE >= 3 && later >= 1)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LPS) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    // The compiler does not see the copies, so it would make the first use of
    // Q wait for every one in flight: Q is waited for here, with the page ids
    // or the first stage, which are needed at this point anyway.
    auto wait_q = [&]() {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int s = 0; s < DS; ++s) asm volatile("" : "+v"(qf[qb][s]));
    };
    if (NSTAGE > 2) wait_q();
    // the next 64 page ids, once stage st has read the last of these
    auto next_pages = [&](int st) {
        if (!all_fresh && ((st + 1) * SP & 63) == 0 && (st + 1) * SP < npg) load_pages((st + 1) * SP);
    };
    // the write-back's pages: loaded before the first copies, kept in LDS after
    const int nwp = writer ? plist ? it.n : ((wb_hi + 15) >> 4) - wpg0 : 0;
    int32_t wpage = 0;
    if (tid < nwp) wpage = a.page_ids[it.page_start + (plist ? lpos >> 4 : wpg0 + tid)];
    constexpr auto yes = std::true_type{};
    constexpr auto no = std::false_type{};
    auto nothing = [](int) {};
    if constexpr (SOLO) {
        // begins below
    } else if constexpr (QUANT) {
        if (NB != 4 && HELP == 0) {
            fetch(0);
            next_pages(0);
        }
    } else {
        for (int k = 0; k < NSTAGE - 1 && k < nstages; ++k) issue_stage(k, k, yes, yes);
    }
    if (TURNS) issue_stage(0, 0, yes, no);
    if (NSTAGE <= 2) wait_q();
    if (tid < nwp) {
        wpages[tid] = wpage;
        if (plist) fpos[tid] = lpos;
    }
    int st = 0;
    if constexpr (SOLO) {
        // One query head: no other wave of the work-group reads the keys of this
        // one, so nothing is shared and nothing waits at a barrier. A wave takes
        // every KW-th block of 32 keys, loads it NSTAGE blocks ahead into
        // registers and converts it there. K goes from them into QK^T directly:
        // the order of the dims in that product is free as long as Q has the
        // same one, and with dims D / 2 hh + 8 n at step n a lane's operands are
        // one half of its key's row, whole blocks that it can load. V, whose
        // operands run along the keys, is turned through a tile of LDS of the
        // wave's own. The page ids of the tile's range stand in LDS.
        // Bound by HBM where there are tiles enough: 64 contexts of 206,649
        // positions in all, 32 heads, e4m3, 355 us (5.3 TB/s are fetched) against
        // 543 for tiles of bf16 values that two waves share, with a barrier per
        // stage. (K loaded in the order of memory and passed to its lanes
        // through LDS takes half the lines per instruction, and 363 us.)
        static_assert(QB == 1 && NB == 1 && NSTAGE <= 2, "a block of 32 keys at a time");
        constexpr int BL = D / 64;                    // blocks of K, and of V, per lane
        constexpr int PAGES = kMaxCachedRange / 16;   // of a tile (an item without cached rows has two at most)
        static_assert(KW * 32 * ROWB + PAGES * 8 <= sizeof(shared.stages), "V tiles, page ids and page_info");
        struct Keys {
            typename Cache::Block k[BL], v[BL];
            uint32_t k_scales;  // of k, a byte each
        };
        int32_t* const ids = reinterpret_cast<int32_t*>(smem + KW * 32 * ROWB);
        uint32_t* const infos = reinterpret_cast<uint32_t*>(ids + PAGES);
        for (int k = tid; k < npg; k += NT) {
            ids[k] = a.page_ids[it.page_start + pg0 + k];
            if (plist) infos[k] = a.page_info[it.page_start + pg0 + k];
        }
        __syncthreads();
        const int nblocks = (kv_end - kv_begin + 31) / 32;
        const int first_fresh = plist ? __builtin_amdgcn_readfirstlane(lpos) : it.o;
        auto place_of = [&](int b, int r) {  // row of the pool that holds key r of block b
            return (size_t(uint32_t(ids[2 * b + (r >> 4)])) * a.hkv + t.kv_head) * 16 + (r & 15);
        };
        auto fresh_row = [&](int b, int r) -> int64_t {  // row of k_new / v_new of key r of block b, or -1
            if (plist) {
                const uint32_t inf = infos[2 * b + (r >> 4)], s = r & 15;
                return (inf >> s) & 1u ? int64_t(it.q_start) + (inf >> kPageInfoRowShift) + __builtin_popcount(inf & ((1u << s) - 1u)) : -1;
            }
            const int n = kv_begin + 32 * b + r - it.o;
            return unsigned(n) < unsigned(it.n) ? int64_t(it.q_start) + n : -1;
        };
        const uint8_t* const kc = reinterpret_cast<const uint8_t*>(a.k_cache);
        const uint8_t* const vc = reinterpret_cast<const uint8_t*>(a.v_cache);
        auto load = [&](int b, Keys& x) __attribute__((always_inline)) {
            const int last = kv_end - kv_begin - 32 * b - 1;  // keys past the range: its last one, masked later
            const size_t kr = place_of(b, min(qn, last)) * BPR + hh * BL;
#pragma unroll
            for (int i = 0; i < BL; ++i) x.k[i].load(kc, kr + i);
            x.k_scales = BL == 2 ? uint32_t(*(const uint16_t*)(a.k_scale + kr)) : a.k_scale[kr];
#pragma unroll
            for (int i = 0; i < BL; ++i) {
                const int u = i * 64 + lane;
                x.v[i].load(vc, a.v_scale, place_of(b, min(u / BPR, last)) * BPR + u % BPR);
            }
            asm volatile("" ::: "memory");  // the loads stay up here
        };
        // what was loaded, from here on (the compiler would split the scales,
        // and wait for them, right behind the load)
        auto arrive = [&](Keys& x) __attribute__((always_inline)) {
            asm volatile("" : "+v"(x.k_scales));
#pragma unroll
            for (int i = 0; i < BL; ++i) {
                x.k[i].scale = x.k_scales >> (8 * i) & 255u;
                asm volatile("" : "+v"(x.v[i].scale));
            }
        };
        uint8_t* const vtile = smem + ks * 32 * ROWB;
        const uint32_t va = lds0 + ks * 32 * ROWB + voff;
        // One block, whose K operands and pieces of V `k_piece` and `v_piece`
        // give; `next` is called when both have been taken.
        auto block = [&](int b, auto k_piece, auto v_piece, auto next) __attribute__((always_inline)) {
            const int last = kv_end - kv_begin - 32 * b - 1;
            f32x16 s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
            for (int n = 0; n < DS; ++n)
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k_piece(n)), qf[0][n], s, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < BL; ++i) {
                const int u = i * 64 + lane, r = u / BPR, c = 4 * (u % BPR);
#pragma unroll
                for (int e = 0; e < 4; ++e) *(LDS u32x4*)(vtile + r * ROWB + (((c + e) ^ swz_v<D>(r)) << 4)) = v_piece(i, e);
            }
            asm volatile("" ::: "memory");
            next();
            if (last < 31)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (8 * (i >> 2) + 4 * hh + (i & 3) > last) s[i] = -INFINITY;
            float mx = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
            mx = half_max(mx) * c;
            const bool need = mx > m_used[0] + kRescaleThreshold;
            if (__builtin_amdgcn_ballot_w64(need)) {
                const float alpha = need ? __builtin_amdgcn_exp2f(m_used[0] - mx) : 1.0f;
                m_used[0] = need ? mx : m_used[0];
                l_run[0] *= alpha;
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[0][mb][i] *= alpha;
            }
            const float mneg = m_used[0] == -INFINITY ? 0.0f : -m_used[0];
            bf16x8 pf[2];
            float full = 0.0f, rounded = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, mneg));
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i + 1], c, mneg));
                const bf16x2 pp = {(__bf16)p0, (__bf16)p1};
                full += p0 + p1;
                rounded = __builtin_amdgcn_fdot2_f32_bf16(pp, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, rounded, false);
                pf[i >> 3][i & 7] = pp[0];
                pf[i >> 3][(i & 7) + 1] = pp[1];
            }
            l_run[0] += half_sums(rounded, full);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    const uint32_t vp = (va ^ uint32_t(mb << 6)) + kk * 16 * ROWB;
                    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS bf16x4*)(uintptr_t)vp);
                    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS bf16x4*)(uintptr_t)(vp + 8 * ROWB));
                    o[0][mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}, pf[kk],
                                                                      o[0][mb], 0, 0, 0);
                }
            asm volatile("" ::: "memory");
        };
        // blocks [m0, m1) may hold fresh rows; the others are taken first
        const int m0 = min(nblocks, max(0, first_fresh - kv_begin) / 32);
        const int m1 = last_pos < kv_begin ? m0 : min(nblocks, (last_pos - kv_begin) / 32 + 1);
        const int cached = m0 + nblocks - m1;
        if (computes) {
            Keys x[NSTAGE];
            auto at = [&](int k) { return k < m0 ? k : k + m1 - m0; };
            auto take = [&](int k, Keys& y, auto next) __attribute__((always_inline)) {
                arrive(y);
                block(at(k), [&](int n) { return y.k[n / 4].piece(n % 4); }, [&](int i, int e) { return y.v[i].piece(e); },
                      [&]() { if constexpr (decltype(next)::value) load(at(k + NSTAGE * KW < cached ? k + NSTAGE * KW : k), y); });
            };
            // Every pass loads, past the end a block that it has, and a pair of
            // passes has no way out between: with loads that may not be there
            // the compiler waits for all of them.
            if (ks < cached) {
                int k = ks;
                load(at(k), x[0]);
                if constexpr (NSTAGE == 2) {
                    load(at(k + KW < cached ? k + KW : k), x[1]);
                    for (; k + KW < cached; k += 2 * KW) {
                        take(k, x[0], yes);
                        take(k + KW, x[1], yes);
                    }
                    if (k < cached) take(k, x[0], no);
                } else {
                    for (; k < cached; k += KW) take(k, x[0], yes);
                }
            }
            for (int b = m0 + ks; b < m1; b += KW) {
                const int last = kv_end - kv_begin - 32 * b - 1;
                load(b, x[0]);
                arrive(x[0]);
                const int64_t krow = fresh_row(b, min(qn, last));
                const uint16_t* const kf = a.k_new + ((size_t)(krow < 0 ? 0 : krow) * a.hkv + t.kv_head) * D + D / 2 * hh;
                block(b,
                      [&](int n) {
                          const u32x4 f = *(const u32x4*)(kf + 8 * n);
                          return krow < 0 ? x[0].k[n / 4].piece(n % 4) : f;
                      },
                      [&](int i, int e) {
                          const int u = i * 64 + lane;
                          const int64_t row = fresh_row(b, min(u / BPR, last));
                          const u32x4 f = *(const u32x4*)(a.v_new + ((size_t)(row < 0 ? 0 : row) * a.hkv + t.kv_head) * D + u % BPR * kMxBlock + 8 * e);
                          return row < 0 ? x[0].v[i].piece(e) : f;
                      },
                      []() {});
            }
        }
        if (writer) {  // the fresh rows of the range into their pages, a block per thread
            for (int u = tid; u < it.n * BPR; u += NT) {
                const int row = u / BPR, b = u % BPR;
                const int p = plist ? a.positions[it.pos_start + row] : it.o + row;
                if (p < wb_lo || p >= wb_hi) continue;
                const size_t at = ((size_t(uint32_t(ids[(p >> 4) - pg0])) * a.hkv + t.kv_head) * 16 + (p & 15)) * BPR + b;
                const size_t from = ((size_t)(it.q_start + row) * a.hkv + t.kv_head) * D + b * kMxBlock;
                typename Cache::Block q;
                u32x4 x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = *(const u32x4*)(a.k_new + from + 8 * e);
                q.quantise(x);
                q.store(reinterpret_cast<uint8_t*>(a.k_cache), a.k_scale, at);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = *(const u32x4*)(a.v_new + from + 8 * e);
                q.quantise(x);
                q.store(reinterpret_cast<uint8_t*>(a.v_cache), a.v_scale, at);
            }
        }
    } else if constexpr (QUANT) {
        // Stage st + 1 is on its way into registers while stage st is
        // computed; with two buffers it is placed before the barrier that ends
        // stage st, with one behind it. A whole prefill's stages are copied
        // into LDS, into the other buffer or, with one, at once.
        // (The wide tiles have no registers for that: long prefills, which
        // read no cached rows. A long block over a cached context waits.)
        static_assert(NSTAGE <= 2, "the next stage waits in registers");
        static_assert(HELP == 0 || NSTAGE == 2, "helpers place the next stage beside the others' work");
        constexpr bool LATE = NB == 4;
        auto go_on = []() {};
        auto bring = [&](int s) {  // into LDS
            if (LATE) {
                fetch(s);
                next_pages(s);
            }
            if (all_fresh) issue_stage(s, s % NSTAGE, yes, yes);
            else place(s, s % NSTAGE);
        };
        auto ahead = [&](int s) {  // into registers
            if (LATE || s >= nstages) return;
            fetch(s);
            next_pages(s);
            asm volatile("" ::: "memory");  // the loads stay up here
        };
        auto stage = [&](auto tail) __attribute__((always_inline)) {
            if (NSTAGE == 1) {
                if (st > 0) __syncthreads();
                bring(st);
            }
            if (all_fresh) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (NSTAGE == 1) ahead(st + 1);
            else if (all_fresh && st + 1 < nstages) bring(st + 1);
            if (st >= wst0 && st < wst1) write_back(st, yes, yes);
            const bool more = NSTAGE == 2 && !all_fresh && st + 1 < nstages;
            bool placed = false;
            // The next stage's values are converted beside the last steps of
            // QK^T, where a CU holds two work-groups and a wave has one page:
            // 64 decodes of 32/8 heads of 128 e4m3 93.0 -> 89.9 us, e2m1 84.8 ->
            // 80.5. (Seven and eight waves, one work-group to a CU, lose 1 %; head
            // dim 64 has no registers for it.)
            if constexpr (!decltype(tail)::value && NSTAGE == 2 && PWQ == 1 && QW == 4 && D == 128) {
                if (head_ok && more && (st + 1 < mixed0 || (st + 1 >= mixed1 && st + 1 < full_stages))) {
                    attend(st, tail, go_on, [&](int n) __attribute__((always_inline)) {
                        constexpr int NK = NB * DS, PER = (PIECES + NK - 1) / NK, FIRST = NK - (PIECES + PER - 1) / PER;
#pragma unroll
                        for (int p = (n - FIRST) * PER; p < (n - FIRST + 1) * PER; ++p)
                            if (p >= 0 && p < PIECES) place_piece((st + 1) & 1, p);
                    });
                    placed = true;
                }
            }
            if (!placed && head_ok) attend(st, tail, go_on, nothing);
            if (more) {
                if (!placed) bring(st + 1);
                ahead(st + 2);
            }
        };
        if constexpr (HELP > 0) {
            // The helpers take the waves' places on the SIMDs that have one
            // fewer, and the others no time off for the staging. (Two loops:
            // neither's registers are the other's.)
            auto begin = [&]() __attribute__((always_inline)) {  // a stage, after the barrier
                if (all_fresh) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (all_fresh && st + 1 < nstages) issue_stage(st + 1, (st + 1) % NSTAGE, yes, yes);
                if (st >= wst0 && st < wst1) write_back(st, yes, yes);
            };
            if (all_fresh) issue_stage(0, 0, yes, yes);
            if (computes) {
                for (; st < full_stages; ++st) {
                    begin();
                    if (head_ok) attend(st, std::false_type{}, go_on, nothing);
                }
                if (st < nstages) {
                    begin();
                    if (head_ok) attend(st, std::true_type{}, go_on, nothing);
                }
            } else {
                if (!all_fresh) {
                    fetch(0);
                    next_pages(0);
                    place(0, 0);
                    ahead(1);
                }
                for (; st < nstages; ++st) {
                    begin();
                    if (!all_fresh && st + 1 < nstages) {
                        place(st + 1, (st + 1) % NSTAGE);
                        ahead(st + 2);
                    }
                }
            }
        } else {
            if (NSTAGE == 2) {
                bring(0);
                if (!all_fresh) ahead(1);
            }
            for (; st < full_stages; ++st) stage(std::false_type{});
            if (st < nstages) stage(std::true_type{});
        }
    } else if constexpr (TURNS) {
        // a stage: its K is there, V on its way under QK^T, the next K under PV
        auto stage = [&](auto tail) __attribute__((always_inline)) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            issue_stage(st, 0, no, yes);
            next_pages(st);
            if (st >= wst0 && st < wst1) write_back(st, yes, no);
            attend(st, tail, [&]() __attribute__((always_inline)) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (st + 1 < nstages) issue_stage(st + 1, 0, yes, no);
                if (st >= wst0 && st < wst1) write_back(st, no, yes);
            }, nothing);
        };
        for (; st < full_stages; ++st) stage(std::false_type{});
        if (st < nstages) stage(std::true_type{});
    } else {
        auto go_on = []() {};
        for (; st < full_stages; ++st) {
            wait_stage(st);
            __syncthreads();
            if (st + NSTAGE - 1 < nstages) {
                issue_stage(st + NSTAGE - 1, (st + NSTAGE - 1) % NSTAGE, yes, yes);
                next_pages(st + NSTAGE - 1);
            }
            if (st >= wst0 && st < wst1) write_back(st, yes, yes);
            if (head_ok) attend(st, std::false_type{}, go_on, nothing);  // a wave past its tile's GQA group only stages and writes back
        }
        if (st < nstages) {  // the last, partial stage
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (st >= wst0 && st < wst1) write_back(st, yes, yes);
            if (head_ok) attend(st, std::true_type{}, go_on, nothing);
        }
    }

    // Over a quantised cache both sums go on as one value, the rounded weights'
    // in the lower half-wave and the full one in the upper one. O is divided by
    // the former, so that it is an average of V's rows (equal rows give
    // themselves); the LSE, by which splits are weighed, is that of the latter.
    // (The second sum: 48 decodes of 28/4 heads e4m3 39.2 -> 40.6 us, prefills of
    // 2304 and 3328 rows of them 244 -> 250, both in one launch 276 -> 285; 16 MHA
    // decodes beside prefills of 1819 and 1201 rows 165 -> 167.6, MHA decodes alone
    // nothing.)
    if constexpr (QUANT && !SOLO)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) l_run[qb] = half_sums(l_run[qb], l_full[qb]);

    // ---- combine the context sub-ranges of the waves that share query rows:
    // each of the KW waves then holds MBW of the MB 32-dim blocks of O
    constexpr int MBW = MB / KW;
    const int mb0 = ks * MBW;  // first block of this wave
    if constexpr (KW > 1) {
        __syncthreads();
        float* mbuf = reinterpret_cast<float*>(smem) + (size_t)qs * KW * MERGE_REGS * 64;
        float* mine = mbuf + (size_t)ks * MERGE_REGS * 64;
        if (computes) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 16; ++i) mine[(mb * 16 + i) * 64 + lane] = o[0][mb][i];
            mine[(MB * 16) * 64 + lane] = m_used[0];
            mine[(MB * 16 + 1) * 64 + lane] = l_run[0];
        }
        __syncthreads();
        const float* src[KW];
#pragma unroll
        for (int k = 0; k < KW; ++k) src[k] = mbuf + k * MERGE_REGS * 64;
        float m_tot = fmaxf(src[0][(MB * 16) * 64 + lane], src[1][(MB * 16) * 64 + lane]);
#pragma unroll
        for (int k = 2; k < KW; ++k) m_tot = fmaxf(m_tot, src[k][(MB * 16) * 64 + lane]);
        // wave ks = 0 always holds a valid key, so m_tot is finite
        float sc[KW], l[KW];
#pragma unroll
        for (int k = 0; k < KW; ++k) {
            sc[k] = __builtin_amdgcn_exp2f(src[k][(MB * 16) * 64 + lane] - m_tot);
            l[k] = src[k][(MB * 16 + 1) * 64 + lane];
        }
        // Which product of a sum is fused is written out: the compiler may
        // take either, and another build would differ in the last bits.
        const float l1 = sc[1] * l[1];
        l_run[0] = __builtin_fmaf(sc[0], l[0], l1);
#pragma unroll
        for (int k = 2; k < KW; ++k) l_run[0] = __builtin_fmaf(sc[k], l[k], l_run[0]);
#pragma unroll
        for (int mb = 0; mb < MBW; ++mb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int at = ((mb0 + mb) * 16 + i) * 64 + lane;
                const float o0 = sc[0] * src[0][at];
                o[0][mb][i] = __builtin_fmaf(sc[1], src[1][at], o0);
#pragma unroll
                for (int k = 2; k < KW; ++k) o[0][mb][i] = __builtin_fmaf(sc[k], src[k][at], o[0][mb][i]);
            }
        m_used[0] = m_tot;
    }

    // ---- epilogue: O / l and the LSE, to the output or as a split's partial
    float lse_val[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float2 l = QUANT ? both_sums(l_run[qb]) : float2{half_sum(l_run[qb]), 0.0f};
        const float inv = 1.0f / l.x;
        lse_val[qb] = m_used[qb] * 0.69314718055994530942f + logf(QUANT ? l.y : l.x);
#pragma unroll
        for (int mb = 0; mb < MBW; ++mb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[qb][mb][i] *= inv;
    }
    if (split_out) {
        if (!merge_here) {
            // rows of D for merge_kernel: [split][row][head]
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                const int row = row_base + 32 * qb + qn;
                if (!head_ok || row >= it.n) continue;
                const size_t prow = (size_t)(t.split * it.n + row) * a.hq + head;
                float* po = a.ws + it.ws_o + prow * D;
#pragma unroll
                for (int mb = 0; mb < MBW; ++mb)
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4)
                        *(float4*)(po + (mb0 + mb) * 32 + 8 * q4 + 4 * hh) =
                            float4{o[qb][mb][4 * q4], o[qb][mb][4 * q4 + 1], o[qb][mb][4 * q4 + 2], o[qb][mb][4 * q4 + 3]};
                if (hh == 0 && ks == 0) a.ws[it.ws_lse + prow] = lse_val[qb];
            }
            return;
        }
        // For a merge by a tile like this one: [split][head][rows of 32]
        // [D / 4][row] float4 and [split][head][row] LSE, so that a wave's
        // store, and its load by the merging wave, of one register is 16-byte
        // pieces of consecutive rows.
        const size_t rows0 = (size_t)(t.split * a.hq + head) * it.n;  // rows before this (split, head)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int r0 = row_base + 32 * qb, nb = min(32, it.n - r0);
            if (!head_ok || qn >= nb) continue;
            float* po = a.ws + it.ws_o + (rows0 + r0) * D;
#pragma unroll
            for (int mb = 0; mb < MBW; ++mb)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const int d4 = (mb0 + mb) * 8 + q4 * 2 + hh;
                    const float4 v = {o[qb][mb][4 * q4], o[qb][mb][4 * q4 + 1], o[qb][mb][4 * q4 + 2], o[qb][mb][4 * q4 + 3]};
                    store_agent(po + (size_t)(d4 * nb + qn) * 4, v);
                }
            if (hh == 0 && ks == 0) store_agent(a.ws + it.ws_lse + rows0 + r0 + qn, lse_val[qb]);
        }
        // The tile that finds every split of its rows written merges them.
        // Each tile marks its split with the call's nonce, then looks at all
        // marks: both are read-modify-writes, complete before the next, so
        // the last tile to mark finds all of them. Two tiles may, and then
        // write the same bits. The merging tile clears the marks, so that a
        // replayed graph, whose nonce repeats, starts from none; whatever
        // else the workspace held is not this call's 64-bit nonce.
        uint64_t* marks = reinterpret_cast<uint64_t*>(a.ws + merge_marks(it, a.hq)) +
                          (size_t)((t.row0 / kWaveRows) * a.hq + t.q_head0) * it.num_splits;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's partials are in memory
        __syncthreads();
        if (wave == 0) {
            uint64_t before = 0, none = 0;
            if (lane == 0) before = __hip_atomic_exchange(marks + t.split, a.nonce, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(before), "+v"(none)::"memory");
            bool there = true;
            if (lane < it.num_splits)
                there = __hip_atomic_fetch_or(marks + lane, none, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.nonce;
            const bool all = __builtin_amdgcn_ballot_w64(there) == ~0ull;
            if (all && lane < it.num_splits)
                __hip_atomic_store(marks + lane, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (lane == 0) shared.merging = all;
        }
        __syncthreads();
        if (!shared.merging) return;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int r0 = row_base + 32 * qb, nb = min(32, it.n - r0);
            if (!head_ok || nb <= 0) continue;
            const int row = min(qn, nb - 1);  // lanes past the last row repeat it
            const size_t step = (size_t)a.hq * it.n;  // rows between splits
            const size_t first = (size_t)head * it.n + r0;
            float ls[MAXS], mx = -INFINITY;
#pragma unroll
            for (int k = 0; k < MAXS; ++k)
                if (k < it.num_splits) ls[k] = load_agent(a.ws + it.ws_lse + k * step + first + row);
#pragma unroll
            for (int k = 0; k < MAXS; ++k)
                if (k < it.num_splits) mx = fmaxf(mx, ls[k]);
            f32x16 acc[MBW];
            float tot = 0.0f;
#pragma unroll
            for (int mb = 0; mb < MBW; ++mb)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[mb][i] = 0.0f;
#pragma unroll 2
            for (int k = 0; k < it.num_splits; ++k) {
                const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(
                    a.ws + it.ws_o + (k * step + first) * D, 0, nb * D * 4, 0x00027000);
                u32x4 v[MBW * 4];
#pragma unroll
                for (int j = 0; j < MBW * 4; ++j) {
                    const int d4 = (mb0 + j / 4) * 8 + (j & 3) * 2 + hh;
                    v[j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, (d4 * nb + row) * 16, 0, kBufferAgent);
                }
                float w = 0.0f;
#pragma unroll
                for (int m = 0; m < MAXS; ++m)
                    if (m == k) w = __expf(ls[m] - mx);
                tot += w;
#pragma unroll
                for (int j = 0; j < MBW * 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[j / 4][4 * (j & 3) + e] += w * __uint_as_float(v[j][e]);
            }
            const float inv = 1.0f / tot;
#pragma unroll
            for (int mb = 0; mb < MBW; ++mb)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[qb][mb][i] = acc[mb][i] * inv;
            lse_val[qb] = mx + logf(tot);
        }
    }
    // Output rows leave through LDS where it holds them: each lane stages its
    // query's dims in 8-byte pieces, then 16 consecutive lanes store one whole
    // row in 16-byte pieces (stored directly, one instruction would leave
    // 16-byte fragments of 32 rows).
    constexpr int EROW = D * 2 + 16;  // bytes per staged row: 16-byte aligned, shifted by four banks
    constexpr int EBASE = KW > 1 && !SOLO ? QW * KW * MERGE_REGS * 64 * 4 : 0;  // past the waves' partials, or in their place
    constexpr bool ESTAGE = EBASE + QW * QB * 32 * EROW <= sizeof(shared.stages);
    if constexpr (SOLO) __syncthreads();  // every wave has read the partials
    if constexpr (ESTAGE && KW == 1) {
        if (!split_out) __syncthreads();  // every wave is past its last stage's reads
    }
    uint8_t* ebuf = smem + EBASE + qs * (QB * 32 * EROW);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int row = row_base + 32 * qb + qn;
        const bool stored = row < it.n && head_ok;
        uint16_t* op = a.out + ((size_t)(it.q_start + row) * a.hq + head) * D;
#pragma unroll
        for (int mb = 0; mb < MBW; ++mb)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const int dim = (mb0 + mb) * 32 + 8 * q4 + 4 * hh;
                const bf16x4 v = {(__bf16)o[qb][mb][4 * q4], (__bf16)o[qb][mb][4 * q4 + 1],
                                  (__bf16)o[qb][mb][4 * q4 + 2], (__bf16)o[qb][mb][4 * q4 + 3]};
                if (ESTAGE && !computes) continue;
                if (ESTAGE) *(LDS u32x2*)(ebuf + (32 * qb + qn) * EROW + dim * 2) = __builtin_bit_cast(u32x2, v);
                else if (stored) *(u32x2*)(op + dim) = __builtin_bit_cast(u32x2, v);
            }
        if (stored && hh == 0 && ks == 0 && a.lse) a.lse[(size_t)(it.q_start + row) * a.hq + head] = lse_val[qb];
    }
    if constexpr (ESTAGE) {
        // with one wave per query slot a wave reads back only rows it staged
        if constexpr (KW > 1) __syncthreads();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (head_ok) {
            constexpr int CPR = D / 8;           // 16-byte pieces per row
            constexpr int NCE = QB * 32 * CPR;   // pieces per query slot
            static_assert(NCE % (64 * KW) == 0, "whole rounds of 64 lanes");
#pragma unroll
            for (int j = 0; j < NCE / (64 * KW); ++j) {
                const int c = (j * KW + ks) * 64 + lane;
                const int r = c / CPR, col = c % CPR;  // staged row r is row row_base + r
                if (row_base + r < it.n) {
                    const u32x4 v = *(const LDS u32x4*)(ebuf + r * EROW + col * 16);
                    *(u32x4*)(a.out + ((size_t)(it.q_start + row_base + r) * a.hq + head) * D + col * 8) = v;
                }
            }
        }
    }
}

}  // namespace
