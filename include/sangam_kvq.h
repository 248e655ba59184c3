/*
 * sangam_kvq.h - C ABI of the quantised KV cache of cached diffusion-LLM
 * serving, for AMD Instinct MI355X (gfx950): the attention call of
 * sangam_attn.h over pages that hold 8 or 4 bits a value, and the export and
 * import of sangam_kv.h for such pages.
 *
 * A cached row of D dims is D / 32 blocks of 32 consecutive dims. A block is
 * 32 codes and one scale byte b; code c stands for the value c 2^(b - 127) (the
 * OCP Microscaling formats MXFP8 and MXFP4):
 *   SANGAM_KV_E4M3   8 bits, e4m3 (no infinity), largest code M = 448
 *   SANGAM_KV_E2M1   4 bits, e2m1 (0, .5, 1, 1.5, 2, 3, 4, 6), M = 6; dim 2 i of
 *                    a row in the low half of byte i, dim 2 i + 1 in the high half
 * A block with largest magnitude A is written with
 *   b = max(10, the smallest b with A <= M 2^(b - 127))
 *   code(x) = x 2^(127 - b) rounded to nearest, ties to even
 * so that no value saturates, and a value is off by at most 2^-4 (e4m3) or 2^-2
 * (e2m1) of itself, or by half the smallest code, 2^(b - 137) or 2^(b - 129),
 * where that is more. What a row reads back as is exact in bf16 (writing it
 * again gives the same values) but for magnitudes within 2^125 of 2^128, which
 * may round to 2^128 and read back as infinity. A block with an infinity or a
 * NaN has b = 255 and codes 0, and reads back as NaN. Blocks that other writers
 * made read as the formats define them; values below 2^-126, under scale bytes
 * below 10, count as 0 in the attention.
 *
 * Layouts (row-major, contiguous, 16-byte aligned):
 *   k, v              [pool_pages, Hkv, 16, D] (e4m3) or [pool_pages, Hkv, 16, D / 2] bytes
 *   k_scale, v_scale  [pool_pages, Hkv, 16, D / 32] bytes
 *   all others as in sangam_attn.h and sangam_kv.h, bf16
 *
 * Ownership and errors: as in sangam_attn.h. Plans are those of
 * sangam_attn_plan and sangam_kv_plan; they do not depend on the cache's format.
 */
#ifndef SANGAM_KVQ_H
#define SANGAM_KVQ_H

#include "sangam_attn.h"
#include "sangam_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SANGAM_KV_E4M3 1
#define SANGAM_KV_E2M1 2

/* A pool of quantised pages (device memory, the caller's); read during the call. */
typedef struct sangam_kvq_cache {
    int32_t format;     /* SANGAM_KV_E4M3 or SANGAM_KV_E2M1 */
    int32_t reserved;   /* 0 */
    int64_t pool_pages; /* pages that each of the four arrays holds */
    void *k;
    void *v;
    void *k_scale;
    void *v_scale;
} sangam_kvq_cache;

/*
 * sangam_attn_forward over a quantised cache: the fresh rows are written into
 * the pages quantised, and every query row attends to the cached rows' values
 * and, as in sangam_attn_forward, to the item's own fresh rows as they are in
 * k_new / v_new, unquantised. One call, the same launches. An output is an
 * average of V's rows by softmax weights rounded to bf16; the LSE is that of
 * unrounded ones. Outputs that an infinity or a NaN reaches are infinite or
 * NaN. events: NULL, or the six of sangam_attn_forward_timed. (No form of it
 * takes split partials to a library array as sangam_attn_forward_noalloc does:
 * the workspace is the caller's.)
 * Errors: as sangam_attn_forward, SANGAM_ERR_INVALID_ARG for a NULL cache, and
 * SANGAM_ERR_UNSUPPORTED for an unknown format.
 */
sangam_status sangam_kvq_forward(const void *plan_host, const void *plan_dev, const void *q,
                                 const void *k_new, const void *v_new,
                                 const sangam_kvq_cache *cache, const int32_t *page_ids_dev,
                                 int64_t num_page_ids, void *out, float *lse, void *workspace,
                                 size_t workspace_bytes, void *stream, void *const *events);

/*
 * The copies of sangam_kv.h between quantised pages and packed bf16 rows:
 * export reads pages back into rows, import quantises rows into pages. Slots
 * >= L_i of a request's last page, and pages that the plan does not list, are
 * neither read nor written. Asynchronous on stream: no allocation, no host
 * synchronisation. Errors: SANGAM_ERR_PLAN, SANGAM_ERR_INVALID_ARG (NULL
 * pointers), SANGAM_ERR_UNSUPPORTED (format), SANGAM_ERR_ALIGN,
 * SANGAM_ERR_BUFFER (pool_pages fewer than the plan addresses), SANGAM_ERR_HIP.
 */
sangam_status sangam_kvq_export(const void *plan_host, const void *plan_dev,
                                const sangam_kvq_cache *cache, void *k_packed, void *v_packed,
                                void *stream);
sangam_status sangam_kvq_import(const void *plan_host, const void *plan_dev, const void *k_packed,
                                const void *v_packed, const sangam_kvq_cache *cache, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SANGAM_KVQ_H */
