/*
 * sangam_sample.h - C ABI of what follows the logits of a diffusion-LLM decode
 * step, for AMD Instinct MI355X (gfx950): a token and a confidence for every
 * row, and the rows of each block that take their token (the paper's
 * confidence-threshold sampler).
 *
 * Device arrays of parameters are read as they are when the launch runs. No
 * value of them leads a kernel out of the buffers whose sizes the call gives.
 *
 * Ownership and errors: as in sangam_attn.h.
 */
#ifndef SANGAM_SAMPLE_H
#define SANGAM_SAMPLE_H

#include "sangam_attn.h"
#include "sangam_rope.h" /* SANGAM_DTYPE_* */

#ifdef __cplusplus
extern "C" {
#endif

#define SANGAM_CONFIDENCE_PROBABILITY 0
#define SANGAM_CONFIDENCE_MARGIN 1
#define SANGAM_CONFIDENCE_ENTROPY 2

/*
 * Rows of logits and how to take a token from each. A row's tokens are ranked
 * by logit, the largest first, equal ones by index. With the largest logit X
 * and the temperature T, token i has the weight w_i = exp((x_i - X) / T). Kept
 * is the first token and, as long as all that is asked for holds, those behind:
 *   top_k > 0          rank < top_k
 *   top_p < 1          the weight of the ranks before it is under top_p times
 *                      that of all (of the first top_k)
 *   min_p > 0          (x_i - X) / T >= ln(min_p)
 * M is the weight of the kept ones. The row's token is the first in rank order
 * up to which the kept weight is above u M (u <= 0: the first; u >= 1: the last
 * of any weight). T = 0 takes the first token; its confidence is that of T = 1.
 * Confidence:
 *   PROBABILITY  w / M of the token
 *   MARGIN       that of the first token less that of the second (0 where only
 *                one is kept)
 *   ENTROPY      sum p ln p over the kept ones, <= 0
 *
 * A logit that is -inf or no number has no weight and is never taken; +inf
 * shares the whole weight with its like. A row without any weight gets token
 * -1, confidence 0. Weights under 2^-64 of the largest count as none; of fp16 and
 * fp32 rows, those up to 2^-63.9 of it may.
 *
 * Logits are exact. Places are found by weights held to 2^-33 of themselves:
 * fp16 and fp32 rows sum them as whole numbers of 2^-44 of the largest, bf16 rows
 * in 64 bits in an order that is always the same. So a row's token does not
 * depend on when what is added, nor on the rows beside it, and equal logits share
 * alike. Confidences come from the same sums, but for the first token of
 * everything of fp16 and fp32 rows (T = 0, nothing filtered): its weights are
 * computed in 32 bits and summed in 32 over a few, then in 64, to 2^-19 of the sum.
 * Within that error these hang on the number of rows as well (rows are summed in
 * parts where there are few), and with them which rows are at a threshold; all
 * other confidences are a row's own, to the last bit.
 *
 * Parameters: an array has num_params entries, of which row r takes entry
 * params_of[r] (NULL: r); a NULL array stands for the value beside it. A row
 * whose entry is outside gets token -1, confidence 0, and its logits are not
 * read (rows that pad a batch). In an array, a temperature that is not above 0
 * counts as 0, top_k below 1, top_p not below 1 and min_p not above 0 as none.
 */
typedef struct sangam_sample_desc {
    const void *logits;      /* [rows, vocab], consecutive in a row */
    int64_t rows;            /* 0 to 2^31 - 1 */
    int64_t row_stride;      /* in elements, 0 to 2^40 */
    int32_t vocab;           /* 1 to 2^18 */
    int32_t dtype;           /* SANGAM_DTYPE_* */
    const float *u;          /* [rows] */
    const int32_t *params_of; /* [rows] or NULL */
    int64_t num_params;
    const float *temperatures;
    const int32_t *top_ks;
    const float *top_ps;
    const float *min_ps;
    float temperature;       /* >= 0 */
    int32_t top_k;           /* >= 0; 0: no limit */
    float top_p;             /* 0 to 1 */
    float min_p;             /* 0 to 1 */
    int32_t confidence;      /* SANGAM_CONFIDENCE_* */
    int32_t forbid;          /* a token that no row takes, as if its logit were -inf; or -1 */
} sangam_sample_desc;

/* Bytes of the workspace that sangam_sample_tokens needs for a descriptor's rows, vocab and dtype (0: none). */
size_t sangam_sample_workspace_bytes(int64_t rows, int32_t vocab, int32_t dtype);

/*
 * tokens [rows] and confidence [rows] (device; confidence may be NULL) on
 * `stream`. Asynchronous: no allocation, no host synchronisation. The workspace
 * (device, 256-byte aligned) needs no content and holds nothing after the call;
 * calls that may overlap need one each.
 * Errors: SANGAM_ERR_INVALID_ARG (a NULL pointer, a size, stride or value out
 * of range), SANGAM_ERR_UNSUPPORTED (dtype), SANGAM_ERR_ALIGN (a pointer not
 * aligned to its elements), SANGAM_ERR_BUFFER (a short workspace),
 * SANGAM_ERR_HIP.
 */
sangam_status sangam_sample_tokens(const sangam_sample_desc *desc, int32_t *tokens, float *confidence, void *workspace,
                                   size_t workspace_bytes, void *stream);

/*
 * The rows of every block that take their token. Block i is rows row_indptr[i]
 * to row_indptr[i + 1]; row r's id is ids[r], or with slots ids[slots[r]] (the
 * slots of sangam_tables_build: ids lie as the KV does). A row is a candidate if
 * its id is mask_id and its token is neither negative nor mask_id. It takes its
 * token if its confidence is at least the block's threshold, or if it is among
 * the block's `count` most confident candidates (equal ones: the lower row; no
 * number: the least).
 *   out [rows]   ids after the step
 *   left [num_blocks] (may be NULL)  rows of the block whose id is still mask_id
 * With slots, ids[slots[r]] of a row that takes its token becomes that token;
 * without, ids stays as it is (out may be ids). A row whose slot is outside
 * [0, num_ids) has no id: out is -1. No slot may stand twice. Rows outside all
 * blocks keep their id.
 */
typedef struct sangam_unmask_desc {
    const int32_t *tokens;     /* [rows] */
    const float *confidence;   /* [rows] */
    int32_t *ids;              /* [num_ids]; num_ids is rows without slots */
    const int64_t *slots;      /* [rows] or NULL */
    const int32_t *row_indptr; /* [num_blocks + 1], not decreasing */
    const int32_t *counts;     /* [num_blocks], or NULL: count */
    const float *thresholds;   /* [num_blocks], or NULL: threshold */
    int64_t rows;              /* 0 to 2^31 - 1 */
    int64_t num_ids;
    int32_t num_blocks;        /* 0 to 4 (2^24 - 1) */
    int32_t mask_id;
    int32_t count;             /* >= 0 (in counts: below 0 counts as 0) */
    float threshold;           /* a number or infinity (in thresholds: no number is never reached) */
} sangam_unmask_desc;

/* One launch on `stream`, without allocation or host synchronisation. Errors: as sangam_sample_tokens. */
sangam_status sangam_sample_unmask(const sangam_unmask_desc *desc, int32_t *out, int32_t *left, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SANGAM_SAMPLE_H */
