/*
 * sangam_rope.h - C ABI of rotary positions, for AMD Instinct MI355X (gfx950):
 * q and k of a batch rotated at their rows' positions, the step between the
 * projections and the attention call of sangam_attn.h.
 *
 * The first rot_dim = R dims of every head are R / 2 pairs; pair j of a row at
 * position p turns by the angle p f_j, with size m:
 *   y0 = m (x0 cos(p f_j) - x1 sin(p f_j))
 *   y1 = m (x1 cos(p f_j) + x0 sin(p f_j))
 * Pair j is dims (j, j + R / 2), or with `interleaved` (2 j, 2 j + 1). Dims R
 * and above pass unchanged. The transpose (sin negated, m kept) is the
 * gradient with respect to x, and for m = 1 the inverse.
 *
 * Rates, f_j = base^(-2 j / R) unscaled; contexts s = factor times longer than
 * the original_len positions that a model was trained on:
 *   SANGAM_ROPE_LINEAR  f_j / s
 *   SANGAM_ROPE_NTK     base s^(R / (R - 2)) in the place of base
 *   SANGAM_ROPE_YARN    g f_j + (1 - g) f_j / s, g = (t - beta_slow) /
 *                       (beta_fast - beta_slow) clipped to [0, 1], t =
 *                       original_len f_j / 2 pi the turns of the pair over the
 *                       original length; m = 0.1 ln(s) + 1 (Peng et al., 2023,
 *                       by the paper's equations)
 *   SANGAM_ROPE_YARN_INDEX  the same with another ramp, linear in the pair and
 *                       not in its turns: g = (hi - j) / (hi - lo) clipped to
 *                       [0, 1], lo = floor(i(beta_fast)) within [0, R - 1] and
 *                       hi = min(R - 1, ceil(i(beta_slow))), i(t) = R ln(original_len
 *                       / 2 pi t) / (2 ln base) the index at which a pair turns
 *                       t times (a step behind lo where hi = lo). It is the one
 *                       that released YaRN checkpoints are trained and served
 *                       with; rates between the two ends differ (R 128, base
 *                       10^6, original_len 32768, s 4: 16 pairs, by up to 1.7)
 * m is 1 otherwise, and `magnitude` in either case where that is not 0.
 *
 * Rates and angles are computed in 64 bits, and turns reduced there: an angle is
 * off by a few 2^-53 of itself where R is a power of two, by ln(base) 2^-53 more
 * elsewhere, and with both YARN by up to s 2^-50 (at 2^31 positions the fastest
 * pair is off by 2^-20 rad). The rotation is done in fp32 and rounded once.
 * Positions are any int32, in any order.
 *
 * Ownership and errors: as in sangam_attn.h.
 */
#ifndef SANGAM_ROPE_H
#define SANGAM_ROPE_H

#include "sangam_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SANGAM_ROPE_NONE 0
#define SANGAM_ROPE_LINEAR 1
#define SANGAM_ROPE_NTK 2
#define SANGAM_ROPE_YARN 3
#define SANGAM_ROPE_YARN_INDEX 4

#define SANGAM_DTYPE_BF16 0
#define SANGAM_DTYPE_FP16 1
#define SANGAM_DTYPE_FP32 2

typedef struct sangam_rope_desc {
    int32_t rot_dim;     /* R: even, 2 to 512 (4 at least for SANGAM_ROPE_NTK) */
    int32_t interleaved; /* 0 or 1 */
    int32_t scaling;     /* SANGAM_ROPE_* */
    int32_t reserved;    /* 0 */
    double base;         /* > 1 */
    double factor;       /* s >= 1; read unless scaling is SANGAM_ROPE_NONE */
    double original_len; /* > 0; both SANGAM_ROPE_YARN (_INDEX: so long that hi >= lo) */
    double beta_fast;    /* > beta_slow; both SANGAM_ROPE_YARN (32 in the paper) */
    double beta_slow;    /* >= 0; both SANGAM_ROPE_YARN (1 in the paper) */
    double magnitude;    /* m, or 0: 0.1 ln(s) + 1 with both SANGAM_ROPE_YARN, else 1 */
} sangam_rope_desc;

/*
 * Host only (no HIP call). Validates the descriptor and writes a position
 * independent plan into plan_buf; the caller copies the same bytes to device
 * memory. SANGAM_ERR_BUFFER with *used = the bytes needed where cap is too
 * small (plan_buf may be NULL with cap 0 to ask); SANGAM_ERR_INVALID_ARG.
 */
sangam_status sangam_rope_plan(const sangam_rope_desc *desc, void *plan_buf, size_t cap, size_t *used);

/* A tensor [rows, heads, head_dim] and its rotated one. Strides count elements;
 * the dims of a head are consecutive. Views of a fused projection's output and
 * both orders of rows and heads are such tensors. */
typedef struct sangam_rope_tensor {
    const void *in;
    void *out; /* in itself (with its strides), or memory that no input overlaps */
    int64_t in_row_stride;   /* >= 0 */
    int64_t in_head_stride;  /* >= 0 */
    int64_t out_row_stride;  /* no two (row, head) of out may overlap */
    int64_t out_head_stride;
    int32_t heads;           /* 1 to 65536 */
    int32_t reserved;        /* 0 */
} sangam_rope_tensor;

/*
 * Rotates q and k (k may be NULL) on `stream` in one launch: row r at position
 * positions_dev[r]. Asynchronous: no allocation, no host synchronisation.
 * plan_host is the plan in host memory, plan_dev the same bytes in device
 * memory. head_dim is R to 512; rows 0 or more; dtype a SANGAM_DTYPE_*;
 * transpose 0 or 1.
 * Strides are 2^40 at most, rows and heads times theirs 2^48; the stride of a
 * single row or head is not read.
 * Errors: SANGAM_ERR_PLAN, SANGAM_ERR_INVALID_ARG (a NULL pointer, a size or
 * stride out of range), SANGAM_ERR_UNSUPPORTED (dtype), SANGAM_ERR_ALIGN (a
 * pointer not aligned to its elements), SANGAM_ERR_HIP. An output that may
 * share an element with an input (but for itself in place) or with the other
 * output is SANGAM_ERR_INVALID_ARG: where the spans of the two overlap, unless
 * both step from row to row alike and lie side by side in the rows.
 */
sangam_status sangam_rope_rotate(const void *plan_host, const void *plan_dev, const sangam_rope_tensor *q,
                                 const sangam_rope_tensor *k, int32_t head_dim, int32_t dtype,
                                 const int32_t *positions_dev, int64_t rows, int32_t transpose,
                                 void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SANGAM_ROPE_H */
