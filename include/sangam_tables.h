/*
 * sangam_tables.h - C ABI of the page tables of a paged KV cache on the device,
 * for AMD Instinct MI355X (gfx950): a block table that follows the lengths of
 * its requests, and what a batch's calls read of it (page list, positions,
 * slots), so that lengths are all that the host sends from one iteration to
 * the next.
 *
 * A page holds 16 positions. The block table is int32 [requests, max_pages]:
 * entry (r, j) is the page of positions [16 j, 16 j + 16) of request r, -1
 * behind its last one.
 *
 * Device arrays are read as they are when the launch runs. No entry of them
 * leads a kernel out of the buffers whose sizes the call gives: what points
 * outside is handled as said below. The host arguments are checked.
 *
 * Ownership and errors: as in sangam_attn.h.
 */
#ifndef SANGAM_TABLES_H
#define SANGAM_TABLES_H

#include "sangam_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sangam_block_table {
    int32_t *pages;      /* device, [requests, max_pages] */
    int64_t row_stride;  /* in entries, >= max_pages */
    int32_t requests;    /* 0 to 2^30 */
    int32_t max_pages;   /* of a request, >= 0 */
} sangam_block_table;

/*
 * Every request r of the table gets exactly ceil(lengths[r] / 16) pages, in one
 * launch on `stream` (no allocation, no host synchronisation):
 *   1. A request that holds more gives its last ones back, requests in order,
 *      onto the stack `free` above its num_free entries, so that the first
 *      request's first page comes off first; its entries become -1.
 *   2. A request that holds fewer takes the rest off the stack, requests in
 *      order, the top first. One that the stack does not hold enough for takes
 *      none, nor does any later one.
 * held[r] (pages that r holds) and num_free[0] follow. short_of[0] becomes the
 * number of requests that got none of what they wanted, or whose length is
 * beyond max_pages (they keep what they have).
 *
 * lengths below 0 count as 0; held[r] as at most max_pages, num_free[0] as at
 * most free_cap. Pages that come back to a full stack of free_cap are lost: give
 * it room for all pages. Entries of `free` above the top are left as they are, and so
 * are those of the table that nothing moves into or out of.
 *
 * Errors: SANGAM_ERR_INVALID_ARG (a NULL pointer, a size out of range),
 * SANGAM_ERR_ALIGN (a pointer not 4-byte aligned), SANGAM_ERR_HIP.
 */
sangam_status sangam_tables_resize(const sangam_block_table *table, int32_t *held, const int32_t *lengths,
                                   int32_t *free_pages, int32_t free_cap, int32_t *num_free, int32_t *short_of, void *stream);

/* A batch over some requests of a table: item i is request request[i] (NULL:
 * i), whose kv_len[i] positions its rows attend to; its rows are q_indptr[i] to
 * q_indptr[i + 1], at positions q_offset[i] and on, or where q_pos is not NULL
 * at q_pos[row]. All device arrays; q_pos holds `rows` entries. */
typedef struct sangam_tables_batch {
    int32_t num_items; /* 0 to 2^30 */
    int32_t reserved;  /* 0 */
    const int32_t *request;  /* [num_items] or NULL */
    const int32_t *kv_len;   /* [num_items] */
    const int32_t *q_indptr; /* [num_items + 1], not decreasing */
    const int32_t *q_offset; /* [num_items] */
    const int32_t *q_pos;    /* [rows] or NULL */
} sangam_tables_batch;

/*
 * What the batch's calls read, in one launch (two from 1025 items on), without
 * allocation or host synchronisation:
 *   page_indptr [num_items + 1]  pages before each item, ceil(kv_len / 16) each
 *                                (at most max_pages)
 *   page_ids [pages]             the items' pages one after the other; -1 where
 *                                the table has none, and behind the last item
 *   positions [rows]             of every row
 *   slots [rows]                 16 page + position mod 16, int64: where the
 *                                row's KV lies in the pool; -1 where its
 *                                position is outside [0, kv_len), or the table
 *                                has no page for it
 *   items [rows]                 of every row
 * Rows before the first or behind the last item get position 0, slot -1, item
 * -1. What exceeds `pages` or `rows` is not written. Any output may be NULL but
 * page_indptr.
 *
 * An item whose request is outside the table has no page. An entry -1 of
 * page_ids must not reach sangam_attn_forward.
 *
 * Errors: as sangam_tables_resize (slots must be 8-byte aligned).
 */
sangam_status sangam_tables_build(const sangam_block_table *table, const sangam_tables_batch *batch, int32_t *page_indptr,
                                  int32_t *page_ids, int64_t pages, int32_t *positions, int64_t *slots, int32_t *items,
                                  int64_t rows, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SANGAM_TABLES_H */
