/*
 * specmoe_pages.h -- block tables and slot maps of a paged KV cache made on
 * the GPU from the requests' lengths, on MI355X (gfx950).
 *
 * The paged calls (specmoe_verify_attn_paged, specmoe_append_kv and the others)
 * take a block table.  Acceptance updates the lengths on the GPU, so a table
 * that follows them needs no copy to the host: this step hands every request
 * the pages that its next chunk needs and takes back those that it no longer
 * does.
 *
 * Status codes are the SPECMOE_* values of specmoe_verify.h.  All functions
 * are plain C; pointers named "device" are HIP device pointers.
 */
#ifndef SPECMOE_PAGES_H
#define SPECMOE_PAGES_H

#include <stddef.h>
#include <stdint.h>

#include "specmoe_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Sizes (host struct). */
typedef struct specmoe_pages_desc {
  int32_t B;             /* requests (rows of the table); 0 returns SPECMOE_OK at once */
  int32_t C_max;         /* chunk capacity: columns of slots                           */
  int32_t page_size;     /* tokens per page: a power of two in [8, 65536]              */
  int32_t pages_per_seq; /* columns of the block table                                 */
  int32_t num_pages;     /* entries of free_pages                                      */
} specmoe_pages_desc;

/*
 * specmoe_assign_pages
 *
 * Request b needs n_b = ceil((l_b + c_b) / page_size) pages and holds h_b, the
 * first entries of its row of the table.
 *   1. Requests with h_b > n_b give back the entries [n_b, h_b): they go on the
 *      stack of free pages, requests in order, entries in order.  (l_b = c_b = 0:
 *      a request that has ended gives back all.)
 *   2. Requests with h_b < n_b then take n_b - h_b pages each off the top of
 *      the stack, in order: entry h_b first, the top page first.  The first request
 *      that finds too few gets none, and neither does any after it.
 * Entries of a row past its pages keep what they held, and so do those of the
 * stack past its top (after step 1).
 *
 *   ctx_lens     int32 [B], device: l_b (clamped to >= 0).
 *   chunk_lens   int32 [B], device: c_b (clamped into [0, C_max]); l_b + c_b is
 *                clamped to page_size * pages_per_seq.
 *   block_table  int32 [B, pages_per_seq], device, in and out.
 *   held         int32 [B], device, in and out: h_b (clamped into
 *                [0, pages_per_seq]).
 *   free_pages   int32 [num_pages], device, in and out: the stack, its bottom
 *                first; not part of the table's memory.
 *   free_count   int32 [1], device, in and out: pages on the stack (clamped into
 *                [0, num_pages]).
 *   missing      int32 [B], device, out: the pages that a request which needs
 *                more did not get; 0 for all others.  May be NULL.
 *   slots        int64 [B, C_max], device, 8-byte aligned, out: of token
 *                i < c_b, page * page_size + row of position l_b + i; -1 where
 *                the request holds no page for it, and for i >= c_b.  May be
 *                NULL.
 *   stream       hipStream_t (NULL: the null stream).
 *
 * A precondition: no page is held or free twice (then the stack never
 * overflows; what would pass its end is dropped).  The result depends on the
 * arguments alone, not on timing.  The caller owns every buffer, nothing is
 * allocated, nothing synchronises with the host.
 *
 * Errors, in this order: SPECMOE_ERR_NULL_POINTER (desc), SPECMOE_ERR_SHAPE
 * (B < 0, B >= 2^16, C_max < 1, B C_max >= 2^31 with slots), SPECMOE_ERR_PAGES (page_size,
 * pages_per_seq or num_pages < 1, page_size pages_per_seq >= 2^31, B
 * pages_per_seq >= 2^31); then, with B > 0, SPECMOE_ERR_NULL_POINTER,
 * SPECMOE_ERR_ALIGN, and from HIP SPECMOE_ERR_LAUNCH.
 */
int specmoe_assign_pages(const int32_t* ctx_lens, const int32_t* chunk_lens, int32_t* block_table, int32_t* held,
                         int32_t* free_pages, int32_t* free_count, int32_t* missing, int64_t* slots,
                         void* stream, const specmoe_pages_desc* desc);

#ifdef __cplusplus
}
#endif

#endif /* SPECMOE_PAGES_H */
