/*
 * specmoe_append.h -- a chunk's queries, keys and values put in place for the
 * verification attention, on MI355X (gfx950).
 *
 * specmoe_verify_attn (specmoe_verify.h) takes rotated queries and a KV cache
 * that already holds the chunk's own rows.  This step makes them from the
 * projections' output: for every sequence b and draft token i < c_b, at
 * position
 *
 *   pos = l_b + i                          (chain drafts)
 *   pos = l_b + max(seen, 1) - 1           (tree drafts; seen: the draft tokens
 *                                           k < c_b in token i's mask word,
 *                                           itself among them)
 *
 * and for every head row x (D entries) of q and k:
 *
 *   norm      (with a weight)  x <- x / sqrt(mean(x^2) + eps) * weight
 *   rotation  (rot_dim > 0)    with angle_j = pos * inv_freq[j],
 *                              j < rot_dim / 2, and the pair (x_a, x_b):
 *                              x_a <- x_a cos - x_b sin, x_b <- x_b cos + x_a sin;
 *                              SPECMOE_ROPE_HALVES: a = j, b = j + rot_dim / 2,
 *                              SPECMOE_ROPE_PAIRS:  a = 2 j, b = 2 j + 1;
 *                              entries from rot_dim on stay
 *
 * q goes to q_out, k and (unchanged) v to row l_b + i of the sequence's cache,
 * one slab per sequence or pages.  The arithmetic is in fp32 (the angles in
 * fp64, so that far positions lose nothing) with one rounding to dtype at the
 * end.  Prompts go in the same way: C_max has no upper limit here.
 *
 * Status codes are the SPECMOE_* values of specmoe_verify.h.  All functions
 * are plain C; pointers named "device" are HIP device pointers.
 */
#ifndef SPECMOE_APPEND_H
#define SPECMOE_APPEND_H

#include <stddef.h>
#include <stdint.h>

#include "specmoe_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Which two entries of a head row are rotated together. */
typedef enum {
  SPECMOE_ROPE_HALVES = 0, /* j and j + rot_dim / 2 */
  SPECMOE_ROPE_PAIRS = 1   /* 2 j and 2 j + 1       */
} specmoe_rope_style;

typedef struct specmoe_append_desc {
  int32_t B;          /* sequences; 0 returns SPECMOE_OK at once                        */
  int32_t Hq;         /* query heads; 0: keys and values only (q, q_out ignored)        */
  int32_t Hkv;        /* KV heads                                                       */
  int32_t D;          /* head dimension: 64 or 128                                      */
  int32_t C_max;      /* chunk capacity: token rows of q, k, v, q_out per sequence      */
  int32_t S_max;      /* token capacity of the KV cache per (sequence, KV head)         */
  int32_t dtype;      /* specmoe_dtype of q, k, v, the weights, q_out and the cache     */
  int32_t rot_dim;    /* rotated entries of a head row: a multiple of 16 up to D, or 0  */
  int32_t rope_style; /* specmoe_rope_style                                             */
  float norm_eps;     /* eps of the norms; finite and >= 0                              */
  int64_t q_stride;   /* elements from one token's row of q (k, v) to the next token's; */
  int64_t k_stride;   /* 0: Hq D (Hkv D).  A row's heads lie side by side.  At least    */
  int64_t v_stride;   /* the row's length, and a multiple of 16 bytes                   */
} specmoe_append_desc;

/*
 * specmoe_append_kv
 *
 *   q, k, v      device, dtype, 16-byte aligned: the row of token i of
 *                sequence b starts (b C_max + i) stride elements in.  Rows
 *                i >= c_b are never used.
 *   q_weight     device, dtype [D], 16-byte aligned, shared by the query
 *   k_weight     (key) heads; NULL: no norm.
 *   inv_freq     device, float64 [rot_dim / 2], 8-byte aligned; not looked at
 *                with rot_dim = 0.
 *   ctx_lens     int32 [B], device: l_b.
 *   chunk_lens   int32 [B], device: c_b.
 *   draft_mask   uint64 [B, C_max], device, 8-byte aligned: the words of
 *                specmoe_verify_attn_tree, whose positions the tokens get;
 *                NULL: chain drafts (or a prompt).  C_max <= 64 with it.
 *   block_table  int32 [B, pages_per_seq], device, with paged: the cache is
 *                the pool of pages of specmoe_verify_attn_paged.  Both NULL:
 *                a slab per sequence.
 *   q_out        device, dtype [B, C_max, Hq, D], 16-byte aligned; rows
 *                i >= c_b are left as they are.  May be q itself when q's rows
 *                are contiguous.
 *   k_cache      device, dtype, 16-byte aligned: [B, Hkv, S_max, D], or
 *   v_cache      [num_pages, Hkv, page_size, D].  Only the rows
 *                [l_b, l_b + c_b) are written.
 *   stream       hipStream_t (NULL: the null stream).
 *
 * Device-side preconditions (the lengths live in device memory): l_b >= 0,
 * 0 <= c_b <= C_max, l_b + c_b <= S_max, table entries in [0, num_pages), no
 * page row written twice.  c_b and a negative l_b are clamped; a K/V row
 * past S_max or in a page outside the pool is not written.
 *
 * Ownership as in specmoe_verify_attn: the caller owns every buffer, nothing
 * is allocated, nothing synchronises with the host, no workspace is needed.
 * All host checks run before any HIP call.  Errors, in this order:
 * SPECMOE_ERR_NULL_POINTER (desc), SPECMOE_ERR_DTYPE, SPECMOE_ERR_HEAD_DIM,
 * SPECMOE_ERR_SHAPE (B, Hq < 0, Hkv, C_max or S_max < 1, B C_max >= 2^23,
 * Hq or Hkv > 2^20, a bad stride), SPECMOE_ERR_ROPE (rot_dim, rope_style or
 * norm_eps), SPECMOE_ERR_MASK, SPECMOE_ERR_PAGES; then, with B > 0,
 * SPECMOE_ERR_NULL_POINTER, SPECMOE_ERR_ALIGN, and from HIP
 * SPECMOE_ERR_LAUNCH.
 */
int specmoe_append_kv(const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight,
                      const double* inv_freq, const int32_t* ctx_lens, const int32_t* chunk_lens,
                      const uint64_t* draft_mask, const int32_t* block_table, void* q_out, void* k_cache,
                      void* v_cache, void* stream, const specmoe_append_desc* desc, const specmoe_paged_kv* paged);

#ifdef __cplusplus
}
#endif

#endif /* SPECMOE_APPEND_H */
