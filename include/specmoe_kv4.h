/*
 * specmoe_kv4.h -- a KV cache held in 4 bits, on MI355X (gfx950): the append
 * that fills it, the verification and decode attention over it, the move of an
 * accepted tree path's rows, and rows handed back in 16 or 32 bits.
 *
 * Verification and decoding are bound by the bytes of the cache.  Here a head
 * row of D entries takes D / 2 + D / 32 bytes (68 for D = 128, where bfloat16
 * takes 256): blocks of 32 consecutive entries, each with one scale byte and
 * 32 codes of 4 bits.
 *
 *   scale byte e   1..254: the block's unit is 2^(e - 127); 0: 2^-127; 255:
 *                  all of the block's entries are NaN.
 *   code           1 sign bit (8) and 3 bits that stand for 0, 1/2, 1, 3/2, 2,
 *                  3, 4, 6 units.  Entry 2 j is the low half of byte j of the
 *                  row, entry 2 j + 1 the high half.
 *
 * (The element and scale types of the OCP Microscaling format MXFP4.)  A block
 * x is written with the smallest unit u >= 2^-126 at which max |x| / u < 7, so
 * that its largest entry rounds to at most 6 units, none cut down to it; every code
 * is x / u to the nearest value, ties to the even code.  A block that holds an
 * infinity or NaN becomes a NaN block.  Codes of 4 and 6 units with byte 253, and
 * of 2 and more with 254, stand for values from 2^128 on, past the range of
 * float32 and bfloat16: they are infinities wherever values are taken in a type.
 * Of finite entries only those from 1.75 2^127 on come to that (4 units of 2^126).
 *
 * Status codes are the SPECMOE_* values of specmoe_verify.h.  All functions
 * are plain C; pointers named "device" are HIP device pointers.
 */
#ifndef SPECMOE_KV4_H
#define SPECMOE_KV4_H

#include <stddef.h>
#include <stdint.h>

#include "specmoe_append.h"
#include "specmoe_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A 4-bit cache (host struct of device pointers, 16-byte aligned): one slab per
 * sequence, or a pool of pages when a call gets a block table. */
typedef struct specmoe_kv4 {
  void* k_codes;  /* uint8 [B, Hkv, S_max, D / 2] or [num_pages, Hkv, page_size, D / 2]   */
  void* k_scales; /* uint8 [B, Hkv, S_max, D / 32] or [num_pages, Hkv, page_size, D / 32] */
  void* v_codes;  /* as k_codes  */
  void* v_scales; /* as k_scales */
} specmoe_kv4;

/*
 * specmoe_append_kv4 -- specmoe_append_kv into a 4-bit cache.
 *
 * Arguments, positions, norms, rotation, preconditions, ownership and errors
 * are those of specmoe_append_kv, with the cache in place of k_cache and
 * v_cache (SPECMOE_ERR_NULL_POINTER also for a NULL cache or member,
 * SPECMOE_ERR_ALIGN for a misaligned member).  desc->dtype is the type of q, k,
 * v, the weights and q_out.  A key's norm and rotation are computed in fp64 up
 * to its codes, so that a key next to a border between two codes goes to the
 * right one; values are encoded as they are.  Values past float32's largest
 * count as infinities.  Only the rows [l_b, l_b + c_b) are written.
 */
int specmoe_append_kv4(const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight,
                       const double* inv_freq, const int32_t* ctx_lens, const int32_t* chunk_lens,
                       const uint64_t* draft_mask, const int32_t* block_table, void* q_out, const specmoe_kv4* cache,
                       void* stream, const specmoe_append_desc* desc, const specmoe_paged_kv* paged);

/*
 * specmoe_verify_attn_kv4 -- verification attention over a 4-bit cache.
 *
 * The operation of specmoe_verify_attn (chains; C_max = 1 is decoding),
 * specmoe_verify_attn_tree (with a draft_mask) and specmoe_verify_attn_paged
 * (with block_table and paged; both NULL: slabs), on the keys and values that
 * the cache's codes stand for.
 *
 *   q            device, dtype [B, C_max, Hq, D], 16-byte aligned; rows
 *                i >= c_b are never read.
 *   cache        host pointer to the cache.  Rows >= l_b + c_b are never read.
 *   out          device, 16-byte aligned: [B, C_max, Hq, D] of dtype (the type
 *                that the projection after it takes).
 *   lse          device, float32 [B, C_max, Hq].  q, out and lse share no
 *                memory (SPECMOE_ERR_OVERLAP, after all other checks).
 *   desc         as in specmoe_verify_attn; dtype is the type of q and out.
 *                grid_blocks 0: 512 workgroups, two per CU.
 *
 * The codes' products with the queries are summed in fp32, and so are the
 * statistics of the softmax.  Queries are taken exactly, but for entries under
 * 2^-13 of the largest of their block of 32 in a 16-bit type with D = 128: such
 * an entry is off by at most 2^-22 (bfloat16) or 2^-27 (float16) of that largest
 * one.  A query that holds an infinity or NaN gets NaN, and so does one whose
 * score with a key it sees passes float32's range upwards, or downwards with every
 * key that it sees; a key whose score alone passes it downwards (-inf) has no
 * weight.  For their product with the values, probabilities are rounded to
 * bfloat16 when dtype is bfloat16, and kept to 16 bits for float16 and 24 for
 * float32.  Padding rows and tokens that see no key get out = 0 and lse = -inf.
 * Keys that a token does not see leave its results
 * alone whatever they hold, NaN blocks and values past float32's range included.
 * Such values are infinities to the tokens that see them: their entries of the
 * result are infinities or NaN.  (Sums over the values are divided by the
 * probabilities' sum at the end and taken with weights up to 2^8 until then: over
 * 2^24 keys values from 2^96 on can pass float32's range on the way, and become
 * infinities too.)
 *
 * The workspace is one of specmoe_verify_attn (same zeroed region, initialised
 * by specmoe_verify_attn_workspace_init) of at least
 * specmoe_verify_attn_kv4_workspace_bytes; calls of the two can share it, one
 * after the other.  Preconditions, clamping, ownership and determinism are those
 * of specmoe_verify_attn, and so are the errors (of specmoe_verify_attn_paged
 * with a table; SPECMOE_ERR_NULL_POINTER also for a NULL cache or member or a
 * table without its geometry).  desc->flags must be 0 (SPECMOE_ERR_FLAGS):
 * nothing waits in these kernels.
 */
int specmoe_verify_attn_kv4(const void* q, const specmoe_kv4* cache, const int32_t* block_table,
                            const int32_t* ctx_lens, const int32_t* chunk_lens, const uint64_t* draft_mask, float scale,
                            void* out, float* lse, void* stream, const specmoe_verify_desc* desc,
                            const specmoe_paged_kv* paged);

/* Bytes of workspace specmoe_verify_attn_kv4 needs for `desc`; 0 for an invalid
 * descriptor.  At least specmoe_verify_attn_workspace_bytes(desc). */
size_t specmoe_verify_attn_kv4_workspace_bytes(const specmoe_verify_desc* desc);

/* Sizes of the calls that read and move rows (host struct). */
typedef struct specmoe_kv4_desc {
  int32_t B;      /* sequences; 0 returns SPECMOE_OK at once                   */
  int32_t Hkv;    /* KV heads                                                  */
  int32_t D;      /* head dimension: 64 or 128                                 */
  int32_t N_max;  /* rows of k_out and v_out per sequence (specmoe_read_kv4)   */
  int32_t S_max;  /* token capacity of the cache per (sequence, KV head)       */
  int32_t dtype;  /* specmoe_dtype of k_out and v_out (specmoe_read_kv4)       */
} specmoe_kv4_desc;

/*
 * specmoe_read_kv4 -- rows of a 4-bit cache as the values they stand for.
 *
 * For every sequence b and i < n_b, the rows f_b + i of its KV heads go to
 * k_out[b, i] and v_out[b, i]: a prefix for a cache of 16 bits, a prompt's rows
 * for its own attention, a request for another machine.  Values are exact in
 * float32 and bfloat16, rounded once (to nearest even) in float16; those past the
 * type's range are infinities.
 *
 *   first        int32 [B], device: f_b (clamped to >= 0).
 *   rows         int32 [B], device: n_b (clamped into [0, N_max]).
 *   block_table  as in specmoe_verify_attn_paged, with paged; both NULL: slabs.
 *   k_out, v_out device, dtype [B, N_max, Hkv, D], 16-byte aligned.  Rows
 *                i >= n_b, rows past S_max and rows of pages outside the pool
 *                are left as they are.
 * Asynchronous on `stream`; allocates nothing.  Errors, in this order:
 * SPECMOE_ERR_NULL_POINTER (desc), SPECMOE_ERR_DTYPE, SPECMOE_ERR_HEAD_DIM,
 * SPECMOE_ERR_SHAPE (B < 0, Hkv, N_max or S_max < 1, Hkv > 2^20,
 * B N_max >= 2^31 or B * ceil(N_max / 4) >= 2^24 - 1), SPECMOE_ERR_PAGES; then, with
 * B > 0, SPECMOE_ERR_NULL_POINTER, SPECMOE_ERR_ALIGN, SPECMOE_ERR_LAUNCH.
 */
int specmoe_read_kv4(const specmoe_kv4* cache, const int32_t* block_table, const int32_t* first, const int32_t* rows,
                     void* k_out, void* v_out, void* stream, const specmoe_kv4_desc* desc,
                     const specmoe_paged_kv* paged);

/*
 * specmoe_compact_accepted_kv4 -- specmoe_compact_accepted_kv for a 4-bit
 * cache, in slabs or pages: the rows l_b + k of the set bits k of path[b]
 * (ascending) move to rows l_b + 0, 1, ...; all rows are read before any is
 * written.  Rows past S_max or in pages outside the pool are neither read nor
 * written.  Pages must not be shared between sequences in the rows that move.
 *
 *   ctx_lens     int32 [B], device: l_b before the step.
 *   path         uint64 [B], device, 8-byte aligned.
 *   desc         B, Hkv, D and S_max are used.
 * Asynchronous on `stream`; allocates nothing.  Errors as specmoe_read_kv4's
 * without SPECMOE_ERR_DTYPE (SPECMOE_ERR_SHAPE also for B Hkv >= 2^23).
 */
int specmoe_compact_accepted_kv4(const specmoe_kv4* cache, const int32_t* block_table, const int32_t* ctx_lens,
                                 const uint64_t* path, void* stream, const specmoe_kv4_desc* desc,
                                 const specmoe_paged_kv* paged);

#ifdef __cplusplus
}
#endif

#endif /* SPECMOE_KV4_H */
