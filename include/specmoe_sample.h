/*
 * specmoe_sample.h -- sampling of tokens from given random numbers, and the
 * acceptance of draft tokens by sampling, on MI355X (gfx950).
 *
 * A token is drawn from a row of logits x_0 .. x_{V-1} with a uniform number
 * u in [0, 1):
 *
 *   w_i = exp((x_i - max x) / T), the tokens in order of falling x_i, equal
 *   ones by their index.  Kept are, one after the other:
 *     top_k  the first top_k tokens;
 *     top_p  of these the shortest prefix whose share of their mass (the sum
 *            of their w_i) is at least top_p, never less than one token;
 *     min_p  of these the tokens with w_i >= min_p.
 *   The token is the first one of the order whose cumulative share of the kept
 *   mass passes u; its log-probability is log(w_i / kept mass).
 *
 * u = 0 gives the most probable token.  T <= 0 (or NaN) is greedy: the most
 * probable token whatever u, at log-probability 0, by the rule of
 * specmoe_accept_greedy (a row of -inf elects its first one, a row of NaN
 * none).  top_k <= 0 or >= V, top_p >= 1 or NaN, and min_p <= 0 or NaN keep
 * everything; top_p <= 0 keeps one token, min_p >= 1 those equal to the best.
 * u below 0 or NaN counts as 0, u >= 1 as the end of the kept mass.  Logits
 * of -inf are never drawn, nor are NaN ones, which count as -inf; with +inf
 * among the logits, those share the mass.  A row without any mass gives token
 * -1 at log-probability -inf.
 *
 * Weights are computed in fp64 and summed as 64-bit integers, in units of
 * 2^-42 of the best token's: sums are exact, so a result depends neither on
 * the order of the additions nor on timing, nor on the other rows of a call.  A
 * token below half a unit is never drawn and adds nothing to a mass, borders of
 * top_p included.
 *
 * Status codes are the SPECMOE_* values of specmoe_verify.h.  All functions
 * are plain C; pointers named "device" are HIP device pointers.
 */
#ifndef SPECMOE_SAMPLE_H
#define SPECMOE_SAMPLE_H

#include <stddef.h>
#include <stdint.h>

#include "specmoe_accept.h"
#include "specmoe_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Sampling settings, one value per row (specmoe_sample) or sequence; device
 * pointers in a host struct.  A NULL pointer leaves its setting off (T = 1). */
typedef struct specmoe_sampling {
  const float* temperature;  /* T      */
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
} specmoe_sampling;

typedef struct specmoe_sample_desc {
  int32_t N;          /* rows; 0 returns SPECMOE_OK at once                     */
  int32_t V;          /* vocabulary size, in [1, 2^20]                          */
  int32_t dtype;      /* specmoe_dtype of the logits (SPECMOE_F32, SPECMOE_BF16) */
  int32_t flags;      /* reserved, must be 0                                    */
  int64_t stride;     /* elements from one row of logits to the next, >= V;
                         0: V                                                   */
} specmoe_sample_desc;

/*
 * specmoe_sample -- one token for each of N rows.
 *
 *   logits     device, dtype, aligned to its elements: row n starts n stride
 *              elements in.  Any V and stride do; rows at multiples of 16
 *              bytes are read fastest.
 *   uniforms   float32 [N], device: u of each row.
 *   sampling   host struct of device pointers to [N] settings; NULL: all off.
 *   tokens     int32 [N] out, device.
 *   logprobs   float32 [N] out, device; NULL: not wanted.
 *   stream     hipStream_t (NULL: the null stream).
 *
 * The caller owns every buffer; nothing is allocated, nothing synchronises
 * with the host, no workspace is needed, and calls may overlap.  All host
 * checks run before any HIP call: SPECMOE_ERR_NULL_POINTER (desc),
 * SPECMOE_ERR_DTYPE, SPECMOE_ERR_FLAGS, SPECMOE_ERR_SHAPE (N < 0 or >= 2^22, V,
 * stride); then, with N > 0, SPECMOE_ERR_NULL_POINTER, SPECMOE_ERR_ALIGN, and
 * from HIP SPECMOE_ERR_LAUNCH.
 */
int specmoe_sample(const void* logits, const float* uniforms, const specmoe_sampling* sampling, int32_t* tokens,
                   float* logprobs, void* stream, const specmoe_sample_desc* desc);

/*
 * specmoe_accept_sample -- acceptance of a batch of verified chunks by
 * sampling.
 *
 * The rule of specmoe_accept_greedy with a sampled token in the place of the
 * argmax: at every chunk position i < c_b a token s_i is drawn from the
 * logits there with the sequence's settings and u[b, i]; a_b = the number of
 * leading drafts with token[i+1] == s_i; the next token is s_{a_b}.  When the
 * drafts were chosen without looking at u, the tokens that a sequence takes
 * are distributed exactly as if each had been sampled from the target one at
 * a time, whatever the draft model proposes.  With temperature 0 the result
 * is specmoe_accept_greedy's.
 *
 *   uniforms   float32 [B, C_max], device; entries i >= c_b are not used.
 *   sampling   host struct of device pointers to [B] settings; NULL: all off.
 *   sampled    int32 [B, C_max] out: s_i for i < c_b, -1 beyond.
 *   logprobs   float32 [B, C_max] out: the log-probability of s_i, 0 beyond;
 *              NULL: not wanted.
 * Every other argument, the workspace (one can serve both, and its size and
 * initialisation are those of specmoe_accept_greedy; desc->split is ignored),
 * ownership and the errors are those of specmoe_accept_greedy; in addition
 * V <= 2^20 and B C_max < 2^22 (SPECMOE_ERR_SHAPE).
 */
int specmoe_accept_sample(const void* logits, const int32_t* tokens, const int32_t* ctx_lens,
                          const int32_t* chunk_lens, const float* uniforms, const specmoe_sampling* sampling,
                          int32_t* sampled, float* logprobs, int32_t* accepted, int32_t* next_token,
                          int32_t* new_ctx_lens, void* stream, const specmoe_accept_desc* desc);

/*
 * specmoe_accept_sample_tree -- the same for tree drafts: the rule of
 * specmoe_accept_greedy_tree (a node is accepted when its parent is and its
 * token equals the one sampled at the parent; the deepest accepted node wins,
 * the lowest index among equally deep ones).
 *
 *   draft_mask   uint64 [B, C_max], device, 8-byte aligned; C_max <= 64.
 *   path         uint64 [B] out, device, 8-byte aligned.
 */
int specmoe_accept_sample_tree(const void* logits, const int32_t* tokens, const uint64_t* draft_mask,
                               const int32_t* ctx_lens, const int32_t* chunk_lens, const float* uniforms,
                               const specmoe_sampling* sampling, int32_t* sampled, float* logprobs,
                               int32_t* accepted, int32_t* next_token, int32_t* new_ctx_lens, uint64_t* path,
                               void* stream, const specmoe_accept_desc* desc);

#ifdef __cplusplus
}
#endif

#endif /* SPECMOE_SAMPLE_H */
