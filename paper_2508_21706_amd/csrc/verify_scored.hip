// Verification attention with scores of their own (capped, lowered with the
// distance, hidden by a window or a first key) for MI355X (gfx950, CDNA4): the
// kernel of verify_kernel.h with the scores' changes compiled in, so the calls
// without them keep theirs.
//
// The changes cost the consumer waves a few instructions per score and the
// stream nothing; what a window or a first key hides from all of a sequence's
// tokens is neither loaded nor scheduled.
//
// Where the stream binds, the calls run as those without changes (64 sequences
// of 512 to 2048 keys, chunks of 5, bf16, capped: 350 MB in 66 us, 5.3 TB/s; 32
// of 16384 to 32768, capped, with starts: 2.6 GB in 399 us, 6.5 TB/s).  With four
// and more 16-row blocks per KV head the consumers do: trees of 16 with slopes
// 83 us for 359 MB, ragged chunks of 1 to 16 under a window of 1024 in pages
// 66 us for 270 MB.
//
// The capped figures are of scores within a quarter of the cap, the series of
// cap_scores.  With larger ones in every wave (an eighth of the scores of 64
// sequences, two fifths of the long ones'), which take the exponential, they are
// 65.7 -> 67.7 us, 397 -> 396 and, capped trees of 16, 83.9 -> 91.3.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "specmoe_verify.h"
#include "verify_kernel.h"

extern "C" int specmoe_verify_attn_scored(const void* q, const void* k_cache, const void* v_cache,
                                          const int32_t* block_table, const int32_t* ctx_lens,
                                          const int32_t* chunk_lens, const uint64_t* draft_mask, float scale, void* out,
                                          float* lse, void* stream, const specmoe_verify_desc* desc,
                                          const specmoe_paged_kv* paged, const specmoe_score* score) {
  if (!score) return SPECMOE_ERR_NULL_POINTER;
  const bool tree = draft_mask != nullptr;
  int st = validate_call(desc, tree, paged);
  if (st != SPECMOE_OK) return st;
  if (!(score->softcap >= 0.f) || !isfinite(score->softcap) || score->window < 0) return SPECMOE_ERR_SCORE;
  if (block_table && !paged) return SPECMOE_ERR_NULL_POINTER;
  if (desc->B == 0) return SPECMOE_OK;   // nothing to read or write
  ScoredParams p;
  Plan pl;
  st = make_params(q, k_cache, v_cache, ctx_lens, chunk_lens, draft_mask, tree, scale, out, lse, desc, block_table,
                   paged, p, pl);
  if (st != SPECMOE_OK) return st;
  if ((reinterpret_cast<uintptr_t>(score->slopes) | reinterpret_cast<uintptr_t>(score->starts)) & 3u)
    return SPECMOE_ERR_ALIGN;
  p.cap_in = score->softcap > 0.f ? scale / score->softcap : 0.f;
  if (!isfinite(p.cap_in)) return SPECMOE_ERR_SCORE;
  p.cap2 = score->softcap * kLog2e;
  p.slopes = score->slopes;
  p.starts = score->starts;
  p.window = score->window;
  (void)hipGetLastError();  // clear a stale error from unrelated work
  launch_for<true>(desc->dtype, desc->D, tree, paged != nullptr, p, pl, static_cast<hipStream_t>(stream));
  return hipGetLastError() == hipSuccess ? SPECMOE_OK : SPECMOE_ERR_LAUNCH;
}
