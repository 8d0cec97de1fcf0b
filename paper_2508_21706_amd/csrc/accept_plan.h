// Descriptor checks and workspace layout of the acceptance entry points, greedy
// (accept.hip) and by sampling (sample.hip), which can share a workspace.
#pragma once
#include <stdint.h>

#include "specmoe_accept.h"

namespace {

constexpr int kWavesPerGroup = 8;
constexpr int kGroupsPerCU = 2;
constexpr int kCUs = 256;                  // MI355X
constexpr int kVecBytes = 16;
constexpr int kItemBytes = 8192;           // default item: 8 KB of logits
constexpr int kSplitUnit = 512;            // item granularity (entries)
constexpr int kMaxChunk = 1024;            // C_max limit
constexpr int kMaxSeqs = 65536;            // B limit (fixed counter region)
constexpr int kGroupSeqs = 16;             // sequences a workgroup counts through LDS

inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

inline int elt_of(const specmoe_accept_desc* d) { return d->dtype == SPECMOE_BF16 ? 2 : 4; }

inline int split_of(const specmoe_accept_desc* d) { return d->split ? d->split : kItemBytes / elt_of(d); }

inline int validate(const specmoe_accept_desc* d) {
  if (!d) return SPECMOE_ERR_NULL_POINTER;
  if (d->dtype != SPECMOE_F32 && d->dtype != SPECMOE_BF16) return SPECMOE_ERR_DTYPE;
  if (d->flags != 0) return SPECMOE_ERR_FLAGS;
  if (d->B < 0 || d->B > kMaxSeqs || d->C_max < 1 || d->C_max > kMaxChunk || d->V < 1) return SPECMOE_ERR_SHAPE;
  const int64_t elt = elt_of(d);
  if ((d->V * elt) % kVecBytes != 0) return SPECMOE_ERR_SHAPE;
  if (d->split < 0 || d->split % kSplitUnit != 0) return SPECMOE_ERR_SHAPE;
  const int64_t S = (d->V + (int64_t)split_of(d) - 1) / split_of(d);
  // row offsets in elements, item indices and partial offsets in bytes stay
  // in 32 bits
  if ((int64_t)d->B * d->C_max * d->V >= ((int64_t)1 << 31)) return SPECMOE_ERR_SHAPE;
  if ((int64_t)d->B * d->C_max * S * 8 >= ((int64_t)1 << 31)) return SPECMOE_ERR_SHAPE;
  return SPECMOE_OK;
}

struct Plan {
  int S, N, q, groups, grouped;
  size_t counter_bytes, part_off, bytes;
};

inline Plan make_plan(const specmoe_accept_desc* d) {
  Plan pl;
  pl.S = (d->V + split_of(d) - 1) / split_of(d);
  pl.N = d->B * d->C_max * pl.S;
  // contiguous ranges of q items for at most the persistent grid's waves
  const int waves = kCUs * kGroupsPerCU * kWavesPerGroup;
  pl.q = pl.N > 0 ? (pl.N + waves - 1) / waves : 1;
  const int used = pl.N > 0 ? (pl.N + pl.q - 1) / pl.q : 0;
  pl.groups = (used + kWavesPerGroup - 1) / kWavesPerGroup;
  // a range of gq items meets at most (gq - 1) / CS + 2 sequences
  const int64_t gq = (int64_t)kWavesPerGroup * pl.q, CS = (int64_t)d->C_max * pl.S;
  pl.grouped = (gq - 1) / CS + 2 <= kGroupSeqs;
  pl.counter_bytes = align256((size_t)kMaxSeqs * sizeof(int));
  pl.part_off = pl.counter_bytes;
  pl.bytes = pl.part_off + (size_t)pl.N * 8;
  return pl;
}

}  // namespace
