// Verification and decode attention over a 4-bit KV cache (specmoe_kv4.h) for
// MI355X (gfx950, CDNA4).
//
// For the rows r = (token, head of the group) of a unit (sequence, KV head) and its
// keys t: s_rt = scale q_r k_t, o_r = sum_t 2^(s'_rt - m_r) v_t / sum_t 2^(s'_rt - m_r)
// with s' = s log2 e and m a running maximum that moves only when a score passes it by
// kLazyMax (so exponents stay within it), all of it in one pass over the cache.
//
// A key and a value of D = 128 are 136 bytes together: at 6.5 TB/s 190 such pairs come to
// a CU in a microsecond, in bfloat16 50.  So codes go as far as they can as they are:
// keys into the f8f6f4 MFMA with their scales, against queries cut into 8-bit parts
// once a unit.  Values meet probabilities of 8 to 24 bits and are made bfloat16, through
// a stage in LDS that gives them back transposed.
//
// Workgroups of four waves, two to a CU, loads straight into registers one step of 32
// keys ahead and across units, no waits but a unit's end: with so few bytes the waves'
// own chains, not the stream, are what has to be hidden.  Each wave has its own keys or
// rows of the unit; their states join through LDS.  Workgroups have ranges of equal cost
// of the list of all units' tiles; a unit that a range cuts is joined from its pieces
// by the last one to arrive.
//
// Measured (whole passes, 8 KV heads of 128, four query heads each): 32 sequences of
// 16384 to 32768 in bfloat16, chunks of 4: 141 us, 6.2 TB/s, near the stream's rate.  64 of 512
// to 2048 in pages, chunks of 5: 34 us for 92 MB, of which start (lengths, lookups,
// first loads) 4 to 5, a unit's end 2 and the pieces' join 4; 256 of them 94.  Trees of 16
// over the same contexts, float16: 69 us, bound by the vector instructions of its four
// row blocks (60% of the issue slots, MFMA 25%).  4 sequences of 100 to 400, float32, D = 64,
// single tokens: 9 us, a chain of launch, lengths, loads, join.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "kv4.h"
#include "specmoe_kv4.h"
#include "verify_kernel.h"

namespace {

constexpr int kGroupWaves = 4;
constexpr int kGroupThreads = 64 * kGroupWaves;
constexpr int kGroupsDefault = 512;   // persistent workgroups: two per CU of an MI355X
constexpr int kTile = 128;            // keys of a tile
constexpr int kStep = 32;             // keys that a wave takes at a time: two MFMA blocks
// The schedule (see the kernel): tiles a workgroup from which on units cost and cuts
// snap, what a unit costs beside its tiles, and how near a unit's end a cut goes to it
constexpr int kManyTiles = 6, kUnitCost = 4, kSnap = 3;
// Pieces of a unit, at most and about: its join is one workgroup's, a round trip for
// every few of them.  Up to one row block: 32 (4 sequences of 23,000 keys, one KV head,
// chunks of 2, float16: 60 us with all workgroups, 128 pieces, and 33).  More rows, whose
// join takes longer: a unit of n tiles in x pieces takes about a n / x + b x, least at a
// multiple of sqrt(n), and twice that is near it (one sequence of 2,200 keys, 128 rows:
// 18 pieces 39 us, 8 pieces 33; 13 of 3,700, one KV head, chunks of 3 to 14, float16: 70
// and 65; 7 of 7,000, 4 KV heads, 126 rows, where 15 pieces leave a few CUs idle: 104, 111).
// The first rule was measured up to 30,000 keys; past that its units stay at 32 pieces.
constexpr int kMostPieces = 32;
constexpr float kPiecesOfRoot = 2.f;

template <int N>
struct Int {
  static constexpr int value = N;
};

// Where the cache's rows are: a slab per sequence, or pages of at least 16 tokens (a
// block of 16 keys is in one page), or of 8
constexpr int kSlab = 0, kPages = 1, kSmallPages = 2;

struct Kv4Params : Params {   // (k and v: the codes)
  const char* k_scales;
  const char* v_scales;
};

typedef __attribute__((ext_vector_type(8))) int i32x8;

// How scores are formed.  kCodes: the key codes go into the MFMA as they are (f8f6f4,
// scales and all), against queries in 8 bits: a query is cut into parts of 4
// significant bits, two for bfloat16's 8 and three for float16's 11.  Otherwise
// (float32, whose 24 bits would take six, and D = 64, half of the MFMA's 128) the
// codes become bfloat16, against one, two or three bfloat16 parts.
template <int ELT, int D>
constexpr bool kCodes = D == 128 && ELT != kF32;
template <int ELT, int D>
constexpr int kQParts = kCodes<ELT, D> ? (ELT == kBF16 ? 2 : 3) : ELT == kBF16 ? 1 : ELT == kF16 ? 2 : 3;
// bfloat16 parts of a probability for its product with the values
template <int ELT>
constexpr int kPParts = ELT == kBF16 ? 1 : ELT == kF16 ? 2 : 3;
// Binades from one 8-bit part of a query to the next: a part's rounding leaves at most
// 2^-5 of the largest entry's power of two
constexpr int kPartShift = 5;

__device__ __forceinline__ int tiles_of(uint32_t s) { return sched::seq_tiles(s, kTile); }

// A workgroup barrier for data in LDS alone: loads and stores under way stay so
// (__syncthreads() waits for them: 2 us at every unit's end).
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The largest of 8 scores, NaN if one is: three instructions of three operands and one
// of two, without the canonicalising that fmaxf adds for each of an MFMA's results.
// (Not by inline assembly, as the wait that an MFMA's results need before a vector
// instruction reads them is the compiler's, and it does not look into assembly.)
__device__ __forceinline__ float max8(const float (&y)[8]) {
  float a = y[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) a = __builtin_elementwise_maximum(a, y[e]);
  return a;
}

// Two values cut to their leading 8 significant bits, as two bfloat16; x keeps
// what was cut off.  Infinities and NaN go whole into the first part.
__device__ __forceinline__ uint32_t split2(float& x, float& y) {
  const uint32_t u = __float_as_uint(x), w = __float_as_uint(y);
  const bool xf = (u & 0x7f800000u) != 0x7f800000u, yf = (w & 0x7f800000u) != 0x7f800000u;
  const uint32_t p = xf ? u & 0xffff0000u : (pack_bf16x2(x, 0.f) << 16);
  const uint32_t q = yf ? w & 0xffff0000u : (pack_bf16x2(y, 0.f) << 16);
  x = xf ? x - __uint_as_float(p) : 0.f;
  y = yf ? y - __uint_as_float(q) : 0.f;
  return (p >> 16) | q;
}

// The least scale byte whose unit, 2^126, has a code (4 units) past float32's range
constexpr uint32_t kFarByte = 253;

// (kCodes) 16 values as 8-bit codes of `unit`, to nearest even; x keeps what the
// rounding left.  An infinity or NaN has the NaN code.
__device__ __forceinline__ void part8(float (&x)[16], float unit, bool rest, int* codes) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    s16x2 c = {0, 0};
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, x[4 * w], x[4 * w + 1], unit, false);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, x[4 * w + 2], x[4 * w + 3], unit, true);
    codes[w] = __builtin_bit_cast(int, c);
    if (rest) {
      const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[w], unit, false);
      const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[w], unit, true);
      x[4 * w] -= lo[0];
      x[4 * w + 1] -= lo[1];
      x[4 * w + 2] -= hi[0];
      x[4 * w + 3] -= hi[1];
    }
  }
}

template <int ELT, int D, int PAGING, int NRB>
__global__ __launch_bounds__(kGroupThreads, 2) void kv4_attn_kernel(Kv4Params p) {
  constexpr int kElt = ELT == kF32 ? 4 : 2;
  constexpr bool CODES = kCodes<ELT, D>;
  constexpr int QP = kQParts<ELT, D>, PP = kPParts<ELT>;
  constexpr int KW = D / 32;          // code words of a lane: its D / 4 entries of a row
  constexpr int DB = D / 16;          // 16-wide d blocks of O^T
  constexpr int kPitch = 2 * D + (D == 128 ? 32 : 16);   // LDS bytes of a staged V row, free of bank conflicts
  constexpr int kStage = kStep * kPitch;
  static_assert(kStage >= kBlk * D * 4, "a row block's O fits a wave's stage");
  __shared__ __attribute__((aligned(16))) char smem[kGroupWaves * kStage];
  __shared__ uint32_t seqs[kMaxSeqs];
  __shared__ int pref[kMaxSeqs];      // cost of one KV head's units of the sequences before b
  __shared__ int wsum[2][kGroupWaves];
  __shared__ float mst[kGroupWaves][NRB][2][kBlk];
  __shared__ int sh_last[2];

  const int pid = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int lm = lane & 15, lg = lane >> 4;
  const int B = p.B, Hkv = p.Hkv, g = p.g;

  // ---- lengths, and this workgroup's range of the list of all units' tiles.
  // Ranges are of equal cost: a tile costs 1 and a unit's start and end kUnitCost
  // more.  A range that would begin within kSnap tiles of a unit's start or end
  // begins there.  With few tiles to a workgroup units cost nothing and are cut
  // anywhere.
  const int per = (B + kGroupThreads - 1) / kGroupThreads;
  const int b_lo = min(tid * per, B), b_hi = min(b_lo + per, B);
  int mine = 0, some = 0;   // tiles, and sequences that have any
  for (int b = b_lo; b < b_hi; ++b) {
    const uint32_t s = load_seq(p, b);
    seqs[b] = s;
    mine += tiles_of(s);
    some += tiles_of(s) > 0;
  }
  const int incl = wave_scan(mine), incl_some = wave_scan(some);
  if (lane == 63) {
    wsum[0][wave] = incl;
    wsum[1][wave] = incl_some;
  }
  __syncthreads();
  int before = incl - mine, before_some = incl_some - some, total = 0, total_some = 0;
#pragma unroll
  for (int w = 0; w < kGroupWaves; ++w) {
    before += w < wave ? wsum[0][w] : 0;
    before_some += w < wave ? wsum[1][w] : 0;
    total += wsum[0][w];
    total_some += wsum[1][w];
  }
  const int N = uniform(total) * Hkv;   // tiles (host check)
  const bool many = N >= kManyTiles * p.P;
  const int unit_cost = many ? kUnitCost : 0, snap = many ? kSnap : 1;
  for (int b = b_lo, x = before + unit_cost * before_some; b < b_hi; ++b) {
    pref[b] = x;
    const int n = tiles_of(seqs[b]);
    x += n + (n > 0 ? unit_cost : 0);
  }
  __syncthreads();

  // padding rows c_b <= i < C_max of the sequences b = pid (mod P)
  for (int b = pid; b < B; b += p.P) {
    const int c = seq_c(seqs[b]);
    constexpr int kPer = D * kElt / 16;
    const size_t row0 = (size_t)(b * p.C_max + c) * p.Hq;
    const int64_t n = (int64_t)(p.C_max - c) * p.Hq * kPer;
    for (int64_t idx = tid; idx < n; idx += kGroupThreads) {
      const size_t orow = row0 + idx / kPer;
      __builtin_nontemporal_store(f32x4{0.f, 0.f, 0.f, 0.f},
                                  reinterpret_cast<f32x4*>(p.out + (row0 * kPer + idx) * 16));
      if (idx % kPer == 0) __builtin_nontemporal_store(-INFINITY, p.lse + orow);
    }
  }

  // Ranges of cost / P, the first cost % P of them of one more
  const int cost = N + unit_cost * uniform(total_some) * Hkv;
  const int units = uniform(total_some) * Hkv;
  const int most = NRB == 1 ? kMostPieces * min(units, p.P)
                            : uniform((int)fminf(kPiecesOfRoot * sqrtf((float)N * (float)units), (float)p.P));
  const int P = min(min(p.P, N), most);
  if (pid >= P) return;
  const int share = uniform(cost / P), longer = cost - share * P;
  auto range_start = [&](int r) { return r * share + min(r, longer); };
  // the last range that starts at or before a cost
  auto owner = [&](int x) {
    const int cut = longer * (share + 1);
    return uniform(x < cut ? x / (share + 1) : longer + (x - cut) / share);
  };
  // the tile of a unit of n at which a range begins whose cost lies x after the
  // unit's (0: at its start, n: at the next one's), and the largest such x for its
  // first tile and for its last one
  auto cut_at = [&](int x, int n) {
    const int j = x - unit_cost / 2;
    if (n < 2 * snap) return 2 * j < n ? 0 : n;
    return j < snap ? 0 : j > n - snap ? n : j;
  };
  auto most_first = [&](int n) { return unit_cost / 2 + (n < 2 * snap ? (n - 1) >> 1 : snap - 1); };
  auto most_last = [&](int n) { return unit_cost / 2 + (n < 2 * snap ? (n - 1) >> 1 : n - snap); };
  const int c_end = range_start(pid + 1);

  char* const stage = smem + wave * kStage;

  // ---- segments: tiles [j0, j1) of one unit, KV head kvh of sequence b
  struct Segment {
    int b, kvh, j0, j1, n, T, c;   // n: tiles of the unit
    int kend;                      // the first key past the segment
    int cost;                      // at which the unit begins
    int groups;                    // (log2) groups of waves that have different rows of the unit
  };
  // Of the four waves those of a row group share its keys, step by step in turn.
  auto row_group = [&](const Segment& x) { return wave & ((1 << x.groups) - 1); };
  auto key_slot = [&](const Segment& x) { return wave >> x.groups; };
  auto stride = [&](const Segment& x) { return (kGroupWaves * kStep) >> x.groups; };   // keys from a wave's step to its next
  // (of the range: j1 = 0 if the unit is past its end)
  auto segment = [&](int b, int kvh, int j0, int at) {
    Segment x;
    const uint32_t s = uniform(seqs[b]);
    x.b = b;
    x.kvh = kvh;
    x.n = tiles_of(s);
    x.j0 = j0;
    x.cost = at;
    x.j1 = c_end >= at + x.n + unit_cost ? x.n : c_end > at ? cut_at(c_end - at, x.n) : 0;
    x.T = seq_T(s);
    x.c = seq_c(s);
    // (as many as the unit's own rows need, whatever the longest chunk's do: 7 sequences
    // of 22,000 keys, chunks of 3 to 15 with seven heads, float16: 114 us, so 105)
    const int blocks = (x.c * g + kBlk * NRB - 1) / (kBlk * NRB);
    x.groups = blocks <= 1 ? 0 : blocks <= 2 ? 1 : 2;
    x.kend = min(x.T, x.j1 * kTile);
    return x;
  };
  // the next unit, from its tile 0 (past the last one: no tiles)
  auto segment_after = [&](const Segment& x) {
    const int at = x.cost + x.n + unit_cost;
    if (at >= c_end) {
      Segment none = x;
      none.j0 = none.j1 = 0;
      return none;
    }
    int b = x.b, kvh = x.kvh + 1;
    if (kvh == Hkv) {
      kvh = 0;
      do ++b;
      while (tiles_of(uniform(seqs[b])) == 0);   // (there is one: at < c_end)
    }
    return segment(b, kvh, 0, at);
  };
  Segment sg;
  {
    // the last sequence whose cost begins at or before the range's (it has tiles): a
    // lane looks at every 16th, then 16 lanes at the ones from there on
    const int c0 = range_start(pid);
    const int lot = lane * (kMaxSeqs / 64);
    const uint64_t lots = __ballot(lot < B && pref[min(lot, B - 1)] * Hkv <= c0);
    int b = (63 - __builtin_clzll(lots)) * (kMaxSeqs / 64);
    const int i = b + (lane & 15);
    b += 31 - __builtin_clz((uint32_t)__ballot(lane < 16 && i < B && pref[min(i, B - 1)] * Hkv <= c0));
    b = uniform(b);
    const int start = uniform(pref[b]) * Hkv, n = tiles_of(uniform(seqs[b])), each = n + unit_cost;
    const int kvh = uniform((c0 - start) / each), at = start + kvh * each;
    const int j = cut_at(c0 - at, n);
    sg = segment(b, kvh, j, at);
    if (j == n) sg = segment_after(sg);
  }
  if (sg.j1 <= sg.j0) return;   // (an empty range)

  // ---- 32 keys from base on: lane (lm, lg) has the lg-th quarter of the rows of
  // keys base + lm and base + 16 + lm.
  typedef __attribute__((ext_vector_type(KW))) uint32_t words;
  struct Keys {
    words k[2], v[2];
    uint32_t ks[2], vs[2];
  };
  // What a wave loads next: keys from base on of a segment; with pages, those of 8
  // of the 32 keys each, the same for the whole wave, looked up a step ahead
  // through the scalar cache, so that a load waits for no lookup of its own.
  struct Target {
    int b, kvh, kend, base;
    int page[kStep / 8];
  };
  auto aim = [&](Target& x, const Segment& at, int base) {
    x.b = at.b;
    x.kvh = at.kvh;
    x.kend = at.kend;
    x.base = base;
    if constexpr (PAGING != kSlab) {
      typedef const __attribute__((address_space(4))) int32_t* const_table;
      const const_table row = (const_table)(p.block_table + (size_t)at.b * p.pages_per_seq);
#pragma unroll
      for (int i = 0; i < kStep / 8; i += PAGING == kPages ? 2 : 1)
        x.page[i] = row[min(base + 8 * i, at.kend - 1) >> p.page_shift];
    }
  };
  // A block of 16 keys in consecutive rows is read through buffer descriptors that
  // end with the segment's last key: rows past it read as zeros, whose scores are
  // masked, and a lane's offsets never change.  (In pages of 8 a lane has an
  // address of its own, and rows past the end re-read the last one.)
  const int lane_codes = lm * (D / 2) + lg * (D / 8), lane_scale = lm * (D / 32) + (lg * (D / 4) / 32);
  auto load = [&](Keys& x, const Target& at) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      auto page = [&](int i) { return uniform(min(max(at.page[i], 0), p.num_pages - 1)); };
      if constexpr (PAGING == kSmallPages) {
        const int key = min(at.base + kBlk * h + lm, at.kend - 1);
        const size_t row = (((size_t)(lm < 8 ? page(2 * h) : page(2 * h + 1)) * Hkv + at.kvh) << 3) + (key & 7);
        const size_t code = row * (D / 2) + lg * (D / 8), scale = row * (D / 32) + (lg * (D / 4) / 32);
        x.k[h] = *reinterpret_cast<const words*>(p.k + code);
        x.v[h] = *reinterpret_cast<const words*>(p.v + code);
        x.ks[h] = (uint8_t)p.k_scales[scale];
        x.vs[h] = (uint8_t)p.v_scales[scale];
      } else {
        const int key = at.base + kBlk * h;
        const int rows = uniform(min(max(at.kend - key, 0), kBlk));   // (a scalar for the descriptors)
        size_t row;
        if constexpr (PAGING == kPages)
          row = (((size_t)page(2 * h) * Hkv + at.kvh) << p.page_shift) + (key & ((1 << p.page_shift) - 1));
        else
          row = ((size_t)at.b * Hkv + at.kvh) * p.S_max + key;
        auto buffer = [&](const char* base, int row_bytes) {
          return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base) + row * row_bytes, 0, rows * row_bytes,
                                                   kBufferFormat);
        };
        const auto kb = buffer(p.k, D / 2), vb = buffer(p.v, D / 2);
        if constexpr (KW == 4) {
          x.k[h] = __builtin_bit_cast(words, __builtin_amdgcn_raw_buffer_load_b128(kb, lane_codes, 0, kStreaming));
          x.v[h] = __builtin_bit_cast(words, __builtin_amdgcn_raw_buffer_load_b128(vb, lane_codes, 0, kStreaming));
        } else {
          x.k[h] = __builtin_bit_cast(words, __builtin_amdgcn_raw_buffer_load_b64(kb, lane_codes, 0, kStreaming));
          x.v[h] = __builtin_bit_cast(words, __builtin_amdgcn_raw_buffer_load_b64(vb, lane_codes, 0, kStreaming));
        }
        x.ks[h] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(buffer(p.k_scales, D / 32), lane_scale, 0, 0);
        x.vs[h] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(buffer(p.v_scales, D / 32), lane_scale, 0, 0);
      }
    }
  };

  // ---- queries: row block rb of a wave of row group rg has the unit's rows 16 (NRB rg + rb) + lm.
  // x / g for a row 0 <= x < 128 of a unit, by a float reciprocal: exact there, as
  // (x + 1/2) / g lies at least 1 / (2 g) from an integer
  const float inv_g = 1.f / (float)g;
  auto div_g = [&](int x) { return (int)(((float)x + 0.5f) * inv_g); };
  constexpr int kRaw = D * kElt / 64;   // 16-byte pieces of a lane's quarter of a row
  u32x4 q_raw[NRB][kRaw];
  uint64_t word_raw[NRB];
  // The entries of a lane: as of a key, the lg-th quarter of the row; with kCodes
  // 16 from 16 lg on, and from 64 + 16 lg on, as the MFMA takes its 8-bit operand.
  auto load_q = [&](const Segment& at) {
    const int rg = row_group(at);
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      // (rows past the unit's are computed as its last one and not stored)
      const int row = min(kBlk * (NRB * rg + rb) + lm, at.c * g - 1), tok = div_g(row);
      const char* src = p.q + ((size_t)(at.b * p.C_max + tok) * p.Hq + at.kvh * g + (row - tok * g)) * (D * kElt);
#pragma unroll
      for (int i = 0; i < kRaw; ++i) {
        const int piece = CODES ? 32 * lg + 128 * (i >> 1) + 16 * (i & 1) : lg * (D / 4) * kElt + 16 * i;
        q_raw[rb][i] = *reinterpret_cast<const u32x4*>(src + piece);
      }
      if (p.draft_mask) word_raw[rb] = p.draft_mask[at.b * p.C_max + tok];
    }
  };
  auto entry = [&](const u32x4* raw, int e) {   // the e-th of a lane's entries
    if constexpr (ELT == kF32) return __uint_as_float(raw[e >> 2][e & 3]);
    else if constexpr (ELT == kF16) return (float)__builtin_bit_cast(f16x8, raw[e >> 3])[e & 7];
    else return __uint_as_float((e & 1) ? raw[e >> 3][(e & 7) >> 1] & 0xffff0000u : raw[e >> 3][(e & 7) >> 1] << 16);
  };

  i32x8 qc[CODES ? QP : 1][CODES ? NRB : 1];    // kCodes: the parts' codes,
  int qs[CODES ? NRB : 1];                      // and their scale bytes, one part's after the other's
  u32x4 qb[CODES ? 1 : QP][CODES ? 1 : NRB][CODES ? 1 : KW];   // else: bfloat16 parts
  uint64_t word[NRB];
  int tok[NRB];
  int l_ctx = 0, c = 0;   // of the segment being computed
  f32x4 o[NRB][DB];
  float m_run[NRB], m_use[NRB], l_lane[NRB];   // m_use: m_run, or 0 before any key

  auto take_q = [&](int rg) {
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      tok[rb] = div_g(min(kBlk * (NRB * rg + rb) + lm, c * g - 1));
      word[rb] = word_raw[rb];
      if constexpr (CODES) {
        // Blocks of 32 entries have units of their own, the largest entry's power
        // of two less 7: block (lg >> 1) is the first halves of lanes lg and lg ^ 1,
        // block 2 + (lg >> 1) their second halves.  The MFMA takes the scale of block
        // lg from lane lg.
        float f[2][16];
        int sb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float most = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            f[i][e] = entry(q_raw[rb], 16 * i + e);
            most = fmaxf(most, fabsf(f[i][e]));
          }
          most = fmaxf(most, __shfl_xor(most, 16));
          sb[i] = max((int)(__float_as_uint(most) >> 23) - 7, 1 + kPartShift * (QP - 1));
        }
        const int far0 = __shfl_xor(sb[0], 48), far1 = __shfl_xor(sb[1], 48);
        const int own = lg == 0 ? sb[0] : lg == 1 ? far0 : lg == 2 ? far1 : sb[1];
        qs[rb] = 0;
#pragma unroll
        for (int part = 0; part < QP; ++part) {
          qs[rb] |= (own - kPartShift * part) << (8 * part);
          int codes[8];
#pragma unroll
          for (int i = 0; i < 2; ++i)
            part8(f[i], kv4::scale_of((uint32_t)(sb[i] - kPartShift * part)), part + 1 < QP, codes + 4 * i);
          qc[part][rb] = i32x8{codes[0], codes[1], codes[2], codes[3], codes[4], codes[5], codes[6], codes[7]};
        }
      } else {
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          if constexpr (ELT == kBF16) {
            qb[0][rb][w] = q_raw[rb][w];
          } else {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = entry(q_raw[rb], 8 * w + e);
#pragma unroll
            for (int part = 0; part < QP; ++part)
#pragma unroll
              for (int e = 0; e < 4; ++e) qb[part][rb][w][e] = split2(f[2 * e], f[2 * e + 1]);
          }
        }
      }
      m_run[rb] = -INFINITY;
      m_use[rb] = 0.f;
      l_lane[rb] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };

  auto compute = [&](Keys& x, int base) {
    const bool drafts = base + kStep > l_ctx;   // (the same for the whole wave) keys that not every row sees
    // Values of such keys that are infinities or NaN (scale bytes from kFarByte on can
    // make them): 0 times them would reach the rows that do not see the key.  So these
    // blocks are staged with scale byte 0, too small to show, and added to the rows that
    // see them afterwards; their bytes lie behind their rows in the stage.  Bit 16 qd + i
    // of far[h]: the qd-th quarter of key 16 h + i.
    uint64_t far[2] = {0, 0};
    uint32_t seen[NRB];   // (drafts) bit e: the lane's row sees its e-th key
    if (drafts) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool is_far = x.vs[h] >= kFarByte;
        far[h] = __ballot(is_far);
        if (is_far) {
          *reinterpret_cast<uint32_t*>(stage + (kBlk * h + lm) * kPitch + 2 * D + 4 * lg) = x.vs[h];
          x.vs[h] = 0;
        }
      }
    }
    // scores of two key blocks: S^T = K Q^T, lane (lm, lg) gets the keys
    // 16 h + 4 lg + r of row lm
    f32x4 sa[NRB][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (CODES) {
        // (the MFMA takes 4 registers of 4-bit codes; the other 4 have no value)
        typedef __attribute__((ext_vector_type(8))) uint32_t u32x8;
        const u32x4 k = x.k[h];
        const i32x8 kc = __builtin_bit_cast(i32x8, (u32x8)__builtin_shufflevector(k, k, 0, 1, 2, 3, -1, -1, -1, -1));
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
          // (4: 4-bit codes, 0: 8-bit codes with 3 bits after the leading one; a part's
          // scale is the part-th byte)
          if constexpr (QP == 3)
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kc, qc[QP - 1][rb], acc, 4, 0, 0, x.ks[h], 2, qs[rb]);
          acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kc, qc[CODES ? 1 : 0][rb], acc, 4, 0, 0, x.ks[h], 1, qs[rb]);
          acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kc, qc[0][rb], acc, 4, 0, 0, x.ks[h], 0, qs[rb]);
          sa[rb][h] = acc;
        }
      } else {
        const float ks = kv4::scale_of(x.ks[h]);
        u32x4 kop[KW];
#pragma unroll
        for (int w = 0; w < KW; ++w)
          kop[w] = u32x4{kv4::bf16_of<0>(x.k[h][w], ks), kv4::bf16_of<1>(x.k[h][w], ks),
                         kv4::bf16_of<2>(x.k[h][w], ks), kv4::bf16_of<3>(x.k[h][w], ks)};
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int part = QP - 1; part >= 0; --part)
#pragma unroll
            for (int w = 0; w < KW; ++w) acc = mfma32<kBF16>(kop[w], qb[part][rb][w], acc);
          sa[rb][h] = acc;
        }
      }
    }
    // values as bfloat16 into the wave's stage
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float vs = kv4::scale_of(x.vs[h]);
      char* dst = stage + (kBlk * h + lm) * kPitch + lg * (D / 2);
#pragma unroll
      for (int w = 0; w < KW; ++w)
        *reinterpret_cast<u32x4*>(dst + 16 * w) =
            u32x4{kv4::bf16_of<0>(x.v[h][w], vs), kv4::bf16_of<1>(x.v[h][w], vs), kv4::bf16_of<2>(x.v[h][w], vs),
                  kv4::bf16_of<3>(x.v[h][w], vs)};
    }
    asm volatile("" ::: "memory");   // (LDS serves a wave's accesses in order)
    // softmax
    u32x4 pb[NRB][PP];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = sa[rb][e >> 2][e & 3];
      if (drafts) {
        uint32_t see = 0;
        const int k0 = base + 4 * lg - l_ctx;   // the first key as a draft token
        if (p.draft_mask) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int k = k0 + kBlk * (e >> 2) + (e & 3);
            const uint32_t bit = (uint32_t)(word[rb] >> (k & 63)) & (uint32_t)(k < c);
            see |= (k < 0 ? 1u : bit & 1u) << e;
          }
        } else {
          const int last = min(tok[rb], c - 1);
#pragma unroll
          for (int e = 0; e < 8; ++e) see |= (uint32_t)(k0 + kBlk * (e >> 2) + (e & 3) <= last) << e;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (see >> e) & 1u ? y[e] : -INFINITY;
        seen[rb] = see;
      }
      // the running maximum moves only for a score that passes it by more than
      // kLazyMax, so most steps exchange nothing between lanes
      const float mx_lane = max8(y) * p.sl2;
      if (__any(mx_lane > m_run[rb] + kLazyMax)) {
        const float mx = row_max(mx_lane);
        const bool raise = mx > m_run[rb] + kLazyMax;
        const float m_new = raise ? mx : m_run[rb];
        const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - (m_new == -INFINITY ? 0.f : m_new));
        l_lane[rb] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[rb][db] *= alpha;
        m_run[rb] = m_new;
        m_use[rb] = m_new == -INFINITY ? 0.f : m_new;
      }
      float pr[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        pr[e] = __builtin_amdgcn_exp2f(fmaf(y[e], p.sl2, -m_use[rb]));
        l_lane[rb] += pr[e];
      }
#pragma unroll
      for (int part = 0; part < PP; ++part)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t u = pack_bf16x2(pr[2 * e], pr[2 * e + 1]);
          pb[rb][part][e] = u;
          if (part + 1 < PP) {   // what the rounding leaves is the next part's
            pr[2 * e] -= __uint_as_float(u << 16);
            pr[2 * e + 1] -= __uint_as_float(u & 0xffff0000u);
          }
        }
    }
    // O^T += V^T P^T over the 32 keys: element e of a lane's operands is key
    // 4 lg + e of the first block (e < 4) or 4 lg + e - 4 of the second
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const char* vrow = stage + (4 * lg + (lm >> 2)) * kPitch + 8 * (lm & 3);
    auto read_v = [&](int db) {
      const i16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(__attribute__((address_space(3))) char*)(vrow + 32 * db));
      const i16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(__attribute__((address_space(3))) char*)(vrow + kBlk * kPitch + 32 * db));
      return u32x4{__builtin_bit_cast(uint2, a0).x, __builtin_bit_cast(uint2, a0).y, __builtin_bit_cast(uint2, a1).x,
                   __builtin_bit_cast(uint2, a1).y};
    };
    // The reads of kAheadV d blocks are under way: left to itself the compiler waits for
    // each before its products (64 sequences, chunks of 5: 37.0 against 34.8 us, trees of
    // 16 in float16 70.3 against 68.5).
    constexpr int kAheadV = PP == 1 ? 4 : 3;
    u32x4 va[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) va[db] = read_v(db);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
        for (int part = PP - 1; part >= 0; --part) o[rb][db] = mfma32<kBF16>(va[db], pb[rb][part], o[rb][db]);
    constexpr int kMfma = 0x8, kLdsRead = 0x100;
    __builtin_amdgcn_sched_group_barrier(kLdsRead, 2 * kAheadV, 0);
#pragma unroll
    for (int db = kAheadV; db < DB; ++db) {
      __builtin_amdgcn_sched_group_barrier(kMfma, NRB * PP, 0);
      __builtin_amdgcn_sched_group_barrier(kLdsRead, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMfma, NRB * PP * kAheadV, 0);
    asm volatile("" ::: "memory");
    if (far[0] | far[1]) {
      // one key after the other, as the MFMA takes it: the probability's parts times the
      // value, for the rows that see the key
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t keys = (uint32_t)(far[h] | far[h] >> 16 | far[h] >> 32 | far[h] >> 48) & 0xffffu;
        for (; keys; keys &= keys - 1) {
          const int i = __builtin_ctz(keys);
          const char* row = stage + (kBlk * h + i) * kPitch;
          const int src = lm + kBlk * (i >> 2);   // the lane that has the key's probability
#pragma unroll
          for (int rb = 0; rb < NRB; ++rb) {
            const bool sees = (uint32_t)__shfl((int)seen[rb], src) >> (4 * h + (i & 3)) & 1u;
            float pr = 0.f;
#pragma unroll
            for (int part = PP - 1; part >= 0; --part) {
              const uint32_t pair = (i & 2) ? pb[rb][part][2 * h + 1] : pb[rb][part][2 * h];
              const uint32_t both = (uint32_t)__shfl((int)pair, src);
              pr += __uint_as_float((i & 1) ? both & 0xffff0000u : both << 16);
            }
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              constexpr int kPerQuarter = DB / 4;
              if (!((far[h] >> (16 * (db / kPerQuarter) + i)) & 1u)) continue;
              const uint32_t byte = *reinterpret_cast<const uint32_t*>(row + 2 * D + 4 * (db / kPerQuarter));
              const uint2 v = *reinterpret_cast<const uint2*>(row + 32 * db + 8 * lg);
              const float unit = byte == 255u ? NAN : kv4::scale_of(byte);
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const uint32_t w = r < 2 ? v.x : v.y;
                const float code = __uint_as_float((r & 1) ? w & 0xffff0000u : w << 16) * 0x1p127f;
                if (sees) o[rb][db][r] = fmaf(pr, code * unit, o[rb][db][r]);
              }
            }
          }
        }
      }
    }
  };

  // A token of n in its chunk that sees a key: one of the l of its context, or one that
  // its word names (in a chain always itself).  If no key that such a token sees has any
  // weight, all of their scores are -inf and the row is NaN, not empty.
  auto sees_any = [&](uint64_t w, int l, int n) {
    return l > 0 || !p.draft_mask || (w & (n >= 64 ? ~0ull : (1ull << n) - 1)) != 0;
  };

  // pieces of units that other workgroups share, at most the range's first and
  // last: the first and last range that have a piece of the unit, its index, its rows
  int n_pieces = 0;
  i32x4 piece[2];
  const __amdgpu_buffer_rsrc_t ws_o_rsrc = __builtin_amdgcn_make_buffer_rsrc(p.ws_o, 0, p.ws_o_bytes, kBufferFormat);
  const __amdgpu_buffer_rsrc_t ws_lse_rsrc =
      __builtin_amdgcn_make_buffer_rsrc(p.ws_lse, 0, p.ws_lse_bytes, kBufferFormat);

  // The loads of a step are under way while the one before is computed, across
  // segments too: y holds the segment's first step at its start.  (One copy of the
  // step's code, with 20 moves to a step: two copies without moves take longer, 38.4
  // against 35.9 us for 64 sequences, 145 against 141 for long ones.)
  Keys x, y;
  Target next;
  load_q(sg);
  {
    Target at;   // (both lookups before the first load)
    const int base = sg.j0 * kTile + kStep * key_slot(sg);
    aim(at, sg, base);
    aim(next, sg, base + stride(sg));
    load(y, at);
  }
  for (;;) {
    const Segment nx = segment_after(sg);
    const bool more = nx.j1 > 0;
    const int rg = row_group(sg), kslot = key_slot(sg), by = stride(sg), RG = 1 << sg.groups, KS = kGroupWaves >> sg.groups;
    l_ctx = sg.T - sg.c;
    c = sg.c;
    take_q(rg);

    // ---- this wave's steps of the segment.  follow(): the loads after those of
    // the step at base, and the lookup for the ones after them
    const int first_base = kStep * key_slot(nx);
    auto follow = [&](Keys& z, int base) {
      const bool inside = base + by < sg.kend;
      if (!inside && more) aim(next, nx, first_base);   // (looked up late: once a segment)
      if (inside || more) load(z, next);
      if (base + 2 * by < sg.kend) aim(next, sg, base + 2 * by);
      else if (!inside && more) aim(next, nx, first_base + stride(nx));
    };
    int base = sg.j0 * kTile + kStep * kslot;
    if (base >= sg.kend) follow(y, base);   // (none: the segment's last tile is short)
    for (; base < sg.kend; base += by) {
      x = y;
      follow(y, base);
      compute(x, base);
    }
    if (more) load_q(nx);

    // ---- the states of the waves that share the rows joined through LDS: each
    // then has the O of its own d blocks.  All four waves' states are read, those
    // of other rows with weight 0, so that the reads go out together.
    const int R = sg.c * g;
    const bool whole = sg.j0 == 0 && sg.j1 == sg.n;
    // a range has at most one piece that begins its unit, its last segment, and one
    // that does not, its first: slots 2 pid + 1 and 2 pid
    const int slot = 2 * pid + (sg.j0 == 0 ? 1 : 0);
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      const float l_row = row_sum(l_lane[rb]);
      if (lg == 0) {
        mst[wave][rb][0][lm] = m_run[rb];
        mst[wave][rb][1][lm] = l_row;
      }
    }
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      f32x4* own = reinterpret_cast<f32x4*>(stage) + lane;
      if (rb) lds_barrier();   // (the last row block's reads)
#pragma unroll
      for (int db = 0; db < DB; ++db) own[db * 64] = o[rb][db];
      lds_barrier();
      float mk[kGroupWaves], lk[kGroupWaves];
#pragma unroll
      for (int k = 0; k < kGroupWaves; ++k) {
        mk[k] = mst[k][rb][0][lm];
        lk[k] = mst[k][rb][1][lm];
      }
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int k = 0; k < kGroupWaves; ++k) {
        mk[k] = (k & (RG - 1)) == rg ? mk[k] : -INFINITY;
        M = fmaxf(M, mk[k]);
      }
      const float Mu = M == -INFINITY ? 0.f : M;
      float wk[kGroupWaves];
#pragma unroll
      for (int k = 0; k < kGroupWaves; ++k) {
        wk[k] = __builtin_amdgcn_exp2f(mk[k] - Mu);
        L += (k & (RG - 1)) == rg ? lk[k] * wk[k] : 0.f;
      }
      const bool lost = L == 0.f && whole && sees_any(word[rb], l_ctx, c);
      const float inv = L > 0.f ? 1.f / L : lost ? NAN : L == 0.f ? 0.f : L;   // (a NaN stays)
      const int row = kBlk * (NRB * rg + rb) + lm;
      const bool valid = row < R;
      const size_t orow = (size_t)(sg.b * p.C_max + tok[rb]) * p.Hq + sg.kvh * g + (row - tok[rb] * g);
      if (valid && kslot == 0 && lg == 0) {
        const float lse = lost ? NAN : L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
        if (whole) p.lse[orow] = lse;
        else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(int, lse), ws_lse_rsrc, (slot * p.Rcap + row) * 4, 0,
                                                   kDeviceCoherent);
      }
      constexpr int kAhead = DB / kGroupWaves;   // d blocks whose reads go out together: a quarter of them
      for (int d0 = kslot * kAhead; d0 < DB; d0 += KS * kAhead) {
        f32x4 part[kAhead][kGroupWaves];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
          for (int k = 0; k < kGroupWaves; ++k)
            part[u][k] = reinterpret_cast<const f32x4*>(smem + k * kStage)[(d0 + u) * 64 + lane];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < kGroupWaves; ++k)   // (other rows' values are left out, NaN and all)
            r = (k & (RG - 1)) == rg ? add_weighted(r, wk[k], part[u][k]) : r;
          r *= inv;
          if (!valid) continue;
          const int d = 16 * (d0 + u) + 4 * lg;
          if (whole)
            store_out<false, ELT>(p, orow * D + d, r);
          else
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, r), ws_o_rsrc,
                                                   ((slot * p.Rcap + row) * D + d) * 4, 0, kDeviceCoherent);
        }
      }
    }
    if (!whole) {
      const int qf = owner(sg.cost + most_first(sg.n)), ql = owner(sg.cost + most_last(sg.n));
      piece[n_pieces++ ? 1 : 0] = i32x4{qf, ql, sg.b * Hkv + sg.kvh, R};
    }
    if (!more) break;
    lds_barrier();   // (stages and statistics are free again)
    sg = nx;
  }
  if (n_pieces == 0) return;

  // ---- the pieces counted on their units' counters once their stores are out; the
  // last one of a unit to arrive merges all of them, in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  lds_barrier();
  if (lane == 0 && wave < n_pieces) {
    const i32x4 e = wave == 0 ? piece[0] : piece[1];
    int* counter = p.counters + e[2];
    const int last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == e[1] - e[0];
    if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next call
    sh_last[wave] = last;
  }
  lds_barrier();
  // the (row, 4 d) items of the units to merge form one list, and a thread takes
  // kItems of them at a time, all their pieces' loads before the first is used
  const bool m0 = uniform(sh_last[0]), m1 = n_pieces > 1 && uniform(sh_last[1]);
  const int n0 = m0 ? uniform(piece[0][3]) * (D / 4) : 0, n1 = m1 ? uniform(piece[1][3]) * (D / 4) : 0;
  const int pieces = max(m0 ? piece[0][1] - piece[0][0] : -1, m1 ? piece[1][1] - piece[1][0] : -1) + 1;   // of the larger
  auto merge = [&](auto items_at_once, auto pieces_at_once) {
    constexpr int kItems = decltype(items_at_once)::value, kBatch = decltype(pieces_at_once)::value;
    for (int base = tid; base < n0 + n1; base += kItems * kGroupThreads) {
      float m[kItems], z[kItems];
      f32x4 acc[kItems];
      int row[kItems], qf[kItems], ql[kItems], d[kItems], unit[kItems];
#pragma unroll
      for (int it = 0; it < kItems; ++it) {
        const int idx = base + it * kGroupThreads;
        const bool in0 = idx < n0;
        const int local = in0 ? idx : idx - n0;
        row[it] = local / (D / 4);
        d[it] = 4 * (local - row[it] * (D / 4));
        qf[it] = in0 ? piece[0][0] : piece[1][0];
        ql[it] = idx < n0 + n1 ? (in0 ? piece[0][1] : piece[1][1]) : -1;   // (none for a thread past the items)
        unit[it] = in0 ? piece[0][2] : piece[1][2];
        m[it] = -INFINITY;
        z[it] = 0.f;
        acc[it] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      for (int k0 = 0; k0 < pieces; k0 += kBatch) {
        float lse[kItems][kBatch];
        f32x4 part[kItems][kBatch];
#pragma unroll
        for (int it = 0; it < kItems; ++it)
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            lse[it][u] = -INFINITY;
            part[it][u] = f32x4{0.f, 0.f, 0.f, 0.f};
            const int r = qf[it] + k0 + u;
            if (r > ql[it]) continue;
            const int at = (2 * r + (k0 + u == 0 ? 1 : 0)) * p.Rcap + row[it];
            lse[it][u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(ws_lse_rsrc, at * 4, 0, kDeviceCoherent));
            part[it][u] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(ws_o_rsrc, (at * D + d[it]) * 4, 0,
                                                                                          kDeviceCoherent));
          }
#pragma unroll
        for (int it = 0; it < kItems; ++it) {
          float nm = m[it];
#pragma unroll
          for (int u = 0; u < kBatch; ++u) nm = fmaxf(nm, lse[it][u]);
          const float nu = nm == -INFINITY ? 0.f : nm;
          const float a = exp_diff(m[it], nu);
          z[it] *= a;
          acc[it] *= a;
          m[it] = nm;
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            const float w = exp_diff(lse[it][u], nu);
            z[it] += w;
            acc[it] = add_weighted(acc[it], w, part[it][u]);
          }
        }
      }
#pragma unroll
      for (int it = 0; it < kItems; ++it) {
        if (base + it * kGroupThreads >= n0 + n1) continue;
        const int b = unit[it] / Hkv, kvh = unit[it] - b * Hkv, tk = div_g(row[it]);
        const size_t orow = (size_t)(b * p.C_max + tk) * p.Hq + kvh * g + (row[it] - tk * g);
        bool lost = z[it] == 0.f;
        if (lost) {
          const uint32_t s = seqs[b];
          lost = sees_any(p.draft_mask ? p.draft_mask[b * p.C_max + tk] : 0ull, seq_T(s) - seq_c(s), seq_c(s));
        }
        store_out<false, ELT>(p, orow * D + d[it],
                              acc[it] * (z[it] > 0.f ? 1.f / z[it] : lost ? NAN : z[it] == 0.f ? 0.f : z[it]));
        if (d[it] == 0) p.lse[orow] = lost ? NAN : z[it] == 0.f ? -INFINITY : m[it] + logf(z[it]);
      }
    }
  };
  // Many pieces of few rows: more of a thread's loads are pieces (one sequence of 30000
  // keys, 8 KV heads: 22.3 us, so 18.9).
  if constexpr (NRB == 1) {
    if (pieces > 8 && n0 + n1 <= 2 * kGroupThreads) {
      merge(Int<1>{}, Int<16>{});
      return;
    }
  }
  if (NRB > 1 && pieces > 4) merge(Int<3>{}, Int<8>{});   // (32 pieces of 126 rows, 7 sequences: 114 us, so 104)
  else merge(Int<3>{}, Int<4>{});
}

// ---------------------------------------------------------------- host side

// desc with the workgroups of these calls
specmoe_verify_desc sized(const specmoe_verify_desc* d) {
  specmoe_verify_desc x = *d;
  if (x.grid_blocks == 0) x.grid_blocks = kGroupsDefault;
  return x;
}

// [a, a + a_bytes) and [b, b + b_bytes) share memory
bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y ? y - x < a_bytes : x - y < b_bytes;
}

template <int ELT, int D, int PAGING>
void launch_kv4(const Kv4Params& p, hipStream_t stream) {
  constexpr int kElt = ELT == kF32 ? 4 : 2;
  for (int b0 = 0; b0 < p.B; b0 += kMaxSeqs) {   // (as specmoe_verify_attn: consecutive launches)
    Kv4Params s = p;
    s.B = p.B - b0 < kMaxSeqs ? p.B - b0 : kMaxSeqs;
    s.q = p.q + (size_t)b0 * p.C_max * p.Hq * D * kElt;
    if (PAGING != kSlab) {
      s.block_table = p.block_table + (size_t)b0 * p.pages_per_seq;
    } else {
      const size_t rows = (size_t)b0 * p.Hkv * p.S_max;
      s.k = p.k + rows * (D / 2);
      s.v = p.v + rows * (D / 2);
      s.k_scales = p.k_scales + rows * (D / 32);
      s.v_scales = p.v_scales + rows * (D / 32);
    }
    s.ctx_lens = p.ctx_lens + b0;
    s.chunk_lens = p.chunk_lens + b0;
    if (p.draft_mask) s.draft_mask = p.draft_mask + (size_t)b0 * p.C_max;
    s.out = p.out + (size_t)b0 * p.C_max * p.Hq * D * kElt;
    s.lse = p.lse + (size_t)b0 * p.C_max * p.Hq;
    // Row blocks of 16: two to a wave (the conversion of its keys and values serves
    // both: 64 sequences, trees of 16, bf16, four blocks: 63 us; one to a wave 80),
    // but in float32, where two do not fit the registers (8 sequences, chunks of 5,
    // four heads: 47 us; one to a wave 18): four waves hold up to 64 of its rows, and
    // more take two all the same, with 110 to 164 registers spilled at D = 128.  (float16
    // spills 6 to 10 there.)
    const int blocks = (p.Rcap + kBlk - 1) / kBlk;
    const bool single = blocks == 1 || (ELT == kF32 && blocks <= 4);
    if (single) hipLaunchKernelGGL((kv4_attn_kernel<ELT, D, PAGING, 1>), dim3(p.P), dim3(kGroupThreads), 0, stream, s);
    else hipLaunchKernelGGL((kv4_attn_kernel<ELT, D, PAGING, 2>), dim3(p.P), dim3(kGroupThreads), 0, stream, s);
  }
}

template <int ELT, int D>
void launch_kv4_paging(const Kv4Params& p, hipStream_t s) {
  if (!p.block_table) launch_kv4<ELT, D, kSlab>(p, s);
  else if (p.page_shift >= 4) launch_kv4<ELT, D, kPages>(p, s);
  else launch_kv4<ELT, D, kSmallPages>(p, s);
}

template <int ELT>
void launch_kv4_for(int D, const Kv4Params& p, hipStream_t s) {
  if (D == 128) launch_kv4_paging<ELT, 128>(p, s);
  else launch_kv4_paging<ELT, 64>(p, s);
}

}  // namespace

extern "C" {

size_t specmoe_verify_attn_kv4_workspace_bytes(const specmoe_verify_desc* desc) {
  if (validate_desc(desc) != SPECMOE_OK) return 0;
  const specmoe_verify_desc d = sized(desc);
  return validate_desc(&d) == SPECMOE_OK ? make_plan(&d).ws_bytes : 0;
}

int specmoe_verify_attn_kv4(const void* q, const specmoe_kv4* cache, const int32_t* block_table,
                            const int32_t* ctx_lens, const int32_t* chunk_lens, const uint64_t* draft_mask, float scale,
                            void* out, float* lse, void* stream, const specmoe_verify_desc* desc,
                            const specmoe_paged_kv* paged) {
  const bool tree = draft_mask != nullptr;
  int st = validate_call(desc, tree, paged);
  if (st != SPECMOE_OK) return st;
  if (desc->flags != 0) return SPECMOE_ERR_FLAGS;
  if (block_table && !paged) return SPECMOE_ERR_NULL_POINTER;
  // (tiles here hold 128 keys whatever the type)
  if ((int64_t)kMaxSeqs * desc->Hkv * ((desc->S_max + (int64_t)kTile - 1) / kTile + kUnitCost) >= ((int64_t)1 << 31))
    return SPECMOE_ERR_SHAPE;
  const specmoe_verify_desc d = sized(desc);
  st = validate_desc(&d);
  if (st != SPECMOE_OK) return st;
  if (desc->B == 0) return SPECMOE_OK;   // nothing to read or write
  if (!cache) return SPECMOE_ERR_NULL_POINTER;
  Kv4Params p;
  Plan pl;
  if (!cache->k_scales || !cache->v_scales) return SPECMOE_ERR_NULL_POINTER;
  st = make_params(q, cache->k_codes, cache->v_codes, ctx_lens, chunk_lens, draft_mask, tree, scale, out, lse, &d,
                   block_table, paged, p, pl);
  if (st != SPECMOE_OK) return st;
  if (!aligned16(cache->k_scales) || !aligned16(cache->v_scales)) return SPECMOE_ERR_ALIGN;
  // (workgroups read the queries of some units while others store results)
  const size_t rows = (size_t)desc->B * desc->C_max * desc->Hq;
  const size_t row_bytes = (size_t)desc->D * (desc->dtype == SPECMOE_F32 ? 4 : 2);
  if (overlap(q, rows * row_bytes, out, rows * row_bytes) || overlap(q, rows * row_bytes, lse, rows * sizeof(float)) ||
      overlap(out, rows * row_bytes, lse, rows * sizeof(float)))
    return SPECMOE_ERR_OVERLAP;
  if (!paged) p.block_table = nullptr;
  p.k_scales = static_cast<const char*>(cache->k_scales);
  p.v_scales = static_cast<const char*>(cache->v_scales);
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();  // clear a stale error from unrelated work
  if (desc->dtype == SPECMOE_BF16) launch_kv4_for<kBF16>(desc->D, p, s);
  else if (desc->dtype == SPECMOE_F16) launch_kv4_for<kF16>(desc->D, p, s);
  else launch_kv4_for<kF32>(desc->D, p, s);
  return hipGetLastError() == hipSuccess ? SPECMOE_OK : SPECMOE_ERR_LAUNCH;
}

}  // extern "C"
