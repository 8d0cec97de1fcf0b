// Sampling of tokens from given random numbers, and acceptance by sampling, for
// MI355X (gfx950, CDNA4).
//
// The tokens of a row, in order of falling logit x (equal ones by index), have
// weights w = exp((x - max) / T).  Each setting keeps a prefix of that order,
// so what it keeps is known by its mass: top_k's is the mass of k tokens,
// top_p's the smallest prefix mass that reaches a share of it, min_p's the mass
// of all w >= min_p.  The kept mass Z is the least of them, and the token is
// the one at which the running mass passes u Z.  All three are searches for a
// position (a count or a mass) in the same order:
//   * weights are integers in units of 2^-42 of the best one's, so sums are
//     exact and the same in every order: histograms are filled with atomics;
//   * histogram bins are runs of the logits' own bit patterns, in order: the
//     leading bits name a bin without arithmetic, and bins are fine where
//     floating-point numbers are.  bf16 logits have a bin per value, so a bin's
//     tokens weigh the same: the pass over the row only counts (weighing every
//     token in fp64 took 11 of a row's 22 us), masses are counts times one
//     weight, and a position in a bin is a division.  fp32 logits take 64 bins
//     per octave and add their weights; a bin's tokens are listed and put in
//     order by comparing all with all;
//   * bins cover the numbers from the maximum to where weights vanish.  Where
//     those have too many patterns, the ones nearest to 0 (there are patterns
//     without end, but hardly a token) share one bin that is searched by list.
//     bf16 logits below 64, as nearly all are, need no maximum for that: one
//     layout of bins does for them, and a row is counted while it is loaded;
//   * with a small top_k only the best tokens matter: a histogram of the
//     threads' maxima gives a bin edge that at least k tokens pass, and those
//     alone are listed and weighed.
// One workgroup per row holds the row in LDS when it fits (two rows of up to
// 62.5 KB per CU), so the logits are read from HBM once.  2048 bf16 rows of
// 32000 tokens (131 MB, 26 us at a copy's rate) take 59 us with everything
// kept, 42 with top-50 and 26 greedily: what a row does after its load, 1000
// instructions per wave and a dozen barriers, is not hidden by the one other
// row on its CU.  64 fp32 rows take 28 us (the fp64 weights of a row on one
// CU), one bf16 row with every setting on 8.
#include <hip/hip_runtime.h>

#include <limits.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "accept_plan.h"
#include "specmoe_sample.h"

namespace {

typedef unsigned long long u64;

constexpr int kList = 256;                 // tokens put in order at once
constexpr int kBest = 128;                 // top_k for which about 150 tokens pass the 512 threads' maxima
constexpr int kMaxVocab = 1 << 20;         // weights of 2^42 add up below 2^63
constexpr int kMaxRows = 1 << 22;          // (a launch holds less than 2^32 threads)
constexpr int kUnit = 42;                  // weights are in units of 2^-42
constexpr double kMost = 43.0;             // from 2^-43 on a weight is less than half a unit
constexpr int kModeIeee = 1 | (9 << 6);    // s_setreg operand: bit 9 of the MODE register

// Rows of up to kRowSmall bytes (fp32: kRowSmallF32, whose bins hold masses too) leave room for two
// workgroups in a CU's 160 KB of LDS beside 16.3 (24.3) KB of bins and 200 bytes, with 1 (0.5) KB to
// spare; rows up to kRowLarge for one; longer ones are read again from the caches.
constexpr int kLds = 160 << 10;
constexpr int kRowSmall = 64000, kRowSmallF32 = 56320, kRowLarge = 138240;

struct Params {
  const char* logits;
  const float* uniforms;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* sampled;
  float* logprobs;
  int64_t stride;   // bytes
  int V, C_max;
  // acceptance only
  const int32_t* chunk_lens;
  const int32_t* ctx_lens;
  const int32_t* tokens;
  const uint64_t* draft_mask;
  int32_t* accepted;
  int32_t* next_token;
  int32_t* new_ctx;
  uint64_t* path;
  int* counters;
};

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// A token in the list: by falling logit, then by rising index, and its weight.
struct Entry {
  u64 order;    // (key << 32) | ~index: larger ones come first
  u64 weight;
};

// values that every lane holds, moved to scalar registers
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ u64 uniform(u64 x) {
  return (u64)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ __forceinline__ double uniform(double x) { return __longlong_as_double(uniform((u64)__double_as_longlong(x))); }

// bits that sort as the values do (no NaN); -0 counts as 0
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

// the leading 16 bits of a key as they are, -0 below 0
__device__ __forceinline__ int key_bits(float x) {
  const uint32_t u = __float_as_uint(x);
  return (int)((u ^ ((uint32_t)((int)u >> 31) | 0x80000000u)) >> 16);
}

__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// Fold of the wave's values, in every lane; inclusive prefix sums: shifts within
// each 16-lane row, then row ends broadcast into the rows after them (DPP
// moves; shuffles go through LDS).
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp(int old, int x) { return __builtin_amdgcn_update_dpp(old, x, CTRL, ROWS, 0xf, false); }
template <class OP>
__device__ __forceinline__ int wave_all(int x, OP op) {
  x = op(x, dpp<0x111, 0xf>(x, x));   // row_shr:1
  x = op(x, dpp<0x112, 0xf>(x, x));   // row_shr:2
  x = op(x, dpp<0x114, 0xf>(x, x));   // row_shr:4
  x = op(x, dpp<0x118, 0xf>(x, x));   // row_shr:8
  x = op(x, dpp<0x142, 0xa>(x, x));   // row_bcast:15 into rows 1 and 3
  x = op(x, dpp<0x143, 0xc>(x, x));   // row_bcast:31 into rows 2 and 3
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ int wave_max(int x) { return wave_all(x, [](int a, int b) { return max(a, b); }); }
__device__ __forceinline__ float wave_max(float x) {
  return __int_as_float(wave_all(__float_as_int(x), [](int a, int b) {
    return __float_as_int(fmaxf(__int_as_float(a), __int_as_float(b)));
  }));
}
__device__ __forceinline__ int wave_prefix(int x) {
  x += dpp<0x111, 0xf>(0, x);
  x += dpp<0x112, 0xf>(0, x);
  x += dpp<0x114, 0xf>(0, x);
  x += dpp<0x118, 0xf>(0, x);
  x += dpp<0x142, 0xa>(0, x);
  x += dpp<0x143, 0xc>(0, x);
  return x;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp64(u64 x) {
  return (u64)(uint32_t)dpp<CTRL, ROWS>(0, (int)(x >> 32)) << 32 | (uint32_t)dpp<CTRL, ROWS>(0, (int)x);
}
template <class T>
__device__ __forceinline__ T row_prefix(T x) {   // within each 16 lanes
  if constexpr (sizeof(T) == 8) {
    x += dpp64<0x111, 0xf>(x);
    x += dpp64<0x112, 0xf>(x);
    x += dpp64<0x114, 0xf>(x);
    x += dpp64<0x118, 0xf>(x);
  } else {
    x += dpp<0x111, 0xf>(0, x);
    x += dpp<0x112, 0xf>(0, x);
    x += dpp<0x114, 0xf>(0, x);
    x += dpp<0x118, 0xf>(0, x);
  }
  return x;
}
__device__ __forceinline__ u64 lane_of(u64 x, int lane) {
  return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}
__device__ __forceinline__ u64 wave_prefix(u64 x) {
  x += dpp64<0x111, 0xf>(x);
  x += dpp64<0x112, 0xf>(x);
  x += dpp64<0x114, 0xf>(x);
  x += dpp64<0x118, 0xf>(x);
  x += dpp64<0x142, 0xa>(x);
  x += dpp64<0x143, 0xc>(x);
  return x;
}

// A constant in scalar registers: fp64 operations take no literals, and vector
// registers are short.
__device__ __forceinline__ double scalar(double x) {
  asm("" : "+s"(x));
  return x;
}

// 2^f for |f| <= 1/2: the polynomial of degree 9 through 2^f at the Chebyshev
// nodes of the interval, off by less than 2^-45 absolutely (2^-45.05 at 1/2) and
// by 2^-44.6 of the value (at -1/2): a quarter of the half unit, 2^-43 of the
// best token's, by which a weight is rounded.
__device__ __forceinline__ double exp2_poly(double f) {
  double q = fma(scalar(1.020590550210069e-07), f, scalar(1.3259645241948732e-06));
  q = fma(q, f, scalar(1.5252672924257465e-05));
  q = fma(q, f, scalar(0.0001540343375126647));
  q = fma(q, f, scalar(0.0013333558200796013));
  q = fma(q, f, scalar(0.00961812919393429));
  q = fma(q, f, scalar(0.05550410866465166));
  q = fma(q, f, scalar(0.2402265069564034));
  q = fma(q, f, scalar(0.6931471805599462));
  return fma(q, f, 1.0);
}

// One row's sampling, by all threads of a workgroup.
template <bool BF16, int kRowLds, int kThreads>
struct Row {
  static constexpr int kWaves = kThreads / 64;
  static constexpr int kElt = BF16 ? 2 : 4;
  static constexpr int kPer = 16 / kElt;             // logits per 16-byte vector
  static constexpr int kBins = BF16 ? 4096 : 2048;   // fp32 ones have a mass of 8 bytes each beside the count
  static constexpr int kOwn = kBins / kThreads;      // bins per thread
  static constexpr int kGroup = BF16 ? 8 : kOwn;     // patterns of one sign and octave, whatever kThreads
  static constexpr int kDrop = BF16 ? 16 : 17;       // key bits that a bin does not look at
  static constexpr int kZero = 0x80000000u >> kDrop; // the bin pattern of +0; -0 has the one below

  struct Shared {
    __attribute__((aligned(16))) char row[kRowLds ? kRowLds : 16];
    union {
      struct {
        int count[kBins + 64];   // (and a spare one per lane)
        u64 mass[BF16 ? 1 : kBins];
      } hist;
      Entry list[kList];
      int indices[kList];
    };
    u64 part_mass[kWaves];
    int part_count[kWaves];
    float part_max[kWaves];
    u64 middle, middle_above;   // mass of the tokens nearest to 0, and of those that min_p keeps
    u64 above;                  // mass that min_p keeps
    u64 found_mass, before, weight;
    float found_logit;
    int found_index, bin, count_before, n, n_list;
  };

  const Params& p;
  Shared& sh;
  const char* src;   // the row in memory
  int tid, lane, wave, nvec;
  float m;
  double md, c;      // the maximum, log2(e) / T
  double cut;        // min_p in weight units (0: off)
  // The bins of the patterns K (keys without their last bits), in order: those
  // from base (top, the maximum's, rounded up to a whole group) down to base -
  // reach.  A thread's bins are patterns of one group.  Where there are too
  // many, whole groups around 0 share the kOwn bins from `mid` on (-1: none),
  // down to the pattern base - skip - kOwn + 1.  Layouts, and so what shares
  // bins, do not depend on kThreads for bf16.
  int top, base, reach, mid, skip;

  __device__ __forceinline__ Row(const Params& p_, Shared& sh_, const char* src_)
      : p(p_), sh(sh_), src(src_), tid(threadIdx.x), lane(threadIdx.x & 63), wave(uniform((int)threadIdx.x >> 6)),
        nvec((p_.V + kPer - 1) / kPer) {}

  static __device__ __forceinline__ float entry(const u32x4& x, int e) {
    if constexpr (BF16) return __uint_as_float((e & 1) ? (x[e >> 1] & 0xffff0000u) : (x[e >> 1] << 16));
    else return __uint_as_float(x[e]);
  }

  // vector v of the row in memory; -inf beyond its end
  __device__ __forceinline__ u32x4 fetch(int v) const {
    u32x4 x;
    const char* at = src + (size_t)v * 16;
    if ((v + 1) * kPer <= p.V) {
      __builtin_memcpy(&x, at, 16);   // (rows may start at any element)
      return x;
    }
    const int left = p.V - v * kPer;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (BF16) {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(at);
        const uint32_t lo = 2 * w < left ? h[2 * w] : 0xff80u, hi = 2 * w + 1 < left ? h[2 * w + 1] : 0xff80u;
        x[w] = lo | hi << 16;
      } else {
        x[w] = w < left ? reinterpret_cast<const uint32_t*>(at)[w] : 0xff800000u;
      }
    }
    return x;
  }
  __device__ __forceinline__ u32x4 vec(int v) const {
    if constexpr (kRowLds > 0) return *reinterpret_cast<const u32x4*>(sh.row + (size_t)v * 16);
    else return fetch(v);
  }

  // a token's logit, by index
  __device__ __forceinline__ float logit_at(int index) const {
    const char* row = kRowLds > 0 ? sh.row : src;
    if constexpr (BF16) return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(row + 2 * (size_t)index) << 16);
    else return *reinterpret_cast<const float*>(row + 4 * (size_t)index);
  }

  // every token that want(x) holds for: f(x, index).  Few do: a vector's are
  // found first, then taken one by one.
  template <class WANT, class F>
  __device__ __forceinline__ void each(WANT want, F f) const {
    constexpr int kAhead = kRowLds ? 1 : 4;   // vectors read at once
    for (int v0 = tid; v0 < nvec; v0 += kAhead * kThreads) {
      u32x4 x[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) x[j] = vec(min(v0 + j * kThreads, nvec - 1));
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int v = v0 + j * kThreads;
        uint32_t found = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) found |= want(entry(x[j], e)) ? 1u << e : 0u;
        while (found && v < nvec) {
          const int index = v * kPer + __builtin_ctz(found);
          found &= found - 1;
          if (index < p.V) f(logit_at(index), index);
        }
      }
    }
  }

  // 2^(units - y) for y >= 0, at most 2^-18 from 2^-60 on and for NaN.  Additions
  // of 1.5 x 2^52 and 2^52 (whole) round to integers in the low bits of a double,
  // and a power of two goes straight into the exponent: the conversions and
  // ldexp take four times an addition's cycles.
  static __device__ __forceinline__ double power(double y, int units) {
    constexpr double kRound = 6755399441055744.0;
    y = fmin(y, 60.0);
    const double t = y + kRound;
    const double q = exp2_poly((t - kRound) - y);
    return __hiloint2double(__double2hiint(q) + ((units - __double2loint(t)) << 20), __double2loint(q));
  }
  static __device__ __forceinline__ u64 whole(double exact) {
#pragma clang fp contract(off)   // (no rounding less where `exact` is a product)
    return (u64)__double_as_longlong(exact + 4503599627370496.0) & 0xfffffffffffffull;
  }
  // weight in units, and the same before it was rounded (finite maximum)
  __device__ __forceinline__ u64 weight(float x, double& exact) const {
    exact = power((md - (double)x) * c, kUnit);
    return whole(exact);
  }

  // loads the row and returns its maximum, -inf for a row without any mass
  __device__ __forceinline__ float load(float& mine) {
    float hi = -INFINITY;
    // 16-byte loads per lane in flight: 8 with 8 waves (2048 rows of 32000 bf16
    // 30.1 -> 26.2 us greedily, top-50 44.5 -> 42) and for fp32 rows that fit no
    // LDS (one of 151936 16.0 -> 14.1 us; 64 of bf16 11.6 -> 12.4)
    constexpr int kBatch = kThreads == 512 ? 8 : kRowLds || BF16 ? 4 : 8;
    for (int v0 = tid; v0 < nvec; v0 += kBatch * kThreads) {
      u32x4 x[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (v0 + u * kThreads < nvec) x[u] = fetch(v0 + u * kThreads);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (v0 + u * kThreads >= nvec) continue;
        if constexpr (kRowLds > 0) *reinterpret_cast<u32x4*>(sh.row + (size_t)(v0 + u * kThreads) * 16) = x[u];
#pragma unroll
        for (int e = 0; e < kPer; ++e) hi = fmaxf(hi, entry(x[u], e));
      }
    }
    mine = hi;
    return row_max(hi);
  }
  __device__ __forceinline__ float row_max(float hi) {
    hi = wave_max(hi);
    if (lane == 0) sh.part_max[wave] = hi;
    __syncthreads();
    return wave_max(sh.part_max[lane & (kWaves - 1)]);
  }

  // (bf16) The bins of most rows, laid before the maximum is known: all
  // patterns of kAround <= |x| < 64, those nearer to 0 in one group.
  static constexpr int kUsualBase = 0xc27f, kUsualMid = kBins / 2 - kGroup;   // (just below 64)
  static constexpr int kAround = kUsualBase + 1 - kZero - kUsualMid;        // (a pattern: 2^-10)
  static constexpr int kUsualSkip = kUsualBase + 1 - kZero + kAround - kOwn;
  static constexpr int kUsualReach = kUsualSkip + kBins - 1 - kUsualMid;
  static constexpr int kNearShift = kRowLds ? 0 : 2;   // vectors of a thread per bit, as a power of two: up to 128 of them
  static_assert(!BF16 || ((kMaxVocab / 8 / kThreads) >> kNearShift) <= 32 || kRowLds > 0, "a bit for each");

  // (bf16) Loads the row and counts its tokens into those bins.  Returns the
  // largest pattern, and in `near` which of the thread's vectors hold tokens
  // around 0.  (load() and fill() one after the other took 12 instructions per
  // token, not 8, and nothing overlapped the loads: 2048 rows of 32000, 80 us
  // with everything kept and 79 with top-p 0.9, then 68 and 68.)
  __device__ __forceinline__ int load_counting(uint32_t& near) {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    typedef __attribute__((ext_vector_type(2))) short i16x2;
    auto both = [](int x) { return u16x2{(unsigned short)x, (unsigned short)x}; };
    // what lies outside the bins, NaN among it, counts in a spare one of its lane
    const u16x2 out2 = both(kUsualReach + 1 + lane);
    char* const counts = reinterpret_cast<char*>(sh.hist.count);
    constexpr int kBatch = 4;   // 16-byte loads per lane in flight, while as many are counted (8: 2 us more)
    u32x4 next[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (tid + u * kThreads < nvec) next[u] = fetch(tid + u * kThreads);
    __syncthreads();   // the bins are clear
    u16x2 best = both(0);
    near = 0;
    int j = 0;
    for (int v0 = tid; v0 < nvec; v0 += kBatch * kThreads) {
      u32x4 x[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) x[u] = next[u];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (v0 + (kBatch + u) * kThreads < nvec) next[u] = fetch(v0 + (kBatch + u) * kThreads);
#pragma unroll
      for (int u = 0; u < kBatch; ++u, ++j) {
        if (v0 + u * kThreads >= nvec) continue;
        if constexpr (kRowLds > 0) *reinterpret_cast<u32x4*>(sh.row + (size_t)(v0 + u * kThreads) * 16) = x[u];
        u16x2 least = both(0x7fff);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t word = x[u][w];
          const uint32_t sign = __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, word) >> (short)15);
          const u16x2 K = __builtin_bit_cast(u16x2, word ^ (sign | 0x80008000u));
          best = __builtin_elementwise_max(best, K);
          least = __builtin_elementwise_min(least, __builtin_bit_cast(u16x2, word & 0x7fff7fffu));
          const u16x2 d = __builtin_elementwise_min((u16x2)(both(kUsualBase) - K), out2);
          const u16x2 bin = (u16x2)(__builtin_elementwise_min(d, both(kUsualMid)) +
                                    __builtin_elementwise_sub_sat(d, both(kUsualSkip))) << (unsigned short)2;
          atomicAdd(reinterpret_cast<int*>(counts + bin[0]), 1);
          atomicAdd(reinterpret_cast<int*>(counts + bin[1]), 1);
        }
        if (least[0] < kAround || least[1] < kAround) near |= 1u << (j >> kNearShift);
      }
    }
    const int hi = wave_max((int)max(best[0], best[1]));
    if (lane == 0) sh.part_count[wave] = hi;
    __syncthreads();
    return uniform(wave_max(sh.part_count[lane & (kWaves - 1)]));
  }
  // The masses of the tokens around 0 in the vectors that `near` names.
  __device__ __forceinline__ void weigh_near(uint32_t near) {
    if (!near) return;
    u64 sum = 0, above = 0;
    for (; near; near &= near - 1) {
      const int j0 = __builtin_ctz(near) << kNearShift;
#pragma unroll 1
      for (int j = j0; j < j0 + (1 << kNearShift); ++j) {
        const int v = tid + j * kThreads;
        if (v >= nvec) break;
        const u32x4 x = vec(v);
        uint32_t found = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) found |= ((x[e >> 1] >> (16 * (e & 1))) & 0x7fffu) < (uint32_t)kAround ? 1u << e : 0u;
        for (; found; found &= found - 1) {
          double exact;
          const u64 w = weight(logit_at(v * kPer + __builtin_ctz(found)), exact);
          sum += w;
          above += exact >= cut ? w : 0;
        }
      }
    }
    atomicAdd(&sh.middle, sum);
    if (cut > 0.0) atomicAdd(&sh.middle_above, above);
  }

  // sums over the workgroup of what the threads before hold, and the total
  __device__ __forceinline__ void scan(int n, u64 w, int& n_before, u64& w_before, int& n_all, u64& w_all) {
    const int ni = wave_prefix(n);
    const u64 wi = wave_prefix(w);
    __syncthreads();   // (the last scan's totals have been read)
    if (lane == 63) {
      sh.part_count[wave] = ni;
      sh.part_mass[wave] = wi;
    }
    __syncthreads();
    // the waves' totals, one per lane, summed in the first lanes
    static_assert(kWaves <= 16, "totals in one row of lanes");
    const int np = row_prefix(sh.part_count[lane & (kWaves - 1)]);
    const u64 wp = row_prefix(sh.part_mass[lane & (kWaves - 1)]);
    n_before = ni - n;
    w_before = wi - w;
    if (wave > 0) {
      n_before += __builtin_amdgcn_readlane(np, wave - 1);
      w_before += lane_of(wp, wave - 1);
    }
    n_all = __builtin_amdgcn_readlane(np, kWaves - 1);
    w_all = lane_of(wp, kWaves - 1);
  }

  __device__ __forceinline__ void clear_hist() {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      sh.hist.count[tid + k * kThreads] = 0;
      if constexpr (!BF16) sh.hist.mass[tid + k * kThreads] = 0;
    }
  }

  // below it, weights vanish
  __device__ __forceinline__ double least_weighed(double T) const { return md - (kMost + 0.01) * 0.69314718055994530942 * T; }

  // the bins of this row: from its maximum down to where weights vanish
  __device__ __forceinline__ void lay_bins(double T) {
    const double end = least_weighed(T);
    const float least = end > -3.4028234663852886e38 ? (float)end : -3.4028234663852886e38f;   // (NaN: the least number)
    top = uniform((int)(key_of(m) >> kDrop));
    int bottom = min(uniform((int)(key_of(least) >> kDrop)), top);
    if (bottom == kZero) --bottom;   // -0 with 0
    base = top | (kGroup - 1);
    reach = base - bottom;
    mid = -1;
    skip = reach + 1;
    if (reach >= kBins) {
      // patterns at least a (a whole group) away from 0's on either side keep
      // their bins
      const int above = base + 1 - kZero, below = kZero - bottom;
      int a = (above + below + kGroup - kBins + 1) / 2;
      if (a > min(above, below)) a = max(above, below) + kGroup - kBins;
      a = (a + kGroup - 1) / kGroup * kGroup;
      mid = max(base + 1 - (kZero + a), 0);
      skip = base - (kZero - 1 - a) - kOwn;
    }
  }
  // (for patterns K from base - reach to base)
  __device__ __forceinline__ int bin_of(int K) const {
    const int d = base - K;
    return (mid >= 0 ? min(d, mid) : d) + max(d, skip) - skip;
  }
  __device__ __forceinline__ bool in_middle(int bin) const { return mid >= 0 && (uint32_t)(bin - mid) < (uint32_t)kOwn; }
  // the largest pattern of a bin (of the middle: of all of them)
  __device__ __forceinline__ int pattern_of(int bin) const {
    return base - (mid < 0 || bin <= mid ? bin : bin - mid + skip);
  }
  // the keys of a bin
  __device__ __forceinline__ void keys_of(int bin, uint32_t& lo, uint32_t& hi) const {
    const int last = in_middle(bin) ? base - mid : pattern_of(bin);
    const int first = in_middle(bin) ? max(base - skip - kOwn + 1, base - reach) : last;
    lo = (uint32_t)first << kDrop;
    hi = ((uint32_t)last << kDrop) | ((1u << kDrop) - 1u);
  }

  // (bf16) the value of a pattern
  static __device__ __forceinline__ float value_at(int K) {
    const uint32_t key = (uint32_t)K << kDrop;
    return value_of(K >= kZero ? key : key | ((1u << kDrop) - 1u));   // (a negative number's key is its complement)
  }

  // Lists the tokens with keys from lo to hi and their weights; returns how many
  // there are, of which the first kList are listed.  TOP: hi is the maximum's
  // key, so that a vector's own maximum tells whether it has any.
  template <bool TOP>
  __device__ __forceinline__ int gather(uint32_t lo, uint32_t hi) {
    __syncthreads();
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    const float least = value_of(lo);
    constexpr int kSpan = 64 / kPer;   // vectors of a lane whose finds fit 64 bits
    constexpr int kAhead = kRowLds ? 2 : 4;   // of them read at once
    for (int c0 = 0; c0 < nvec; c0 += kSpan * kThreads) {
      u64 found = 0;
      for (int j0 = 0; j0 < kSpan; j0 += kAhead) {
        u32x4 x[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) x[j] = vec(min(c0 + (j0 + j) * kThreads + tid, nvec - 1));
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          bool some = c0 + (j0 + j) * kThreads + tid < nvec;
          if constexpr (TOP) {
            float most = entry(x[j], 0);
#pragma unroll
            for (int e = 1; e < kPer; ++e) most = fmaxf(most, entry(x[j], e));
            some = some && most >= least;
          }
          if (some) {
            uint32_t in = 0;
#pragma unroll
            for (int e = 0; e < kPer; ++e)
              in |= (TOP ? entry(x[j], e) >= least : key_of(entry(x[j], e)) - lo <= hi - lo) ? 1u << e : 0u;
            found |= (u64)in << (kPer * (j0 + j));
          }
        }
        if (c0 + (j0 + kAhead) * kThreads >= nvec) break;
      }
      // one place in the list per wave, then one per lane
      const int n = __popcll(found), upto = wave_prefix(n);
      int at = 0;
      if (lane == 63 && upto) at = atomicAdd(&sh.n_list, upto);
      at = __builtin_amdgcn_readlane(at, 63) + upto - n;
      for (; found && at < kList; found &= found - 1, ++at) {
        const int bit = __builtin_ctzll(found);
        sh.list[at].order = (u64)(uint32_t)((c0 + bit / kPer * kThreads + tid) * kPer + bit % kPer);
      }
    }
    __syncthreads();
    // (a thread each: weighed where they were found, nearly every vector of a
    // wave took one wave's time for one token)
    const int n = uniform(sh.n_list);
    if (tid < min(n, kList)) {
      const uint32_t index = (uint32_t)sh.list[tid].order;
      const float x = logit_at(index);
      double exact;
      sh.list[tid] = Entry{(u64)key_of(x) << 32 | ~index, weight(x, exact)};
    }
    __syncthreads();
    return n;
  }

  // The place of list entry tid / g among the n listed: the entries and the
  // mass before it.  g threads share an entry's comparisons, so that each has
  // few and their sums few steps.
  __device__ __forceinline__ int groups(int n) const {   // (n <= kList)
    int g = kThreads / kList;
    while (g < 8 && 2 * g * n <= kThreads) g *= 2;
    return g;
  }
  __device__ __forceinline__ void place(int n, int g, int& rank, u64& before) const {
    const int e = tid >> __builtin_ctz(g);
    rank = 0;
    before = 0;
    if (e < n) {
      const u64 own = sh.list[e].order;
#pragma unroll 4
      for (int f = tid & (g - 1); f < n; f += g) {
        const Entry o = sh.list[f];
        if (o.order > own) {
          ++rank;
          before += o.weight;
        }
      }
    }
    for (int d = 1; d < g; d <<= 1) {
      rank += __shfl_xor(rank, d);
      before += __shfl_xor(before, d);
    }
  }

  // (bf16) Lists the indices of the n <= kList tokens of logit `value`, in any
  // order: words with a half of its bits first (x has a zero half where (x -
  // 0x00010001) & ~x has a half's leading bit, or a half above a zero one).
  __device__ __forceinline__ void list_equal(float value, int n) {
    const uint32_t bits = __float_as_uint(value) >> 16, pair = bits | bits << 16;
    for (int v = tid; v < nvec; v += kThreads) {
      const u32x4 x = vec(v);
      uint32_t hit = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t y = x[w] ^ pair;
        hit |= (y - 0x00010001u) & ~y;
      }
      if (value == 0.f) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t y = x[w] ^ pair ^ 0x80008000u;   // -0 with 0
          hit |= (y - 0x00010001u) & ~y;
        }
      }
      if (hit & 0x80008000u) {
        uint32_t found = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) found |= entry(x, e) == value ? 1u << e : 0u;
        for (; found; found &= found - 1)   // (value is finite: none beyond the row's end)
          sh.indices[n > 1 ? atomicAdd(&sh.n_list, 1) & (kList - 1) : 0] = v * kPer + __builtin_ctz(found);
      }
    }
  }

  // The `nth` token by index among those of logit `value`.
  __device__ __forceinline__ void find_nth(float value, int nth) {
    int seen = 0;
    for (int v0 = 0; v0 < nvec; v0 += kThreads) {
      const int v = v0 + tid;
      int mine = 0;
      u32x4 x = {0u, 0u, 0u, 0u};
      if (v < nvec) {
        x = vec(v);
#pragma unroll
        for (int e = 0; e < kPer; ++e) mine += entry(x, e) == value;
      }
      int nb, na;
      u64 wb, wa;
      scan(mine, 0, nb, wb, na, wa);
      if (nth >= seen + nb && nth < seen + nb + mine) {
        int k = nth - seen - nb;
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          if (entry(x, e) == value && k-- == 0) sh.found_index = v * kPer + e;
      }
      seen += na;
    }
  }

  // The token at position `left` (a count or a mass) among those with keys from
  // lo to hi, with mass `before` before them.
  __device__ __forceinline__ void search_keys(uint32_t lo, uint32_t hi, bool by_count, u64 left, u64 before) {
    int n = gather<false>(lo, hi);
    // Many tokens (nearly equal logits, a bin around 0, long rows): the keys are
    // cut into ranges until one holds a list's or a single key's.  1024 ranges,
    // of counts and masses in the list's place.
    constexpr int kParts = 1024, kHalves = kParts / kThreads;
    static_assert(sizeof(sh.hist) >= kParts * 12, "room for the ranges");
    int* const count = reinterpret_cast<int*>(&sh.hist);
    u64* const mass = reinterpret_cast<u64*>(count + kParts);
    for (int level = 0; level < 4 && n > kList && lo != hi; ++level) {   // (ten bits of the key each)
      const uint32_t span = hi - lo;
      const int shift = max(0, 32 - __builtin_clz(span) - 10);   // span >> shift < kParts
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kHalves; ++k) {
        count[tid + k * kThreads] = 0;
        mass[tid + k * kThreads] = 0;
      }
      __syncthreads();
      each([&](float x) { return key_of(x) - lo <= span; },
           [&](float x, int) {
             double exact;
             const u64 w = weight(x, exact);
             const uint32_t key = key_of(x), part = (hi - key) >> shift;
             // lanes with the first one's key (rows of zeros) add together
             const bool same = key == (uint32_t)uniform((int)key);
             const u64 who = __ballot(same);
             const int times = same ? __popcll(who) : 1;
             if (!same || lane == __builtin_ctzll(who)) {
               if (w) atomicAdd(&mass[part], w * (u64)times);
               atomicAdd(&count[part], times);   // (a count goes over tokens without weight, too)
             }
           });
      __syncthreads();
      int n_in[kHalves], n_sum = 0;
      u64 w_in[kHalves], w_sum = 0;
#pragma unroll
      for (int k = 0; k < kHalves; ++k) {
        n_in[k] = count[tid * kHalves + k];
        w_in[k] = mass[tid * kHalves + k];
        n_sum += n_in[k];
        w_sum += w_in[k];
      }
      int nb, na;
      u64 wb, wa;
      scan(n_sum, w_sum, nb, wb, na, wa);
#pragma unroll
      for (int k = 0; k < kHalves; ++k) {
        const u64 b0 = by_count ? (u64)nb : wb, size = by_count ? (u64)n_in[k] : w_in[k];
        if (left >= b0 && left - b0 < size) {
          sh.bin = tid * kHalves + k;
          sh.before = wb;
          sh.count_before = nb;
          sh.n = n_in[k];
        }
        nb += n_in[k];
        wb += w_in[k];
      }
      __syncthreads();
      n = uniform(sh.n);
      before += sh.before;
      left -= by_count ? (u64)sh.count_before : sh.before;
      hi -= (uint32_t)sh.bin << shift;
      lo = max(lo, hi - ((1u << shift) - 1u));
      if (n <= kList) n = gather<false>(lo, hi);
    }
    if (n <= kList) {
      const int g = groups(n);
      int rank;
      u64 inside;
      place(n, g, rank, inside);
      const int e = tid >> __builtin_ctz(g);
      if (e < n && (tid & (g - 1)) == 0) {
        const Entry own = sh.list[e];
        const u64 at = by_count ? (u64)rank : inside;
        if (left >= at && left - at < (by_count ? 1 : own.weight)) {
          sh.found_index = (int)~(uint32_t)own.order;
          sh.found_logit = value_of((uint32_t)(own.order >> 32));
          sh.found_mass = before + inside + own.weight;
        }
      }
      return;
    }
    // one key: its tokens weigh the same, and are counted by index
    const float value = value_of(lo);
    double exact;
    const u64 w = weight(value, exact);
    const int nth = (int)(by_count ? left : w ? left / w : 0);
    find_nth(value, nth);
    if (tid == 0) {
      sh.found_logit = value;
      sh.found_mass = before + (u64)(nth + 1) * w;
    }
  }

  // the position just before a share of a mass is reached
  static __device__ __forceinline__ u64 share_end(float share, u64 mass) {
    const double want = ceil((double)share * (double)mass);
    const u64 w = want >= 1.0 ? (u64)want : 1;
    return min(w, mass) - 1;
  }
  static __device__ __forceinline__ u64 share_of(float u, u64 mass) {
    const double at = u > 0.f ? (double)u * (double)mass : 0.0;   // (NaN: 0)
    return at < (double)mass ? min((u64)at, mass - 1) : mass - 1;
  }

  // log of a token's share of the kept mass (the same operations in every kernel)
  __device__ __forceinline__ float log_share(float x, u64 kept) const {
#pragma clang fp contract(off)
    const double d = ((double)x - md) * (c * 0.69314718055994530942);
    return (float)(d - log((double)kept * (1.0 / (double)(1ull << kUnit))));
  }

  // The row's token where only the best k <= kBest matter; false where too many
  // tokens tie with them.
  __device__ __forceinline__ bool draw_best(float u, int k, bool by_p, float top_p, float mine, int& token, float& logp) {
    // the bin edge that at least k threads' maxima pass
    const int K = key_of(mine) >> kDrop;
    if ((uint32_t)(base - K) <= (uint32_t)reach) atomicAdd(&sh.hist.count[bin_of(K)], 1);
    __syncthreads();
    int own[kOwn], sum = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      own[i] = sh.hist.count[tid * kOwn + i];
      sum += own[i];
    }
    int nb, na;
    u64 wb, wa;
    scan(sum, 0, nb, wb, na, wa);
    if (tid == 0 && na < k) sh.bin = -1;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      if (nb < k && k <= nb + own[i]) sh.bin = tid * kOwn + i;
      nb += own[i];
    }
    __syncthreads();
    const int edge = sh.bin;
    uint32_t lo = (uint32_t)(base - reach) << kDrop, hi;
    if (edge >= 0) keys_of(edge, lo, hi);
    const int n = gather<true>(lo, key_of(m));
    if (n > kList) return false;
    const int g = groups(n);
    int rank;
    u64 before;
    place(n, g, rank, before);
    const int e = tid >> __builtin_ctz(g);
    const bool owner = e < n && (tid & (g - 1)) == 0;
    Entry own_entry = {0, 0};
    if (owner) own_entry = sh.list[e];
    const u64 weight_e = own_entry.weight;
    const float logit = value_of((uint32_t)(own_entry.order >> 32));
    if (owner) {
      if (rank == min(k, n) - 1) sh.found_mass = before + weight_e;
      if (cut > 0.0) {
        // (min_p's mass: it reaches beyond the listed or ends among them)
        double exact;
        weight(logit, exact);
        if (exact >= cut) atomicMax(&sh.above, before + weight_e);
      }
    }
    __syncthreads();
    u64 kept = sh.found_mass;
    if (by_p) {
      const u64 position = share_end(top_p, kept);
      __syncthreads();
      if (owner && position >= before && position - before < weight_e) sh.found_mass = before + weight_e;
      __syncthreads();
      kept = sh.found_mass;
    }
    if (cut > 0.0) kept = min(kept, sh.above);
    const u64 position = share_of(u, kept);
    if (owner && position >= before && position - before < weight_e) {
      sh.found_index = (int)~(uint32_t)own_entry.order;
      sh.found_logit = logit;
    }
    __syncthreads();
    token = sh.found_index;
    if (wave == 0) logp = log_share(sh.found_logit, kept);
    return true;
  }

  // The token of a row with infinite logits: one of them, all weighing a unit.
  __device__ __forceinline__ void draw_infinite(float u, int k, bool by_p, float top_p, int& token, float& logp) {
    int mine = 0;
    each([&](float x) { return x == m; }, [&](float, int) { ++mine; });
    int nb, n;
    u64 wb, wa;
    scan(mine, 0, nb, wb, n, wa);
    u64 kept = (u64)min(n, k) << kUnit;
    if (by_p) kept = ((share_end(top_p, kept) >> kUnit) + 1) << kUnit;
    find_nth(m, (int)(share_of(u, kept) >> kUnit));
    __syncthreads();
    token = sh.found_index;
    logp = -(float)log((double)(kept >> kUnit));
  }

  // Counts (bf16) or weighs (fp32) every token into its bin.
  __device__ __forceinline__ void fill(bool by_k) {
    if constexpr (BF16) {
      // Two tokens per instruction, in 16-bit halves: with d = base - K, at most
      // reach + 1 (what lies below the bins and NaN, which wraps, too).  A token
      // outside the bins counts in a spare one of its lane: one for all would
      // be added to 64 times over.  (12 instructions per token with a branch or
      // a select for each, now 8.)
      typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
      typedef __attribute__((ext_vector_type(2))) short i16x2;
      auto both = [](int x) { return u16x2{(unsigned short)x, (unsigned short)x}; };
      const int most = mid < 0 ? reach + 1 : mid;
      const int last = min(reach + 1, most) + max(reach + 1 - skip, 0);   // the bin of d = reach + 1
      const u16x2 base2 = both(base), out2 = both(reach + 1), most2 = both(most), skip2 = both(skip),
                  reach2 = both(reach), spare2 = both(kBins + lane - last), mid2 = both(mid), group2 = both(~(kOwn - 1));
      char* const counts = reinterpret_cast<char*>(sh.hist.count);
      u64 around = 0, around_above = 0;
      u32x4 next = vec(min(tid, nvec - 1));   // (read ahead of the additions, which LDS serves in order)
      for (int v = tid; v < nvec; v += kThreads) {
        const u32x4 x = next;
        next = vec(min(v + kThreads, nvec - 1));
        u16x2 near = both(0xffff);   // zero once a token lies around 0: those weigh differently
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          // both halves' keys: negative numbers complemented, others' sign set
          const uint32_t word = x[w];
          const uint32_t sign = __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, word) >> (short)15);
          const u16x2 K = __builtin_bit_cast(u16x2, word ^ (sign | 0x80008000u));
          const u16x2 d = __builtin_elementwise_min((u16x2)(base2 - K), out2);
          u16x2 bin = __builtin_elementwise_min(d, most2);
          if (mid >= 0) {
            bin += (u16x2)(__builtin_elementwise_max(d, skip2) - skip2);
            near = __builtin_elementwise_min(near, (u16x2)((bin ^ mid2) & group2));
          }
          const u16x2 outside = __builtin_elementwise_sub_sat(d, reach2);   // 0 or 1
          bin = (u16x2)((outside * spare2 + bin) << (unsigned short)2);
          atomicAdd(reinterpret_cast<int*>(counts + bin[0]), 1);
          atomicAdd(reinterpret_cast<int*>(counts + bin[1]), 1);
        }
        if (near[0] == 0 || near[1] == 0) {
#pragma unroll 1
          for (int e = 0; e < kPer; ++e) {
            const int index = v * kPer + e;
            const float y = index < p.V ? logit_at(index) : -INFINITY;
            const int K = key_bits(y);
            if ((uint32_t)(base - K) <= (uint32_t)reach && in_middle(bin_of(K))) {
              double exact;
              const u64 u = weight(y, exact);
              around += u;
              around_above += exact >= cut ? u : 0;
            }
          }
        }
      }
      if (around) {
        atomicAdd(&sh.middle, around);
        if (cut > 0.0) atomicAdd(&sh.middle_above, around_above);
      }
    } else {
      // (a vector's weights side by side: one after the other, each waits for
      // its own polynomial)
      u64 passes = 0;
      constexpr int kAhead = kRowLds ? 1 : 4;   // vectors read ahead
      u32x4 next[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) next[j] = vec(min(tid + j * kThreads, nvec - 1));
      for (int v = tid; v < nvec; v += kThreads) {
        const u32x4 x = next[0];
#pragma unroll
        for (int j = 0; j + 1 < kAhead; ++j) next[j] = next[j + 1];
        next[kAhead - 1] = vec(min(v + kAhead * kThreads, nvec - 1));
        u64 w[kPer];
        double exact[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) w[e] = weight(entry(x, e), exact[e]);
        asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));   // (all before the first is used)
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const int K = key_of(entry(x, e)) >> kDrop;
          if (w[e] && (uint32_t)(base - K) <= (uint32_t)reach) {
            const int bin = bin_of(K);
            atomicAdd(&sh.hist.mass[bin], w[e]);
            if (by_k) atomicAdd(&sh.hist.count[bin], 1);
            if (cut > 0.0 && exact[e] >= cut) passes += w[e];
          }
        }
      }
      if (cut > 0.0 && passes) atomicAdd(&sh.above, passes);
    }
  }

  // The row's token, in every thread, and its log-probability, in the first wave's.
  __device__ __forceinline__ void draw(float u, float T, int k, float top_p, float min_p, int& token, float& logp) {
    clear_hist();
    if (tid == 0) {
      sh.middle = 0;
      sh.middle_above = 0;
      sh.above = 0;
      sh.found_index = INT_MAX;
    }
    const bool by_k = k > 0 && k < p.V, by_p = top_p < 1.f;   // (NaN: off)
    float mine = 0.f;
    uint32_t near = 0;
    // most rows whose tokens all have to be weighed are counted as they are
    // loaded, into the usual bins (those with a maximum of 64 or more, or NaN of
    // that sign, or weight below the bins, once more below)
    const bool best = by_k && k <= kBest;
    const bool all = BF16 && T > 0.f && k != 1 && !best && !(by_p && !(top_p > 0.f));
    bool usual = false;
    if (all) {
      top = load_counting(near);
      usual = top <= kUsualBase;
      if (usual) {
        m = top < 0x7f ? -INFINITY : value_at(top);   // (below -inf's pattern: NaN)
      } else {
        float hi = -INFINITY;
        for (int v = tid; v < nvec; v += kThreads) {
          const u32x4 x = vec(v);
#pragma unroll
          for (int e = 0; e < kPer; ++e) hi = fmaxf(hi, entry(x, e));
        }
        m = row_max(hi);
      }
    } else {
      m = load(mine);
    }
    if (!(T > 0.f) || k == 1 || (by_p && !(top_p > 0.f)) || m == -INFINITY) {
      // the first maximum; of a row without mass only greedily, and of one of
      // NaN none
      int at = INT_MAX;
      if (!(T > 0.f) || m > -INFINITY)
        each([&](float x) { return x == m; }, [&](float, int index) { at = min(at, index); });
      if (at < INT_MAX) atomicMin(&sh.found_index, at);
      __syncthreads();
      token = sh.found_index < INT_MAX ? sh.found_index : -1;
      logp = token < 0 ? -INFINITY : 0.f;
      return;
    }
    if (m == INFINITY) {
      // infinite logits share the mass
      draw_infinite(u, by_k ? k : p.V, by_p, top_p, token, logp);
      return;
    }
    md = uniform((double)m);
    c = uniform(1.4426950408889634074 / (double)T);
    cut = uniform(min_p > 0.f ? (double)fminf(min_p, 1.f) * (double)(1ull << kUnit) : 0.0);
    if (usual) usual = least_weighed(T) >= (double)value_at(kUsualBase - kUsualReach);
    if (usual) {
      base = kUsualBase;
      reach = kUsualReach;
      mid = kUsualMid;
      skip = kUsualSkip;
      weigh_near(near);
    } else {
      lay_bins(T);
      if (best && draw_best(u, k, by_p, top_p, mine, token, logp)) return;
      if (all || best) {
        __syncthreads();
        clear_hist();
        __syncthreads();
      }
      fill(by_k);
    }
    __syncthreads();
    if constexpr (BF16) {
      // -0 counts as 0
      const int zero = bin_of(kZero);
      if (kZero <= top && kZero > base - reach && !in_middle(zero)) {
        if (tid == 0) {
          sh.hist.count[zero] += sh.hist.count[zero + 1];
          sh.hist.count[zero + 1] = 0;
        }
        __syncthreads();
      }
    }

    // this thread's bins: counts and masses
    int count[kOwn], n_own = 0;
    u64 mass[kOwn], w_own = 0, own_above = 0;
    const bool is_mid = in_middle(tid * kOwn);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      count[i] = sh.hist.count[tid * kOwn + i];
      if constexpr (!BF16) mass[i] = sh.hist.mass[tid * kOwn + i];
    }
    if constexpr (BF16) {
      // A group's values lie at one distance: the first weight (the maximum's,
      // where it is among them) and a ratio give all, by the same products
      // whatever a thread's part of the group is (a weight of its own for each
      // bin: 2048 rows 57.5 -> 62.6 us).
      const int K0 = pattern_of(tid * kOwn), from = is_mid ? 0 : K0 - min(K0, top);
      const int first = min(K0 | (kGroup - 1), top), last = K0 & ~(kGroup - 1), steps = first - min(K0, top);
      double w, ratio, exact[kOwn];
      weight(value_at(first), w);
      ratio = power(((double)value_at(last + 1) - (double)value_at(last)) * c, 0);
#pragma unroll
      for (int n = 0; n < kGroup - kOwn; ++n) w = n < steps ? w * ratio : w;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        exact[i] = w;
        w = i >= from ? w * ratio : w;
      }
      if (best) {   // (rarely: draw_best's weights, as the number of threads decides which rows end there)
#pragma unroll
        for (int i = 0; i < kOwn; ++i) weight(value_at(K0 - i), exact[i]);
      }
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const bool there = i >= from;   // (above the maximum there are only NaN)
        mass[i] = there ? whole(exact[i]) * (u64)count[i] : 0;
        count[i] = there ? count[i] : 0;
        if (count[i] && exact[i] >= cut) own_above = w_own + mass[i];
        w_own += mass[i];
      }
      if (is_mid) {
        w_own = sh.middle;
        own_above = sh.middle_above;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kOwn; ++i) w_own += mass[i];
    }
#pragma unroll
    for (int i = 0; i < kOwn; ++i) n_own += count[i];
    if (is_mid) {   // one bin
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        mass[i] = i == 0 ? w_own : 0;
        count[i] = i == 0 ? n_own : 0;
      }
    }
    int n_before, n_all;
    u64 w_before, kept;
    scan(n_own, w_own, n_before, w_before, n_all, kept);
    kept = uniform(kept);
    if (BF16 && cut > 0.0) {
      if (own_above) atomicMax(&sh.above, w_before + own_above);
      __syncthreads();
    }
    const u64 above = uniform(cut > 0.0 ? sh.above : kept);

    // the ends of what top_k and top_p keep, then the token
#pragma unroll 1
    for (int stage = 0; stage < 3; ++stage) {
      u64 position;
      if (stage == 0) {
        if (!by_k || k >= n_all) continue;
        position = (u64)(k - 1);
      } else if (stage == 1) {
        if (!by_p) continue;
        position = share_end(top_p, kept);
      } else {
        kept = min(kept, above);
        position = share_of(u, kept);
      }
      const bool by_count = stage == 0;
      const u64 own_from = by_count ? (u64)n_before : w_before, own_size = by_count ? (u64)n_own : w_own;
      if (position >= own_from && position - own_from < own_size) {   // (one thread)
        int nb = n_before, at = 0;
        u64 wb = w_before;
        bool past = true;
#pragma unroll
        for (int i = 0; i < kOwn - 1; ++i) {
          past = past && position >= (by_count ? (u64)(nb + count[i]) : wb + mass[i]);
          if (past) {
            nb += count[i];
            wb += mass[i];
            at = i + 1;
          }
        }
        sh.bin = tid * kOwn + at;
        sh.before = wb;
        sh.count_before = nb;
        if constexpr (BF16) {
          // the place in a bin of equal weights (a quotient below 2^20 is off
          // by at most one in fp64)
          int n = count[0];
#pragma unroll
          for (int i = 1; i < kOwn; ++i) n = at == i ? count[i] : n;
          u64 m_at = mass[0];
#pragma unroll
          for (int i = 1; i < kOwn; ++i) m_at = at == i ? mass[i] : m_at;
          const u64 w = (u64)rint((double)m_at / (double)max(n, 1));   // (exact: n equal weights below 2^43)
          u64 nth = by_count ? position - (u64)nb : 0;
          if (!by_count && w) {
            const u64 left = position - wb;
            nth = (u64)((double)left / (double)w);
            if (nth * w > left) --nth;
            else if ((nth + 1) * w <= left) ++nth;
          }
          sh.n = n;
          sh.found_index = (int)nth;
          sh.found_mass = wb + (nth + 1) * w;
        }
      }
      __syncthreads();
      const int bin = uniform(sh.bin);
      if (!BF16 || in_middle(bin)) {
        uint32_t lo, hi;
        keys_of(bin, lo, hi);
        const u64 before = uniform(sh.before);
        search_keys(lo, min(hi, key_of(m)), by_count, position - (by_count ? (u64)uniform(sh.count_before) : before), before);
      } else if (stage == 2) {
        const float value = value_at(pattern_of(bin));
        const int n = uniform(sh.n), nth = uniform(sh.found_index);
        __syncthreads();
        if (tid == 0) sh.found_logit = value;
        if (n <= kList) {
          if (tid == 0) sh.n_list = 0;
          __syncthreads();
          list_equal(value, n);
          __syncthreads();
          if (tid < n) {
            const int own = sh.indices[tid];
            int rank = 0;
            for (int f = 0; f < n; ++f) rank += sh.indices[f] < own;
            if (rank == nth) sh.found_index = own;
          }
        } else {
          find_nth(value, nth);
        }
      }
      __syncthreads();
      if (stage < 2) {
        kept = uniform(sh.found_mass);
        __syncthreads();   // (read before the next stage's is written)
      }
    }
    token = sh.found_index;
    if (wave == 0) logp = log_share(sh.found_logit, kept);
  }
};

// The acceptance of sequence b from its sampled tokens, by one wave.
__device__ __forceinline__ void accept(const Params& p, int b, int c, int lane) {
  const int32_t* tokens = p.tokens + (size_t)b * p.C_max;
  int32_t* sampled = p.sampled + (size_t)b * p.C_max;
  auto drawn = [&](int k) {   // (written by other workgroups)
    return k < c ? __hip_atomic_load(sampled + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : -1;
  };
  int a = -1, last = 0;   // accepted drafts, the last accepted position
  uint64_t path = 0;
  if (p.draft_mask) {
    // (c <= 64) node k's parent is its highest ancestor; a node is accepted
    // when no edge on its root path is wrong
    const int s = drawn(lane);
    const uint64_t word =
        lane < c ? p.draft_mask[(size_t)b * p.C_max + lane] & (c >= 64 ? ~0ull : (1ull << c) - 1) : 0;
    const uint64_t above = word & ((1ull << lane) - 1);
    const int parent = above ? 63 - __builtin_clzll(above) : -1;
    const int at_parent = __shfl(s, parent & 63);
    const bool wrong = lane >= 1 && lane < c && (parent < 0 || tokens[lane] != at_parent);
    const uint64_t wrongs = __ballot(wrong);
    const bool ok = lane < c && (word & wrongs) == 0;
    int best = ok ? (__popcll(word) - 1) << 8 | (255 - lane) : -1;
    best = wave_max(best);
    last = 255 - (best & 255);
    a = best >> 8;
    path = __shfl(word, last & 63);
  } else {
    for (int k0 = 0; k0 < c && a < 0; k0 += 64) {
      const int k = k0 + lane;
      const uint64_t wrong = __ballot(k >= c - 1 || tokens[k + 1] != drawn(k));   // draft k + 1, or none left
      if (wrong) a = k0 + __builtin_ctzll(wrong);
    }
    last = a;
  }
  if (lane == 0) {
    p.accepted[b] = a;
    p.next_token[b] = drawn(last);
    p.new_ctx[b] = p.ctx_lens[b] + a + 1;
    if (p.path) p.path[b] = path;
    __hip_atomic_store(p.counters + b, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // ready for the next call
  }
}

// One workgroup per row.  (As many as fit the chip, each with every 512th row:
// 2048 rows of 32000 took 107 us, not 94.)
template <bool BF16, int kRowLds, int kThreads, bool ACCEPT>
__global__ __launch_bounds__(kThreads, 4) void sample_kernel(Params p) {
  using R = Row<BF16, kRowLds, kThreads>;
  static_assert(sizeof(typename R::Shared) <= (kThreads == 512 ? kLds / 2 : kLds), "LDS of a CU");
  __shared__ typename R::Shared sh;
  // MODE.IEEE off: a maximum with one NaN operand, signalling or quiet, is the
  // other operand
  __builtin_amdgcn_s_setreg(kModeIeee, 0);
  const int n = blockIdx.x;
  const int b = ACCEPT ? n / p.C_max : n, i = ACCEPT ? n - b * p.C_max : 0;
  int c = 1;
  if constexpr (ACCEPT) {
    c = min(max(p.chunk_lens[b], 0), p.C_max);
    if (i >= c) {
      if (threadIdx.x == 0) {
        p.sampled[n] = -1;
        if (p.logprobs) p.logprobs[n] = 0.f;
        if (i == 0) {   // an empty chunk: no step
          p.accepted[b] = 0;
          p.next_token[b] = -1;
          p.new_ctx[b] = p.ctx_lens[b];
          if (p.path) p.path[b] = 0;
        }
      }
      return;
    }
  }
  const float u = p.uniforms[n];
  const float T = p.temperature ? p.temperature[b] : 1.f;
  const int k = p.top_k ? p.top_k[b] : 0;
  const float top_p = p.top_p ? p.top_p[b] : 1.f, min_p = p.min_p ? p.min_p[b] : 0.f;
  int token;
  float logp = 0.f;
  R row(p, sh, p.logits + (size_t)n * p.stride);
  row.draw(u, T, k, top_p, min_p, token, logp);
  if constexpr (!ACCEPT) {
    if (threadIdx.x == 0) {
      p.sampled[n] = token;
      if (p.logprobs) p.logprobs[n] = logp;
    }
  } else if (threadIdx.x < 64) {
    // the last row of the sequence to finish decides the acceptance
    int old = 0;
    if (threadIdx.x == 0) {
      if (p.logprobs) p.logprobs[n] = logp;
      __hip_atomic_store(p.sampled + n, token, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      old = __hip_atomic_fetch_add(p.counters + b, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (uniform(old) == c - 1) accept(p, b, c, threadIdx.x);
  }
}

// ---------------------------------------------------------------- host side

template <bool BF16, bool ACCEPT>
void launch_rows(const Params& p, unsigned rows, hipStream_t s) {
  constexpr int kSmall = BF16 ? kRowSmall : kRowSmallF32;
  const int64_t bytes = ((int64_t)p.V * (BF16 ? 2 : 4) + 15) / 16 * 16;
  // 16 waves to a row where it has a CU to itself: few rows, or long ones (16
  // rows of 32000 bf16 17.9 -> 15.5 us, 256 of fp32 33.0 -> 30.1, 64 of 151936
  // bf16 66 -> 46); where two rows share one, 8 waves each, with the registers
  // that a row's work takes (2048 rows, everything kept: 80.4 us with 8 waves,
  // 80.3 with 16 of 64 registers, which spill, 106 with 4; with top-p 0.9
  // 79.0, 82.2 and 107; before rows were counted as they are loaded).
  if (bytes <= kSmall && rows > kCUs)
    hipLaunchKernelGGL((sample_kernel<BF16, kSmall, 512, ACCEPT>), dim3(rows), dim3(512), 0, s, p);
  else if (bytes <= kSmall)
    hipLaunchKernelGGL((sample_kernel<BF16, kSmall, 1024, ACCEPT>), dim3(rows), dim3(1024), 0, s, p);
  else if (bytes <= kRowLarge)
    hipLaunchKernelGGL((sample_kernel<BF16, kRowLarge, 1024, ACCEPT>), dim3(rows), dim3(1024), 0, s, p);
  else
    hipLaunchKernelGGL((sample_kernel<BF16, 0, 1024, ACCEPT>), dim3(rows), dim3(1024), 0, s, p);
}

template <bool ACCEPT>
int launch(int dtype, const Params& p, unsigned rows, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (dtype == SPECMOE_BF16) launch_rows<true, ACCEPT>(p, rows, s);
  else launch_rows<false, ACCEPT>(p, rows, s);
  return hipGetLastError() == hipSuccess ? SPECMOE_OK : SPECMOE_ERR_LAUNCH;
}

bool aligned(const void* ptr, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(ptr) & (bytes - 1)) == 0; }

void use_settings(Params& p, const specmoe_sampling* s) {
  if (!s) return;
  p.temperature = s->temperature;
  p.top_k = s->top_k;
  p.top_p = s->top_p;
  p.min_p = s->min_p;
}

int accept_sample(const void* logits, const int32_t* tokens, const uint64_t* draft_mask, const int32_t* ctx_lens,
                  const int32_t* chunk_lens, const float* uniforms, const specmoe_sampling* sampling,
                  int32_t* sampled, float* logprobs, int32_t* accepted, int32_t* next_token, int32_t* new_ctx_lens,
                  uint64_t* path, void* stream, const specmoe_accept_desc* desc) {
  const int st = validate(desc);
  if (st != SPECMOE_OK) return st;
  if (desc->V > kMaxVocab || (int64_t)desc->B * desc->C_max >= kMaxRows) return SPECMOE_ERR_SHAPE;
  if (desc->B == 0) return SPECMOE_OK;
  if (!logits || !tokens || !ctx_lens || !chunk_lens || !uniforms || !sampled || !accepted || !next_token ||
      !new_ctx_lens)
    return SPECMOE_ERR_NULL_POINTER;
  if (!aligned(logits, 16)) return SPECMOE_ERR_ALIGN;
  if (!desc->workspace) return SPECMOE_ERR_NULL_POINTER;
  if (!aligned(desc->workspace, 16)) return SPECMOE_ERR_ALIGN;
  if (desc->workspace_bytes < make_plan(desc).bytes) return SPECMOE_ERR_WORKSPACE;
  Params p = {};
  p.logits = static_cast<const char*>(logits);
  p.uniforms = uniforms;
  use_settings(p, sampling);
  p.sampled = sampled;
  p.logprobs = logprobs;
  p.stride = (int64_t)desc->V * elt_of(desc);
  p.V = desc->V;
  p.C_max = desc->C_max;
  p.chunk_lens = chunk_lens;
  p.ctx_lens = ctx_lens;
  p.tokens = tokens;
  p.draft_mask = draft_mask;
  p.accepted = accepted;
  p.next_token = next_token;
  p.new_ctx = new_ctx_lens;
  p.path = path;
  p.counters = static_cast<int*>(desc->workspace);
  return launch<true>(desc->dtype, p, (unsigned)(desc->B * desc->C_max), stream);
}

}  // namespace

extern "C" {

int specmoe_sample(const void* logits, const float* uniforms, const specmoe_sampling* sampling, int32_t* tokens,
                   float* logprobs, void* stream, const specmoe_sample_desc* desc) {
  if (!desc) return SPECMOE_ERR_NULL_POINTER;
  if (desc->dtype != SPECMOE_F32 && desc->dtype != SPECMOE_BF16) return SPECMOE_ERR_DTYPE;
  if (desc->flags != 0) return SPECMOE_ERR_FLAGS;
  if (desc->N < 0 || desc->N > kMaxRows - 1 || desc->V < 1 || desc->V > kMaxVocab) return SPECMOE_ERR_SHAPE;
  if (desc->stride != 0 && (desc->stride < desc->V || desc->stride >= ((int64_t)1 << 36))) return SPECMOE_ERR_SHAPE;
  if (desc->N == 0) return SPECMOE_OK;
  if (!logits || !uniforms || !tokens) return SPECMOE_ERR_NULL_POINTER;
  const int elt = desc->dtype == SPECMOE_BF16 ? 2 : 4;
  if (!aligned(logits, elt)) return SPECMOE_ERR_ALIGN;
  Params p = {};
  p.logits = static_cast<const char*>(logits);
  p.uniforms = uniforms;
  use_settings(p, sampling);
  p.sampled = tokens;
  p.logprobs = logprobs;
  p.stride = (desc->stride ? desc->stride : desc->V) * elt;
  p.V = desc->V;
  p.C_max = 1;
  return launch<false>(desc->dtype, p, (unsigned)desc->N, stream);
}

int specmoe_accept_sample(const void* logits, const int32_t* tokens, const int32_t* ctx_lens,
                          const int32_t* chunk_lens, const float* uniforms, const specmoe_sampling* sampling,
                          int32_t* sampled, float* logprobs, int32_t* accepted, int32_t* next_token,
                          int32_t* new_ctx_lens, void* stream, const specmoe_accept_desc* desc) {
  return accept_sample(logits, tokens, nullptr, ctx_lens, chunk_lens, uniforms, sampling, sampled, logprobs, accepted,
                       next_token, new_ctx_lens, nullptr, stream, desc);
}

int specmoe_accept_sample_tree(const void* logits, const int32_t* tokens, const uint64_t* draft_mask,
                               const int32_t* ctx_lens, const int32_t* chunk_lens, const float* uniforms,
                               const specmoe_sampling* sampling, int32_t* sampled, float* logprobs,
                               int32_t* accepted, int32_t* next_token, int32_t* new_ctx_lens, uint64_t* path,
                               void* stream, const specmoe_accept_desc* desc) {
  if (desc && validate(desc) == SPECMOE_OK && desc->C_max > 64) return SPECMOE_ERR_MASK;
  if (desc && desc->B > 0 && (!draft_mask || !path)) return SPECMOE_ERR_NULL_POINTER;
  if (!aligned(draft_mask, 8) || !aligned(path, 8)) return SPECMOE_ERR_ALIGN;
  return accept_sample(logits, tokens, draft_mask, ctx_lens, chunk_lens, uniforms, sampling, sampled, logprobs,
                       accepted, next_token, new_ctx_lens, path, stream, desc);
}

}  // extern "C"
