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
//   * one pass adds every token's weight to a histogram over the distance from
//     the maximum, whose prefix sums name the bin of a position; the bin's
//     tokens are then listed and put in order by comparing all with all;
//   * with a small top_k only the best tokens matter: a histogram of the
//     threads' maxima gives a bin edge that at least k tokens pass, and those
//     alone are listed and weighed.
// One workgroup of 16 waves per row holds the row in LDS when it fits (two
// rows of up to 62.5 KB per CU), so the logits are read from HBM once.
#include <hip/hip_runtime.h>

#include <limits.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "accept_plan.h"
#include "specmoe_sample.h"

namespace {

typedef unsigned long long u64;

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = kThreads;            // one histogram bin per thread
constexpr int kList = 256;                 // tokens put in order at once
constexpr int kMaxVocab = 1 << 20;         // weights of 2^42 add up below 2^63
constexpr int kMaxRows = 1 << 22;          // (a launch holds less than 2^32 threads)
constexpr int kUnit = 42;                  // weights are in units of 2^-42
constexpr double kMost = 43.0;             // from 2^-43 on a weight is less than half a unit
constexpr int kModeIeee = 1 | (9 << 6);    // s_setreg operand: bit 9 of the MODE register

// Rows of up to kRowSmall bytes leave room for two workgroups on a CU, rows up
// to kRowLarge for one; longer ones are read again from the caches.
constexpr int kRowSmall = 64000, kRowLarge = 147456;

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

// What a search in the order finds: the token, its logit, and the mass up to it
// and with it.
struct Found {
  int index;
  float logit;
  u64 mass;
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// bits that sort as the values do (no NaN); -0 counts as 0
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

template <class T, class OP>
__device__ __forceinline__ T wave_all(T x, OP op) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) x = op(x, __shfl_xor(x, m));
  return x;
}
__device__ __forceinline__ int wave_prefix(int x, int lane) {   // inclusive
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int y = __shfl_up(x, m);
    if (lane >= m) x += y;
  }
  return x;
}
__device__ __forceinline__ u64 wave_prefix(u64 x, int lane) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const u64 y = __shfl_up(x, m);
    if (lane >= m) x += y;
  }
  return x;
}

// 2^f for |f| <= 1/2: the polynomial of degree 9 through 2^f at the Chebyshev
// nodes of the interval, off by less than 2^-45.6.
__device__ __forceinline__ double exp2_poly(double f) {
  double q = 1.020590550210069e-07;
  q = fma(q, f, 1.3259645241948732e-06);
  q = fma(q, f, 1.5252672924257465e-05);
  q = fma(q, f, 0.0001540343375126647);
  q = fma(q, f, 0.0013333558200796013);
  q = fma(q, f, 0.00961812919393429);
  q = fma(q, f, 0.05550410866465166);
  q = fma(q, f, 0.2402265069564034);
  q = fma(q, f, 0.6931471805599462);
  return fma(q, f, 1.0);
}

// One row's sampling, by all threads of a workgroup.
template <bool BF16, int kRowLds>
struct Row {
  static constexpr int kElt = BF16 ? 2 : 4;
  static constexpr int kPer = 16 / kElt;   // logits per 16-byte vector

  struct Shared {
    __attribute__((aligned(16))) char row[kRowLds ? kRowLds : 16];
    union {
      struct {
        u64 mass[kBins];
        int count[kBins];
      } hist;
      Entry list[kList];
    };
    u64 part_mass[kWaves];
    int part_count[kWaves];
    float part_max[kWaves], part_min[kWaves];
    u64 found_mass, bin_before;
    float found_logit;
    int found_index, bin, bin_count_before, n_list;
    uint32_t key_lo, key_hi;
  };

  const Params& p;
  Shared& sh;
  const char* src;   // the row in memory
  int tid, lane, wave, nvec;
  float m, bin_scale;
  double md, c;      // the maximum, log2(e) / T
  double cut;        // min_p in weight units (0: off)

  __device__ __forceinline__ Row(const Params& p_, Shared& sh_, const char* src_)
      : p(p_), sh(sh_), src(src_), tid(threadIdx.x), lane(threadIdx.x & 63), wave(uniform(threadIdx.x >> 6)),
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

  // every token: f(x, index); whole waves go through together
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    for (int v = tid; v < nvec; v += kThreads) {
      const u32x4 x = vec(v);
#pragma unroll
      for (int e = 0; e < kPer; ++e) f(entry(x, e), v * kPer + e);
    }
  }

  // weight in units, and the same before it was rounded
  __device__ __forceinline__ u64 weight(float x, double& exact) const {
    const double y = x == m ? 0.0 : (md - (double)x) * c;
    if (!(y < kMost)) {   // (also NaN)
      exact = 0.0;
      return 0;
    }
    const double n = rint(y);
    exact = ldexp(exp2_poly(n - y), kUnit - (int)n);
    // round to an integer in the low bits of a double of 2^52 and more
    return (u64)__double_as_longlong(exact + 4503599627370496.0) & 0xfffffffffffffull;
  }
  // (the mask changes no bin: it keeps the index in range whatever x is)
  __device__ __forceinline__ int bin_of(float x) const {
    return (int)fminf((m - x) * bin_scale, (float)(kBins - 1)) & (kBins - 1);
  }

  // loads the row, and its maximum and least finite logit.  The maximum is
  // -inf for a row without any mass.
  __device__ __forceinline__ float load(float& least, float& mine) {
    float hi = -INFINITY, lo = INFINITY;
    auto take = [&](const u32x4& x) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const float y = entry(x, e);
        hi = fmaxf(hi, y);
        lo = y > -INFINITY ? fminf(lo, y) : lo;
      }
    };
    constexpr int kBatch = 4;   // 16-byte loads per lane in flight
    for (int v0 = tid; v0 < nvec; v0 += kBatch * kThreads) {
      u32x4 x[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (v0 + u * kThreads < nvec) x[u] = fetch(v0 + u * kThreads);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (v0 + u * kThreads >= nvec) continue;
        if constexpr (kRowLds > 0) *reinterpret_cast<u32x4*>(sh.row + (size_t)(v0 + u * kThreads) * 16) = x[u];
        take(x[u]);
      }
    }
    mine = hi;
    hi = wave_all(hi, [](float a, float b) { return fmaxf(a, b); });
    lo = wave_all(lo, [](float a, float b) { return fminf(a, b); });
    if (lane == 0) {
      sh.part_max[wave] = hi;
      sh.part_min[wave] = lo;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      hi = fmaxf(hi, sh.part_max[w]);
      lo = fminf(lo, sh.part_min[w]);
    }
    least = lo;
    return hi;
  }

  // sums over the workgroup of what the threads before hold, and the total
  __device__ __forceinline__ void scan(int n, u64 w, int& n_before, u64& w_before, int& n_all, u64& w_all) {
    const int ni = wave_prefix(n, lane);
    const u64 wi = wave_prefix(w, lane);
    __syncthreads();   // (the last scan's totals have been read)
    if (lane == 63) {
      sh.part_count[wave] = ni;
      sh.part_mass[wave] = wi;
    }
    __syncthreads();
    n_before = ni - n;
    w_before = wi - w;
    n_all = 0;
    w_all = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      if (k < wave) {
        n_before += sh.part_count[k];
        w_before += sh.part_mass[k];
      }
      n_all += sh.part_count[k];
      w_all += sh.part_mass[k];
    }
  }

  __device__ __forceinline__ void clear_hist() {
    __syncthreads();
    sh.hist.mass[tid] = 0;
    sh.hist.count[tid] = 0;
    __syncthreads();
  }

  // Lists the tokens for which want(x) holds and that weigh anything; returns
  // how many there are, of which the first kList are listed.
  template <class WANT>
  __device__ __forceinline__ int gather(WANT want) {
    __syncthreads();
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    each([&](float x, int index) {
      if (want(x)) {
        double exact;
        const u64 w = weight(x, exact);
        if (w) {
          const int at = atomicAdd(&sh.n_list, 1);
          if (at < kList) sh.list[at] = Entry{(u64)key_of(x) << 32 | (uint32_t)~index, w};
        }
      }
    });
    __syncthreads();
    return sh.n_list;
  }

  // The place of list entry tid / G among the n listed: the entries and the
  // mass before it.  G threads share an entry's comparisons.
  __device__ __forceinline__ int groups(int n) const {
    int g = kThreads / kList;   // (n <= kList)
    while (g < 64 && n * g * 2 <= kThreads) g *= 2;
    return g;
  }
  __device__ __forceinline__ void place(int n, int g, int& rank, u64& before) const {
    const int e = tid / g;
    rank = 0;
    before = 0;
    if (e < n) {
      const u64 own = sh.list[e].order;
      for (int f = tid % g; f < n; f += g) {
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

  __device__ __forceinline__ Found found() {
    __syncthreads();
    return Found{sh.found_index, sh.found_logit, sh.found_mass};
  }

  // The token at a position of the order: of a count (by_count) or of a mass.
  // Thread t holds what comes before bin t (n0, w0) and in it (n1, w1); the
  // position lies before the end of the last bin.
  __device__ __forceinline__ Found search(bool by_count, u64 position, int n0, u64 w0, int n1, u64 w1) {
    const u64 lo = by_count ? (u64)n0 : w0, size = by_count ? (u64)n1 : w1;
    if (position >= lo && position - lo < size) {
      sh.bin = tid;
      sh.bin_before = w0;
      sh.bin_count_before = n0;
    }
    __syncthreads();
    const int bin = sh.bin;
    u64 before = sh.bin_before;
    u64 left = position - (by_count ? (u64)sh.bin_count_before : before);   // position in the bin
    const int n = gather([&](float x) { return bin_of(x) == bin; });
    if (n <= kList) {
      const int g = groups(n);
      int rank;
      u64 inside;
      place(n, g, rank, inside);
      const int e = tid / g;
      if (e < n && tid % g == 0) {
        const Entry own = sh.list[e];
        const u64 at = by_count ? (u64)rank : inside;
        if (left >= at && left - at < (by_count ? 1 : own.weight)) {
          sh.found_index = (int)~(uint32_t)own.order;
          sh.found_logit = value_of((uint32_t)(own.order >> 32));
          sh.found_mass = before + inside + own.weight;
        }
      }
      return found();
    }
    // Many tokens in one bin (nearly equal logits): the bin's range of keys is
    // cut into bins of its own until one holds a single key, whose tokens are
    // counted by index.
    uint32_t lo_key = 0xffffffffu, hi_key = 0u;
    each([&](float x, int) {
      double exact;
      if (bin_of(x) == bin && weight(x, exact)) {
        lo_key = min(lo_key, key_of(x));
        hi_key = max(hi_key, key_of(x));
      }
    });
    __syncthreads();
    if (tid == 0) {
      sh.key_lo = 0xffffffffu;
      sh.key_hi = 0u;
    }
    __syncthreads();
    atomicMin(&sh.key_lo, lo_key);
    atomicMax(&sh.key_hi, hi_key);
    __syncthreads();
    lo_key = sh.key_lo;
    hi_key = sh.key_hi;
    for (int level = 0; level < 4 && lo_key != hi_key; ++level) {   // (ten bits of the key each)
      const uint32_t span = hi_key - lo_key;
      const int shift = max(0, 32 - __builtin_clz(span) - 10);   // span >> shift < kBins
      clear_hist();
      each([&](float x, int) {
        const uint32_t k = key_of(x);
        if (x == x && k >= lo_key && k <= hi_key) {
          double exact;
          atomicAdd(&sh.hist.mass[(hi_key - k) >> shift], weight(x, exact));
          atomicAdd(&sh.hist.count[(hi_key - k) >> shift], 1);
        }
      });
      __syncthreads();
      const int n_in = sh.hist.count[tid];
      const u64 w_in = sh.hist.mass[tid];
      int nb, na;
      u64 wb, wa;
      scan(n_in, w_in, nb, wb, na, wa);
      const u64 b0 = by_count ? (u64)nb : wb, bs = by_count ? (u64)n_in : w_in;
      if (left >= b0 && left - b0 < bs) {
        sh.bin = tid;
        sh.bin_before = wb;
        sh.bin_count_before = nb;
      }
      __syncthreads();
      before += sh.bin_before;
      left -= by_count ? (u64)sh.bin_count_before : sh.bin_before;
      hi_key -= (uint32_t)sh.bin << shift;
      lo_key = max(lo_key, hi_key - ((1u << shift) - 1u));
      __syncthreads();   // (sh.bin has been read)
    }
    // one key: its tokens weigh the same; the one of place `nth` by index
    const float value = value_of(lo_key);
    double exact;
    const u64 w = weight(value, exact);
    const int nth = (int)(by_count ? left : left / w);
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
        sh.found_logit = value;
        sh.found_mass = before + (u64)(nth + 1) * w;
      }
      seen += na;
    }
    return found();
  }

  // the smallest position at or beyond a share of a mass, less one
  static __device__ __forceinline__ u64 share_end(float share, u64 mass) {
    const double want = ceil((double)share * (double)mass);
    const u64 w = want >= 1.0 ? (u64)want : 1;
    return min(w, mass) - 1;
  }
  static __device__ __forceinline__ u64 share_of(float u, u64 mass) {
    const double at = u > 0.f ? (double)u * (double)mass : 0.0;   // (NaN: 0)
    return at < (double)mass ? min((u64)at, mass - 1) : mass - 1;
  }

  // log of a token's share of the kept mass
  __device__ __forceinline__ float log_share(float x, u64 kept) const {
    const double d = x == m ? 0.0 : ((double)x - md) * (c * 0.69314718055994530942);
    return (float)(d - log((double)kept * (1.0 / (double)(1ull << kUnit))));
  }

  // The row's token and log-probability, in every thread.
  __device__ __forceinline__ void draw(float u, float T, int k, float top_p, float min_p, int& token, float& logp) {
    float least, mine;
    m = load(least, mine);
    const bool by_k = k > 0 && k < p.V, by_p = top_p < 1.f;   // (NaN: off)
    if (!(T > 0.f) || k == 1 || (by_p && !(top_p > 0.f)) || m == -INFINITY) {
      // the first maximum; of a row without mass only greedily, and of one of
      // NaN none
      const bool greedy = !(T > 0.f);
      if (tid == 0) sh.found_index = INT_MAX;
      __syncthreads();
      int at = INT_MAX;
      if (greedy || m > -INFINITY)
        each([&](float x, int index) {
          if (x == m) at = min(at, index);
        });
      if (at < INT_MAX) atomicMin(&sh.found_index, at);
      __syncthreads();
      token = sh.found_index < p.V ? sh.found_index : -1;   // (past the end: a vector's tail)
      logp = token < 0 ? -INFINITY : 0.f;
      return;
    }
    md = (double)m;
    c = 1.4426950408889634074 / (double)T;
    cut = min_p > 0.f ? (double)min_p * (double)(1ull << kUnit) : 0.0;
    if (min_p >= 1.f) cut = (double)(1ull << kUnit);
    const float range = fminf((float)(kMost / c), m - least);
    bin_scale = fminf((float)kBins / range, 3e38f);

    if (by_k && k <= kList) {
      // the bin edge that at least k threads' maxima pass
      clear_hist();
      if (mine > -INFINITY) atomicAdd(&sh.hist.count[bin_of(mine)], 1);
      __syncthreads();
      int nb, na;
      u64 wb, wa;
      const int n_in = sh.hist.count[tid];
      scan(n_in, 0, nb, wb, na, wa);
      if (tid == 0 && na < k) sh.bin = kBins - 1;
      if (nb < k && k <= nb + n_in) sh.bin = tid;
      __syncthreads();
      const int edge = sh.bin;
      const int n = gather([&](float x) { return bin_of(x) <= edge; });
      if (n <= kList) {
        const int g = groups(n);
        int rank;
        u64 before;
        place(n, g, rank, before);
        const int e = tid / g;
        const bool owner = e < n && tid % g == 0;
        Entry own = {0, 0};
        if (owner) own = sh.list[e];
        const float logit = value_of((uint32_t)(own.order >> 32));
        if (owner && rank == min(k, n) - 1) sh.found_mass = before + own.weight;
        // (min_p's mass: among the listed it reaches beyond top_k's or is whole)
        double exact = 0.0;
        if (owner) weight(logit, exact);
        const u64 passes = wave_all(owner && exact >= cut ? own.weight : 0, [](u64 a, u64 b) { return a + b; });
        if (lane == 0) sh.part_mass[wave] = passes;
        __syncthreads();
        u64 kept = sh.found_mass, above = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) above += sh.part_mass[w];
        __syncthreads();
        if (by_p) {
          const u64 position = share_end(top_p, kept);
          if (owner && position >= before && position - before < own.weight) sh.found_mass = before + own.weight;
          __syncthreads();
          kept = sh.found_mass;
        }
        kept = min(kept, above);
        const u64 position = share_of(u, kept);
        if (owner && position >= before && position - before < own.weight) {
          sh.found_index = (int)~(uint32_t)own.order;
          sh.found_logit = logit;
        }
        __syncthreads();
        token = sh.found_index;
        logp = log_share(sh.found_logit, kept);
        return;
      }
    }

    // all tokens' weights over the bins, and the mass that min_p keeps
    clear_hist();
    u64 passes = 0;
    each([&](float x, int) {
      double exact;
      const u64 w = weight(x, exact);
      if (w) {
        const int b = bin_of(x);
        atomicAdd(&sh.hist.mass[b], w);
        if (by_k) atomicAdd(&sh.hist.count[b], 1);
        if (exact >= cut) passes += w;
      }
    });
    __syncthreads();
    const int n1 = sh.hist.count[tid];
    const u64 w1 = sh.hist.mass[tid];
    int n0, n_all;
    u64 w0, kept;
    scan(n1, w1, n0, w0, n_all, kept);
    u64 above = kept;
    if (cut > 0.0) {
      int i0, i1;
      u64 j0;
      scan(0, passes, i0, j0, i1, above);
    }
    if (by_k && k < n_all) {
      const Found f = search(true, (u64)(k - 1), n0, w0, n1, w1);
      kept = f.mass;
    }
    if (by_p) {
      const Found f = search(false, share_end(top_p, kept), n0, w0, n1, w1);
      kept = f.mass;
    }
    kept = min(kept, above);
    const Found f = search(false, share_of(u, kept), n0, w0, n1, w1);
    token = f.index;
    logp = log_share(f.logit, kept);
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
    best = wave_all(best, [](int x, int y) { return max(x, y); });
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

template <bool BF16, int kRowLds, bool ACCEPT>
__global__ __launch_bounds__(kThreads) void sample_kernel(Params p) {
  using R = Row<BF16, kRowLds>;
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
  float logp;
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
  const int64_t bytes = ((int64_t)p.V * (BF16 ? 2 : 4) + 15) / 16 * 16;
  if (bytes <= kRowSmall)
    hipLaunchKernelGGL((sample_kernel<BF16, kRowSmall, ACCEPT>), dim3(rows), dim3(kThreads), 0, s, p);
  else if (bytes <= kRowLarge)
    hipLaunchKernelGGL((sample_kernel<BF16, kRowLarge, ACCEPT>), dim3(rows), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL((sample_kernel<BF16, 0, ACCEPT>), dim3(rows), dim3(kThreads), 0, s, p);
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
