// Verification and decode attention over a 4-bit KV cache (specmoe_kv4.h) for
// MI355X (gfx950, CDNA4).
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

struct Kv4Params : Params {   // (k and v: the codes)
  const char* k_scales;
  const char* v_scales;
  int row_groups;   // waves of a workgroup that have different rows: 1, 2 or 4
};

// bfloat16 parts that a value of the type is the sum of
template <int ELT>
constexpr int kParts = ELT == kBF16 ? 1 : ELT == kF16 ? 2 : 3;

__device__ __forceinline__ int tiles_of(uint32_t s) { return sched::seq_tiles(s, kTile); }

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

template <int ELT, int D, bool PAGED, int NRB>
__global__ __launch_bounds__(kGroupThreads, 2) void kv4_attn_kernel(Kv4Params p) {
  constexpr int kElt = ELT == kF32 ? 4 : 2;
  constexpr int NP = kParts<ELT>;
  constexpr int KW = D / 32;          // code words of a lane: its D / 4 entries of a row
  constexpr int DB = D / 16;          // 16-wide d blocks of O^T
  constexpr int kPitch = 2 * D + (D == 128 ? 32 : 16);   // LDS bytes of a staged V row, free of bank conflicts
  constexpr int kStage = kStep * kPitch;
  static_assert(kStage >= kBlk * D * 4, "a row block's O fits a wave's stage");
  __shared__ __attribute__((aligned(16))) char smem[kGroupWaves * kStage];
  __shared__ uint32_t seqs[kMaxSeqs];
  __shared__ int pref[kMaxSeqs];      // tiles of one KV head of the sequences before b
  __shared__ int wsum[kGroupWaves];
  __shared__ float mst[kGroupWaves][NRB][2][kBlk];
  __shared__ int sh_flag;

  const int pid = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int lm = lane & 15, lg = lane >> 4;
  const int B = p.B, Hkv = p.Hkv, g = p.g;
  const int RG = p.row_groups, KS = kGroupWaves / RG;   // row groups, waves that share a row group's keys
  const int rg = wave % RG, kslot = wave / RG;

  // ---- lengths, tile sums, this workgroup's range [g0, g1) of the list of all
  // units' tiles
  const int per = (B + kGroupThreads - 1) / kGroupThreads;
  const int b_lo = min(tid * per, B), b_hi = min(b_lo + per, B);
  int mine = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    const uint32_t s = load_seq(p, b);
    seqs[b] = s;
    mine += tiles_of(s);
  }
  const int incl = wave_scan(mine);
  if (lane == 63) wsum[wave] = incl;
  __syncthreads();
  int before = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kGroupWaves; ++w) {
    before += w < wave ? wsum[w] : 0;
    total += wsum[w];
  }
  for (int b = b_lo; b < b_hi; ++b) {
    pref[b] = before;
    before += tiles_of(seqs[b]);
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

  const int64_t N = (int64_t)uniform(total) * Hkv;   // (< 2^31: host check)
  const int P = (int)min((int64_t)p.P, N);
  if (pid >= P) return;
  const int g0 = (int)(N * pid / P), g1 = (int)(N * (pid + 1) / P);
  // the range that has tile t
  auto owner = [&](int t) { return (int)((((int64_t)t + 1) * P - 1) / N); };

  // the last sequence whose tiles begin at or before g0 (it has some)
  int b = 0;
  for (int step = 512; step; step >>= 1)
    if (b + step < B && (int64_t)pref[b + step] * Hkv <= g0) b += step;
  b = uniform(b);

  char* const stage = smem + wave * kStage;

  for (int t = g0; t < g1;) {
    // ---- segment: tiles [j0, j1) of KV head kvh of sequence b
    uint32_t s = uniform(seqs[b]);
    int n = tiles_of(s);
    int rel = t - uniform(pref[b]) * Hkv;
    while (rel >= n * Hkv) {   // (the next sequence that has tiles)
      ++b;
      s = uniform(seqs[b]);
      n = tiles_of(s);
      rel = t - uniform(pref[b]) * Hkv;
    }
    const int kvh = rel / n;
    const int j0 = rel - kvh * n, j1 = min(n, j0 + (g1 - t));
    const int T = seq_T(s), c = seq_c(s), l_ctx = T - c, R = c * g;
    const int kend = min(T, j1 * kTile);

    // ---- this lane's rows: row block rb of the wave has the unit's rows
    // 16 (NRB rg + rb) + lm
    int tok[NRB];
    bool valid[NRB];
    uint64_t word[NRB];
    u32x4 q[NP][NRB][KW];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      const int row = kBlk * (NRB * rg + rb) + lm;
      valid[rb] = row < R;
      tok[rb] = valid[rb] ? row / g : 0;
      const int h = kvh * g + (valid[rb] ? row - tok[rb] * g : 0);
      word[rb] = valid[rb] && p.draft_mask ? p.draft_mask[b * p.C_max + tok[rb]] : 0;
      const char* src = p.q + ((size_t)(b * p.C_max + tok[rb]) * p.Hq + h) * (D * kElt) + lg * (D / 4) * kElt;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        if constexpr (ELT == kBF16) {
          q[0][rb][w] = valid[rb] ? *reinterpret_cast<const u32x4*>(src + 16 * w) : u32x4{0u, 0u, 0u, 0u};
        } else {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = 0.f;
          if (valid[rb]) {
            if constexpr (ELT == kF32) {
              const f32x4 lo = *reinterpret_cast<const f32x4*>(src + 32 * w), hi = *reinterpret_cast<const f32x4*>(src + 32 * w + 16);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                x[e] = lo[e];
                x[4 + e] = hi[e];
              }
            } else {
              const f16x8 y = *reinterpret_cast<const f16x8*>(src + 16 * w);
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = (float)y[e];
            }
          }
#pragma unroll
          for (int part = 0; part < NP; ++part)
#pragma unroll
            for (int e = 0; e < 4; ++e) q[part][rb][w][e] = split2(x[2 * e], x[2 * e + 1]);
        }
      }
    }

    f32x4 o[NRB][DB];
    float m_run[NRB], l_lane[NRB];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      m_run[rb] = -INFINITY;
      l_lane[rb] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // ---- 32 keys from base on: lane (lm, lg) has the lg-th quarter of the
    // rows of keys base + lm and base + 16 + lm
    struct Keys {
      uint32_t k[2][KW], v[2][KW];
      uint32_t ks[2], vs[2];
    };
    auto load = [&](Keys& x, int base) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int key = base + kBlk * h + lm;
        const bool in = key < kend;
        size_t row;
        if constexpr (PAGED) {
          int page = 0;
          if (in) page = p.block_table[(size_t)b * p.pages_per_seq + (key >> p.page_shift)];
          page = min(max(page, 0), p.num_pages - 1);
          row = (((size_t)page * Hkv + kvh) << p.page_shift) + (key & ((1 << p.page_shift) - 1));
        } else {
          row = ((size_t)b * Hkv + kvh) * p.S_max + key;
        }
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          x.k[h][w] = 0;
          x.v[h][w] = 0;
        }
        x.ks[h] = 0;
        x.vs[h] = 0;
        if (in) {
          const size_t at = row * (D / 2) + lg * (D / 8), sat = row * (D / 32) + (lg * (D / 4) / 32);
          typedef __attribute__((ext_vector_type(KW))) uint32_t words;
          const words kk = *reinterpret_cast<const words*>(p.k + at), vv = *reinterpret_cast<const words*>(p.v + at);
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            x.k[h][w] = kk[w];
            x.v[h][w] = vv[w];
          }
          x.ks[h] = (uint8_t)p.k_scales[sat];
          x.vs[h] = (uint8_t)p.v_scales[sat];
        }
      }
    };

    auto compute = [&](Keys& x, int base) {
      // NaN blocks among the values of keys that not every row sees: 0 times
      // NaN would reach the rows that do not, so such blocks are staged as
      // zeros, and the rows that see them made NaN afterwards.  Bit 16 qd + i
      // of nan[h]: the qd-th quarter of key 16 h + i.
      uint64_t nan[2] = {0, 0};
      uint32_t seen[NRB];   // (keys of the chunk's region) bit e: the lane's row sees its e-th key
      if (base + kStep > l_ctx) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bool bad = x.vs[h] == 255u;
          nan[h] = __ballot(bad);
          if (bad) {
            x.vs[h] = 0;
#pragma unroll
            for (int w = 0; w < KW; ++w) x.v[h][w] = 0;
          }
        }
      }
      // scores of two key blocks: S^T = K Q^T, lane (lm, lg) gets the keys
      // 16 h + 4 lg + r of row lm
      f32x4 sa[NRB][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
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
          for (int part = NP - 1; part >= 0; --part)
#pragma unroll
            for (int w = 0; w < KW; ++w) acc = mfma32<kBF16>(kop[w], q[part][rb][w], acc);
          sa[rb][h] = acc;
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
      u32x4 pb[NRB][NP];
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = sa[rb][e >> 2][e & 3];
        if (base + kStep > l_ctx) {   // (the same for the whole wave)
          seen[rb] = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int k = base + kBlk * (e >> 2) + 4 * lg + (e & 3) - l_ctx;   // draft key
            const bool sees = p.draft_mask ? k < 0 || (k < c && ((word[rb] >> (k & 63)) & 1u))
                                           : k <= tok[rb] && k < c;
            if (sees) seen[rb] |= 1u << e;
            else y[e] = -INFINITY;
          }
        }
        float mx = y[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, y[e]);
        mx = row_max(mx) * p.sl2;
        const bool raise = mx > m_run[rb] + kLazyMax;
        if (__any(raise)) {
          const float m_new = raise ? mx : m_run[rb];
          const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - (m_new == -INFINITY ? 0.f : m_new));
          l_lane[rb] *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[rb][db] *= alpha;
          m_run[rb] = m_new;
        }
        const float m_use = m_run[rb] == -INFINITY ? 0.f : m_run[rb];
        float pr[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          pr[e] = __builtin_amdgcn_exp2f(fmaf(y[e], p.sl2, -m_use));
          l_lane[rb] += pr[e];
        }
        if constexpr (NP == 1) {
          pb[rb][0] = pack_p<kBF16>(pr);
        } else {
#pragma unroll
          for (int part = 0; part < NP; ++part)
#pragma unroll
            for (int e = 0; e < 4; ++e) pb[rb][part][e] = split2(pr[2 * e], pr[2 * e + 1]);
        }
      }
      // O^T += V^T P^T over the 32 keys: element e of a lane's operands is key
      // 4 lg + e of the first block (e < 4) or 4 lg + e - 4 of the second
      typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
      const char* vrow = stage + (4 * lg + (lm >> 2)) * kPitch + 8 * (lm & 3);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const i16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_i16x4*)(__attribute__((address_space(3))) char*)(vrow + 32 * db));
        const i16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_i16x4*)(__attribute__((address_space(3))) char*)(vrow + kBlk * kPitch + 32 * db));
        const u32x4 va = {__builtin_bit_cast(uint2, a0).x, __builtin_bit_cast(uint2, a0).y,
                          __builtin_bit_cast(uint2, a1).x, __builtin_bit_cast(uint2, a1).y};
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
          for (int part = NP - 1; part >= 0; --part) o[rb][db] = mfma32<kBF16>(va, pb[rb][part], o[rb][db]);
      }
      asm volatile("" ::: "memory");
      if (nan[0] | nan[1]) {
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
          const uint32_t own0 = (seen[rb] & 15u) << (4 * lg), own1 = (seen[rb] >> 4) << (4 * lg);
          uint32_t hit = 0;   // bit qd: the row sees a NaN block in the qd-th quarter
#pragma unroll
          for (int qd = 0; qd < 4; ++qd)
            if (((uint32_t)(nan[0] >> (16 * qd)) & own0) | ((uint32_t)(nan[1] >> (16 * qd)) & own1)) hit |= 1u << qd;
          hit |= (uint32_t)__shfl_xor((int)hit, 16);
          hit |= (uint32_t)__shfl_xor((int)hit, 32);
#pragma unroll
          for (int db = 0; db < DB; ++db)
            if ((hit >> (db / (DB / 4))) & 1u) o[rb][db] = f32x4{NAN, NAN, NAN, NAN};
        }
      }
    };

    {
      const int by = kStep * KS;
      int base = j0 * kTile + kStep * kslot;
      Keys x;
      if (base < kend) load(x, base);
      for (; base < kend; base += by) {
        Keys y;
        if (base + by < kend) load(y, base + by);
        compute(x, base);
        x = y;
      }
    }

    // ---- the states of the waves that share the rows joined through LDS: each
    // then has the O of its own d blocks
    const bool whole = j0 == 0 && j1 == n;
    const int slot = 2 * pid + (t - j0 > g0 ? 1 : 0);
    const __amdgpu_buffer_rsrc_t ws_o_rsrc = __builtin_amdgcn_make_buffer_rsrc(p.ws_o, 0, p.ws_o_bytes, kBufferFormat);
    const __amdgpu_buffer_rsrc_t ws_lse_rsrc =
        __builtin_amdgcn_make_buffer_rsrc(p.ws_lse, 0, p.ws_lse_bytes, kBufferFormat);
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
      if (rb) __syncthreads();   // (the last row block's reads)
#pragma unroll
      for (int db = 0; db < DB; ++db) own[db * 64] = o[rb][db];
      __syncthreads();
      float M = -INFINITY, L = 0.f, wk[kGroupWaves];
      for (int k = 0; k < KS; ++k) M = fmaxf(M, mst[k * RG + rg][rb][0][lm]);
      const float Mu = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int k = 0; k < kGroupWaves; ++k) {
        wk[k] = 0.f;
        if (k < KS) {
          wk[k] = __builtin_amdgcn_exp2f(mst[k * RG + rg][rb][0][lm] - Mu);
          L += mst[k * RG + rg][rb][1][lm] * wk[k];
        }
      }
      const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;   // (a NaN stays)
      const float lse = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
      const int row = kBlk * (NRB * rg + rb) + lm;
      const size_t orow = (size_t)(b * p.C_max + tok[rb]) * p.Hq + kvh * g + (row - tok[rb] * g);
      if (valid[rb] && kslot == 0 && lg == 0) {
        if (whole) p.lse[orow] = lse;
        else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(int, lse), ws_lse_rsrc, (slot * p.Rcap + row) * 4, 0,
                                                   kDeviceCoherent);
      }
      for (int db = kslot; db < DB; db += KS) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kGroupWaves; ++k)
          if (k < KS)
            x = add_weighted(x, wk[k], reinterpret_cast<const f32x4*>(smem + (k * RG + rg) * kStage)[db * 64 + lane]);
        x *= inv;
        if (!valid[rb]) continue;
        if (whole)
          store_out<false, ELT>(p, orow * D + 16 * db + 4 * lg, x);
        else
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, x), ws_o_rsrc,
                                                 ((slot * p.Rcap + row) * D + 16 * db + 4 * lg) * 4, 0, kDeviceCoherent);
      }
    }
    if (!whole) {
      // ---- count the piece once all its stores are out; the last to arrive
      // merges the unit's pieces, in their order
      const int first = t - j0, qf = owner(first), ql = owner(first + n - 1);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (tid == 0) {
        int* counter = p.counters + b * Hkv + kvh;
        const int last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == ql - qf;
        if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next call
        sh_flag = last;
      }
      __syncthreads();
      if (sh_flag) {
        const int f_slot = 2 * qf + (first > (int)(N * qf / P) ? 1 : 0);
        for (int idx = tid; idx < R * (D / 4); idx += kGroupThreads) {
          const int row = idx / (D / 4), d = 4 * (idx - row * (D / 4));
          float m = -INFINITY, z = 0.f;
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
          for (int qq = qf; qq <= ql; ++qq) {
            const int at = (qq == qf ? f_slot : 2 * qq) * p.Rcap + row;
            const float lse = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(ws_lse_rsrc, at * 4, 0, kDeviceCoherent));
            const f32x4 x = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(ws_o_rsrc, (at * D + d) * 4, 0,
                                                                                           kDeviceCoherent));
            const float nm = fmaxf(m, lse), nu = nm == -INFINITY ? 0.f : nm;
            const float a = exp_diff(m, nu), w = exp_diff(lse, nu);
            z = z * a + w;
            acc *= a;
            acc = add_weighted(acc, w, x);
            m = nm;
          }
          const size_t orow = (size_t)(b * p.C_max + row / g) * p.Hq + kvh * g + row % g;
          store_out<false, ELT>(p, orow * D + d, acc * (z > 0.f ? 1.f / z : z == 0.f ? 0.f : z));
          if (d == 0) p.lse[orow] = z == 0.f ? -INFINITY : m + logf(z);
        }
      }
    }
    __syncthreads();   // (stages, statistics and the flag are free again)
    t += j1 - j0;
  }
}

// ---------------------------------------------------------------- host side

// desc with the workgroups of these calls
specmoe_verify_desc sized(const specmoe_verify_desc* d) {
  specmoe_verify_desc x = *d;
  if (x.grid_blocks == 0) x.grid_blocks = kGroupsDefault;
  return x;
}

template <int ELT, int D, bool PAGED>
void launch_kv4(const Kv4Params& p, hipStream_t stream) {
  constexpr int kElt = ELT == kF32 ? 4 : 2;
  for (int b0 = 0; b0 < p.B; b0 += kMaxSeqs) {   // (as specmoe_verify_attn: consecutive launches)
    Kv4Params s = p;
    s.B = p.B - b0 < kMaxSeqs ? p.B - b0 : kMaxSeqs;
    s.q = p.q + (size_t)b0 * p.C_max * p.Hq * D * kElt;
    if (PAGED) {
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
    const int blocks = (p.Rcap + kBlk - 1) / kBlk;
    s.row_groups = blocks <= 2 ? 1 : blocks <= 4 ? 2 : 4;
    if (blocks == 1) hipLaunchKernelGGL((kv4_attn_kernel<ELT, D, PAGED, 1>), dim3(p.P), dim3(kGroupThreads), 0, stream, s);
    else hipLaunchKernelGGL((kv4_attn_kernel<ELT, D, PAGED, 2>), dim3(p.P), dim3(kGroupThreads), 0, stream, s);
  }
}

template <int ELT>
void launch_kv4_for(int D, const Kv4Params& p, hipStream_t s) {
  if (D == 128) {
    if (p.block_table) launch_kv4<ELT, 128, true>(p, s);
    else launch_kv4<ELT, 128, false>(p, s);
  } else {
    if (p.block_table) launch_kv4<ELT, 64, true>(p, s);
    else launch_kv4<ELT, 64, false>(p, s);
  }
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
  if ((int64_t)kMaxSeqs * desc->Hkv * ((desc->S_max + (int64_t)kTile - 1) / kTile) >= ((int64_t)1 << 31))
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
