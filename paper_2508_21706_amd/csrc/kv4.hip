// Rows of the 4-bit KV cache (specmoe_kv4.h) written, read back and moved, for
// MI355X (gfx950, CDNA4).  The attention over it is in kv4_attn.hip.
//
// Append: one workgroup per token, as specmoe_append_kv has it.  A query's items
// are pairs of 16-byte chunks whose entries are rotated with each other; a key's
// or value's items are 8 entries that lie side by side, a quarter of a block, so
// that a block's largest entry takes two exchanges between lanes and a lane's
// codes are one word.  A key's lane loads the chunk that its entries are rotated
// with once more, from the cache that holds the line by then.  Keys are worked out
// in fp64: fp64 runs at half fp32's rate here and a token has few keys, while in
// fp32 a key within 2^-24 of a border between two codes could take either.
//
// Read and move are copies: a lane has 8 entries (read) or 16 bytes of codes.
//
// Measured: one token 3.6 us, a chain of launch, length, sine and store; 8 prompts of
// 9,700 float16 tokens with norms and rotation 54 us for 209 MB (3.9 TB/s; a copy of that
// size 5.4), the rest fp64.  Read: one request's 1,000 rows 3.8 us, 148 MB of ragged
// prompts 26 to 36 us (warm and cold caches; 4.1 to 5.7 TB/s).  Move: 3.7 us for 64 trees of
// 16, 5.4 for 256 of 8 to 64 in pages, a chain of path, lookup, load and store.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "kv4.h"
#include "specmoe_kv4.h"

namespace {

constexpr int kF32 = SPECMOE_F32, kBF16 = SPECMOE_BF16, kF16 = SPECMOE_F16;
constexpr int kMaxThreads = 512;
constexpr int kManyTokens = 1024, kManyThreads = 192;   // (append) tokens from which on workgroups are smaller
constexpr int kMaxDraftBits = 64;
constexpr int64_t kMaxTokens = ((int64_t)1 << 32) / kMaxThreads - 1;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// Where a row of KV head 0 is, counted in rows of the cache, and the rows from
// one KV head to the next; fits: the row is in the cache.
struct Place {
  size_t row, head_step;
  bool fits;
};
struct Paging {
  const int32_t* table;   // NULL: a slab per sequence
  int shift, per_seq, pages;
};
__device__ __forceinline__ Place place_of(const Paging& pg, int Hkv, int S_max, int b, int64_t row) {
  Place x;
  x.fits = row < S_max;
  if (pg.table) {
    int page = -1;
    if (x.fits) page = pg.table[(size_t)b * pg.per_seq + (row >> pg.shift)];
    x.fits = page >= 0 && page < pg.pages;
    x.head_step = (size_t)1 << pg.shift;
    x.row = (((size_t)(x.fits ? page : 0) * Hkv) << pg.shift) + (size_t)(row & ((1 << pg.shift) - 1));
  } else {
    x.head_step = (size_t)S_max;
    x.row = (size_t)b * Hkv * S_max + (size_t)row;
  }
  return x;
}

// ------------------------------------------------------------------- append

struct AppendParams {
  const char* q;
  const char* k;
  const char* v;
  const char* q_weight;
  const char* k_weight;
  const double* inv_freq;
  const int32_t* ctx_lens;
  const int32_t* chunk_lens;
  const uint64_t* draft_mask;
  char* q_out;
  kv4::Cache cache;
  Paging paging;
  int64_t q_stride, k_stride, v_stride;   // bytes
  int Hq, Hkv, C_max, S_max;
  int rot_dim, pairs;
  float eps;
};

// the entries of a 16-byte chunk as fp32, and back with one rounding each
template <int ELT, int VE>
__device__ __forceinline__ void unpack(const u32x4& x, float* y) {
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    if constexpr (ELT == kF32) y[e] = __uint_as_float(x[e]);
    else if constexpr (ELT == kBF16) y[e] = __uint_as_float((e & 1) ? x[e >> 1] & 0xffff0000u : x[e >> 1] << 16);
    else y[e] = (float)__builtin_bit_cast(_Float16, (uint16_t)(x[e >> 1] >> (16 * (e & 1))));
  }
}
template <int ELT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  if constexpr (ELT == kBF16) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, (f16x2{(_Float16)lo, (_Float16)hi}));
  }
}
template <int ELT, int VE>
__device__ __forceinline__ u32x4 pack(const float (&y)[VE]) {
  u32x4 x;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (ELT == kF32) x[w] = __float_as_uint(y[w]);
    else x[w] = pack2<ELT>(y[2 * w], y[2 * w + 1]);
  }
  return x;
}

// 8 entries from the e-th of a row on, as fp32
template <int ELT>
__device__ __forceinline__ void load8(const char* row, int e, float (&y)[8]) {
  if constexpr (ELT == kF32) {
    unpack<ELT, 4>(*reinterpret_cast<const u32x4*>(row + 4 * e), y);
    unpack<ELT, 4>(*reinterpret_cast<const u32x4*>(row + 4 * e + 16), y + 4);
  } else {
    unpack<ELT, 8>(*reinterpret_cast<const u32x4*>(row + 2 * e), y);
  }
}

template <int ELT, int D>
__global__ __launch_bounds__(kMaxThreads) void append_kv4_kernel(AppendParams p) {
  constexpr int kElt = ELT == kF32 ? 4 : 2;
  constexpr int VE = 16 / kElt;      // entries per 16-byte chunk
  constexpr int LP = D / VE / 2;     // items of a query's row: chunk pairs
  constexpr int LK = D / 8;          // items of a key's or value's row
  constexpr int kRow = D * kElt;
  // cosines and sines, for the keys and, in fp32, for the queries
  __shared__ __attribute__((aligned(16))) double turn[2][D / 2];
  __shared__ __attribute__((aligned(16))) float turn_q[2][D / 2];

  const int tid = threadIdx.x;
  const int b = blockIdx.x / p.C_max, i = blockIdx.x - b * p.C_max;
  const int c = min(p.chunk_lens[b], p.C_max);
  const int64_t l = max(p.ctx_lens[b], 0);
  if (i >= c) return;
  const size_t token = (size_t)b * p.C_max + i;
  const int half = p.rot_dim >> 1;
  if (tid < half) {
    int64_t pos = l + i;
    if (p.draft_mask) {
      const uint64_t seen = p.draft_mask[token] & (c >= kMaxDraftBits ? ~0ull : (1ull << c) - 1);
      pos = l + max((int)__popcll(seen), 1) - 1;
    }
    // the angle in turns, less its whole turns: off by at most three roundings
    // of 2^-53 of the angle
    double t = (double)pos * p.inv_freq[tid] * 0.15915494309189533577;
    t -= rint(t);
    double sn, cs;
    sincospi(2.0 * t, &sn, &cs);
    turn[0][tid] = cs;
    turn[1][tid] = sn;
    turn_q[0][tid] = (float)cs;
    turn_q[1][tid] = (float)sn;
  }
  const Place at = place_of(p.paging, p.Hkv, p.S_max, b, l + i);
  __syncthreads();

  const int n_q = (p.Hq * LP + 63) & ~63;   // (whole waves have queries, or keys and values)
  const int n_k = n_q + p.Hkv * LK, n = n_k + p.Hkv * LK;
  const int rot_items = half / VE;
  for (int item = tid; item < ((n + 63) & ~63); item += blockDim.x) {
    if (item < n_q) {
      const int head = item / LP, s = item % LP;
      const bool in = head < p.Hq;
      const bool turned = s < rot_items;
      const bool split = turned && !p.pairs;   // chunks half a rotation apart
      const int ca = split ? s : 2 * s, cb = split ? s + rot_items : 2 * s + 1;
      const char* src = p.q + token * p.q_stride + (size_t)head * kRow;
      u32x4 xa = {0u, 0u, 0u, 0u}, xb = xa;
      if (in) {
        xa = *reinterpret_cast<const u32x4*>(src + 16 * ca);
        xb = *reinterpret_cast<const u32x4*>(src + 16 * cb);
      }
      float a[VE], z[VE];
      unpack<ELT, VE>(xa, a);
      unpack<ELT, VE>(xb, z);
      if (p.q_weight) {
        float g[VE], h[VE];
        unpack<ELT, VE>(*reinterpret_cast<const u32x4*>(p.q_weight + 16 * ca), g);
        unpack<ELT, VE>(*reinterpret_cast<const u32x4*>(p.q_weight + 16 * cb), h);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VE; ++e) ss = fmaf(a[e], a[e], fmaf(z[e], z[e], ss));
#pragma unroll
        for (int m = 1; m < LP; m <<= 1) ss += __shfl_xor(ss, m);
        const float inv = 1.f / sqrtf(ss * (1.f / D) + p.eps);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          a[e] *= inv * g[e];
          z[e] *= inv * h[e];
        }
      }
      if (turned) {
        const float* cs = turn_q[0] + s * VE;
        const float* sn = turn_q[1] + s * VE;
        if (!p.pairs) {
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float u = a[e], w = z[e], co = cs[e], si = sn[e];
            a[e] = u * co - w * si;
            z[e] = w * co + u * si;
          }
        } else {
#pragma unroll
          for (int e = 0; e < VE; e += 2) {
            const float u = a[e], w = a[e + 1], y = z[e], x = z[e + 1];
            const float c0 = cs[e / 2], s0 = sn[e / 2], c1 = cs[VE / 2 + e / 2], s1 = sn[VE / 2 + e / 2];
            a[e] = u * c0 - w * s0;
            a[e + 1] = w * c0 + u * s0;
            z[e] = y * c1 - x * s1;
            z[e + 1] = x * c1 + y * s1;
          }
        }
      }
      if (turned || p.q_weight) {   // (a row that is only copied keeps its bits)
        xa = pack<ELT, VE>(a);
        xb = pack<ELT, VE>(z);
      }
      if (in) {
        char* dst = p.q_out + (token * p.Hq + head) * kRow;
        *reinterpret_cast<u32x4*>(dst + 16 * ca) = xa;
        *reinterpret_cast<u32x4*>(dst + 16 * cb) = xb;
      }
      continue;
    }
    // 8 entries of a key or value: the values to encode in x
    const bool key = item < n_k, in = item < n;
    const int local = key ? item - n_q : item - n_k;
    const int head = in ? local / LK : 0, s = local % LK, e0 = 8 * s;
    const char* src = (key ? p.k + token * p.k_stride : p.v + token * p.v_stride) + (size_t)head * kRow;
    float x[8];
    load8<ELT>(src, e0, x);
    if (key && (p.k_weight || half)) {
      double y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = (double)x[e];
      const bool turned = e0 < p.rot_dim;
      const bool lower = e0 < half;
      const int partner = lower ? e0 + half : e0 - half;   // (halves) first entry that the lane's are rotated with
      float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (turned && !p.pairs) load8<ELT>(src, partner, z);
      double inv = 1.0;
      float g[8], h[8];
      if (p.k_weight) {
        double ss = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fma(y[e], y[e], ss);
#pragma unroll
        for (int m = 1; m < LK; m <<= 1) ss += __shfl_xor(ss, m);
        inv = 1.0 / sqrt(ss * (1.0 / D) + (double)p.eps);
        load8<ELT>(p.k_weight, e0, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= inv * (double)g[e];
      }
      if (turned && p.pairs) {
        const double* cs = turn[0] + e0 / 2;
        const double* sn = turn[1] + e0 / 2;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const double u = y[e], w = y[e + 1];
          y[e] = u * cs[e / 2] - w * sn[e / 2];
          y[e + 1] = w * cs[e / 2] + u * sn[e / 2];
        }
      } else if (turned) {
        const double* cs = turn[0] + (lower ? e0 : partner);
        const double* sn = turn[1] + (lower ? e0 : partner);
        if (p.k_weight) load8<ELT>(p.k_weight, partner, h);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          double w = (double)z[e];
          if (p.k_weight) w *= inv * (double)h[e];
          y[e] = lower ? y[e] * cs[e] - w * sn[e] : y[e] * cs[e] + w * sn[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = kv4::to_odd(y[e]);
    }
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[e]) & 0x7fffffffu);
    most = max(most, (uint32_t)__shfl_xor((int)most, 1));
    most = max(most, (uint32_t)__shfl_xor((int)most, 2));
    const uint32_t byte = kv4::scale_byte(most);
    const uint32_t word = kv4::codes_of(x, byte);
    if (in && at.fits) {
      const size_t row = at.row + head * at.head_step;
      *reinterpret_cast<uint32_t*>((key ? p.cache.k_codes : p.cache.v_codes) + row * (D / 2) + 4 * s) = word;
      if ((s & 3) == 0) (key ? p.cache.k_scales : p.cache.v_scales)[row * (D / 32) + (s >> 2)] = (char)byte;
    }
  }
}

// --------------------------------------------------------------------- read

constexpr int kReadThreads = 256;
constexpr int kReadTokens = 4;   // tokens of a workgroup (16 prefixes of 300 to 4096 rows, 148 MB: 36.5 us, with 16 tokens 41)

struct ReadParams {
  kv4::Cache cache;
  Paging paging;
  const int32_t* first;
  const int32_t* rows;
  char* k_out;
  char* v_out;
  int Hkv, N_max, S_max, tiles;
};

template <int ELT, int D>
__global__ __launch_bounds__(kReadThreads) void read_kv4_kernel(ReadParams p) {
  constexpr int kElt = ELT == kF32 ? 4 : 2;
  constexpr int LK = D / 8;
  const int b = blockIdx.x / p.tiles, i0 = (blockIdx.x - b * p.tiles) * kReadTokens;
  const int n = min(max(p.rows[b], 0), p.N_max) - i0;
  if (n <= 0) return;
  const int64_t first = (int64_t)max(p.first[b], 0) + i0;
  const char* codes = blockIdx.y == 0 ? p.cache.k_codes : p.cache.v_codes;
  const char* scales = blockIdx.y == 0 ? p.cache.k_scales : p.cache.v_scales;
  char* out = (blockIdx.y == 0 ? p.k_out : p.v_out) + ((size_t)b * p.N_max + i0) * p.Hkv * D * kElt;
  const int per = p.Hkv * LK, items = min(n, kReadTokens) * per;
  for (int item = threadIdx.x; item < items; item += kReadThreads) {
    const int i = item / per, local = item - i * per, head = local / LK, s = local % LK;
    const Place at = place_of(p.paging, p.Hkv, p.S_max, b, first + i);
    if (!at.fits) continue;
    const size_t row = at.row + head * at.head_step;
    const uint32_t word = *reinterpret_cast<const uint32_t*>(codes + row * (D / 2) + 4 * s);
    const float scale = kv4::scale_of((uint8_t)scales[row * (D / 32) + (s >> 2)]);
    u32x4 x = {kv4::bf16_of<0>(word, scale), kv4::bf16_of<1>(word, scale), kv4::bf16_of<2>(word, scale),
               kv4::bf16_of<3>(word, scale)};
    char* dst = out + (size_t)item * 8 * kElt;
    if constexpr (ELT == kBF16) {
      *reinterpret_cast<u32x4*>(dst) = x;
    } else {
      float y[8];
      unpack<kBF16, 8>(x, y);
      if constexpr (ELT == kF32) {
        *reinterpret_cast<u32x4*>(dst) = pack<kF32, 4>({y[0], y[1], y[2], y[3]});
        *reinterpret_cast<u32x4*>(dst + 16) = pack<kF32, 4>({y[4], y[5], y[6], y[7]});
      } else {
        *reinterpret_cast<u32x4*>(dst) = pack<kF16, 8>(y);
      }
    }
  }
}

// --------------------------------------------------------------------- move

constexpr int kMoveThreads = 256;

struct MoveParams {
  kv4::Cache cache;
  Paging paging;
  const int32_t* ctx_lens;
  const uint64_t* path;
  int Hkv, S_max;
};

// Row l + node_j to row l + j for the j-th set bit node_j of the path word, K
// (blockIdx.y = 0) or V (1) of one (sequence, KV head) (blockIdx.x): a thread
// has 16 bytes of a row's codes, and one of the first 64 a row's scales.  Every
// row is read before any is written, so overlapping moves are safe.
template <int D>
__global__ __launch_bounds__(kMoveThreads) void move_kv4_kernel(MoveParams p) {
  constexpr int kChunks = D / 32;   // 16-byte chunks of a row's codes, and bytes of its scales
  const int b = blockIdx.x / p.Hkv, head = blockIdx.x - b * p.Hkv;
  const int64_t l = max(p.ctx_lens[b], 0);
  const uint64_t w = p.path[b];
  if ((w & (w + 1)) == 0) return;   // nodes 0, 1, ...: nothing moves
  char* codes = blockIdx.y == 0 ? p.cache.k_codes : p.cache.v_codes;
  char* scales = blockIdx.y == 0 ? p.cache.k_scales : p.cache.v_scales;
  const int rows = __popcll(w);
  // the cache rows that row j of the path goes from and to
  auto places = [&](int j, size_t& from, size_t& to) {
    if (j >= rows) return false;
    uint64_t rest = w;   // the j-th set bit: clear j lowest set bits
    for (int i = 0; i < j; ++i) rest &= rest - 1;
    const int node = __builtin_ctzll(rest);
    if (node == j) return false;
    const Place a = place_of(p.paging, p.Hkv, p.S_max, b, l + node), z = place_of(p.paging, p.Hkv, p.S_max, b, l + j);
    from = a.row + head * a.head_step;
    to = z.row + head * z.head_step;
    return a.fits && z.fits;
  };
  const int tid = threadIdx.x;
  size_t from = 0, to = 0, sfrom = 0, sto = 0;
  const int ch = tid % kChunks;
  const bool move = places(tid / kChunks, from, to), smove = tid < 64 && places(tid, sfrom, sto);
  u32x4 x = {0u, 0u, 0u, 0u};
  uint32_t y = 0;
  if (move) x = *reinterpret_cast<const u32x4*>(codes + from * (D / 2) + 16 * ch);
  if (smove) {
    if constexpr (kChunks == 4) y = *reinterpret_cast<const uint32_t*>(scales + sfrom * kChunks);
    else y = *reinterpret_cast<const uint16_t*>(scales + sfrom * kChunks);
  }
  __syncthreads();
  if (move) *reinterpret_cast<u32x4*>(codes + to * (D / 2) + 16 * ch) = x;
  if (smove) {
    if constexpr (kChunks == 4) *reinterpret_cast<uint32_t*>(scales + sto * kChunks) = y;
    else *reinterpret_cast<uint16_t*>(scales + sto * kChunks) = (uint16_t)y;
  }
}
static_assert(64 * 128 / 32 <= kMoveThreads, "64 rows of codes in one go");

// ---------------------------------------------------------------- host side

bool aligned(const void* ptr, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(ptr) & (bytes - 1)) == 0; }

bool known_dtype(int t) { return t == SPECMOE_F32 || t == SPECMOE_BF16 || t == SPECMOE_F16; }

int validate_pages(const specmoe_paged_kv* pk, int S_max) {
  const int ps = pk->page_size;
  if (ps < 8 || ps > 65536 || (ps & (ps - 1)) != 0) return SPECMOE_ERR_PAGES;
  if (pk->pages_per_seq < 1 || pk->num_pages < 1) return SPECMOE_ERR_PAGES;
  if ((int64_t)ps * pk->pages_per_seq != S_max) return SPECMOE_ERR_PAGES;
  return SPECMOE_OK;
}

// The cache's members: all there, and aligned
int check_cache(const specmoe_kv4* c) {
  if (!c || !c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales) return SPECMOE_ERR_NULL_POINTER;
  return SPECMOE_OK;
}
bool cache_aligned(const specmoe_kv4* c) {
  return aligned(c->k_codes, 16) && aligned(c->k_scales, 16) && aligned(c->v_codes, 16) && aligned(c->v_scales, 16);
}
kv4::Cache cache_of(const specmoe_kv4* c) {
  return {static_cast<char*>(c->k_codes), static_cast<char*>(c->k_scales), static_cast<char*>(c->v_codes),
          static_cast<char*>(c->v_scales)};
}
Paging paging_of(const specmoe_paged_kv* pk, const int32_t* table) {
  if (!pk) return {nullptr, 0, 0, 0};
  return {table, __builtin_ctz((unsigned)pk->page_size), pk->pages_per_seq, pk->num_pages};
}

int validate_append(const specmoe_append_desc* d, bool tree, bool table, const specmoe_paged_kv* pk) {
  if (!d) return SPECMOE_ERR_NULL_POINTER;
  if (!known_dtype(d->dtype)) return SPECMOE_ERR_DTYPE;
  if (d->D != 64 && d->D != 128) return SPECMOE_ERR_HEAD_DIM;
  if (d->B < 0 || d->Hq < 0 || d->Hkv < 1 || d->C_max < 1 || d->S_max < 1) return SPECMOE_ERR_SHAPE;
  // one workgroup per token (a launch holds less than 2^32 threads); items of
  // a token stay in 32 bits
  if ((int64_t)d->B * d->C_max > kMaxTokens || d->Hq > (1 << 20) || d->Hkv > (1 << 20)) return SPECMOE_ERR_SHAPE;
  const int64_t elt = d->dtype == SPECMOE_F32 ? 4 : 2;
  const int64_t strides[3] = {d->q_stride, d->k_stride, d->v_stride}, heads[3] = {d->Hq, d->Hkv, d->Hkv};
  for (int n = 0; n < 3; ++n) {
    if (strides[n] == 0) continue;
    // (offsets of tokens stay below 2^63)
    if (strides[n] < heads[n] * d->D || strides[n] >= ((int64_t)1 << 28) || strides[n] * elt % 16 != 0)
      return SPECMOE_ERR_SHAPE;
  }
  if (d->rot_dim < 0 || d->rot_dim > d->D || d->rot_dim % 16 != 0) return SPECMOE_ERR_ROPE;
  if (d->rope_style != SPECMOE_ROPE_HALVES && d->rope_style != SPECMOE_ROPE_PAIRS) return SPECMOE_ERR_ROPE;
  if (!(d->norm_eps >= 0.f) || !isfinite(d->norm_eps)) return SPECMOE_ERR_ROPE;
  if (tree && d->C_max > kMaxDraftBits) return SPECMOE_ERR_MASK;
  if (pk) return validate_pages(pk, d->S_max);
  return table ? SPECMOE_ERR_NULL_POINTER : SPECMOE_OK;
}

int validate_rows(const specmoe_kv4_desc* d, bool read, bool table, const specmoe_paged_kv* pk) {
  if (!d) return SPECMOE_ERR_NULL_POINTER;
  if (read && !known_dtype(d->dtype)) return SPECMOE_ERR_DTYPE;
  if (d->D != 64 && d->D != 128) return SPECMOE_ERR_HEAD_DIM;
  if (d->B < 0 || d->Hkv < 1 || d->Hkv > (1 << 20) || d->S_max < 1) return SPECMOE_ERR_SHAPE;
  if (read) {
    // (a launch holds less than 2^32 threads; a token's items stay in 32 bits)
    if (d->N_max < 1 || (int64_t)d->B * d->N_max >= ((int64_t)1 << 31)) return SPECMOE_ERR_SHAPE;
    if ((int64_t)d->B * ((d->N_max + (int64_t)kReadTokens - 1) / kReadTokens) >= (1 << 24) - 1) return SPECMOE_ERR_SHAPE;
  } else if ((int64_t)d->B * d->Hkv >= (1 << 23)) {
    return SPECMOE_ERR_SHAPE;
  }
  if (pk) return validate_pages(pk, d->S_max);
  return table ? SPECMOE_ERR_NULL_POINTER : SPECMOE_OK;
}

template <int ELT>
void launch_append(int D, const AppendParams& p, unsigned tokens, hipStream_t s) {
  const int LP = D * (ELT == kF32 ? 4 : 2) / 32;
  const int64_t items = ((p.Hq * LP + 63) & ~63) + 2 * p.Hkv * (D / 8);
  // A prompt's tokens in several rounds of fewer waves, as more tokens to a CU hide
  // more (prompts of 8, 9,700 tokens, 55 us against 67); a few tokens in one round
  // (one token 3.6 us against 4.2).
  const int most = tokens > kManyTokens ? kManyThreads : kMaxThreads;
  const int64_t rounds = (items + most - 1) / most;
  const int threads = (int)(((items + rounds - 1) / rounds + 63) / 64 * 64);
  if (D == 128) hipLaunchKernelGGL((append_kv4_kernel<ELT, 128>), dim3(tokens), dim3(threads), 0, s, p);
  else hipLaunchKernelGGL((append_kv4_kernel<ELT, 64>), dim3(tokens), dim3(threads), 0, s, p);
}

template <int ELT>
void launch_read(int D, const ReadParams& p, unsigned groups, hipStream_t s) {
  if (D == 128) hipLaunchKernelGGL((read_kv4_kernel<ELT, 128>), dim3(groups, 2), dim3(kReadThreads), 0, s, p);
  else hipLaunchKernelGGL((read_kv4_kernel<ELT, 64>), dim3(groups, 2), dim3(kReadThreads), 0, s, p);
}

}  // namespace

extern "C" {

int specmoe_append_kv4(const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight,
                       const double* inv_freq, const int32_t* ctx_lens, const int32_t* chunk_lens,
                       const uint64_t* draft_mask, const int32_t* block_table, void* q_out, const specmoe_kv4* cache,
                       void* stream, const specmoe_append_desc* desc, const specmoe_paged_kv* paged) {
  int st = validate_append(desc, draft_mask != nullptr, block_table != nullptr, paged);
  if (st != SPECMOE_OK) return st;
  if (desc->B == 0) return SPECMOE_OK;
  if (!k || !v || !ctx_lens || !chunk_lens) return SPECMOE_ERR_NULL_POINTER;
  if ((st = check_cache(cache)) != SPECMOE_OK) return st;
  if (desc->Hq > 0 && (!q || !q_out)) return SPECMOE_ERR_NULL_POINTER;
  if (desc->rot_dim > 0 && !inv_freq) return SPECMOE_ERR_NULL_POINTER;
  if (paged && !block_table) return SPECMOE_ERR_NULL_POINTER;
  for (const void* ptr : {q, k, v, q_weight, k_weight, (const void*)q_out})
    if (!aligned(ptr, 16)) return SPECMOE_ERR_ALIGN;
  if (!cache_aligned(cache) || !aligned(inv_freq, 8) || !aligned(draft_mask, 8)) return SPECMOE_ERR_ALIGN;

  const int64_t elt = desc->dtype == SPECMOE_F32 ? 4 : 2;
  AppendParams p;
  p.q = static_cast<const char*>(q);
  p.k = static_cast<const char*>(k);
  p.v = static_cast<const char*>(v);
  p.q_weight = static_cast<const char*>(q_weight);
  p.k_weight = static_cast<const char*>(k_weight);
  p.inv_freq = inv_freq;
  p.ctx_lens = ctx_lens;
  p.chunk_lens = chunk_lens;
  p.draft_mask = draft_mask;
  p.q_out = static_cast<char*>(q_out);
  p.cache = cache_of(cache);
  p.paging = paging_of(paged, block_table);
  p.q_stride = elt * (desc->q_stride ? desc->q_stride : (int64_t)desc->Hq * desc->D);
  p.k_stride = elt * (desc->k_stride ? desc->k_stride : (int64_t)desc->Hkv * desc->D);
  p.v_stride = elt * (desc->v_stride ? desc->v_stride : (int64_t)desc->Hkv * desc->D);
  p.Hq = desc->Hq;
  p.Hkv = desc->Hkv;
  p.C_max = desc->C_max;
  p.S_max = desc->S_max;
  p.rot_dim = desc->rot_dim;
  p.pairs = desc->rope_style == SPECMOE_ROPE_PAIRS;
  p.eps = desc->norm_eps;

  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned tokens = (unsigned)((int64_t)desc->B * desc->C_max);
  (void)hipGetLastError();
  if (desc->dtype == SPECMOE_BF16) launch_append<kBF16>(desc->D, p, tokens, s);
  else if (desc->dtype == SPECMOE_F16) launch_append<kF16>(desc->D, p, tokens, s);
  else launch_append<kF32>(desc->D, p, tokens, s);
  return hipGetLastError() == hipSuccess ? SPECMOE_OK : SPECMOE_ERR_LAUNCH;
}

int specmoe_read_kv4(const specmoe_kv4* cache, const int32_t* block_table, const int32_t* first, const int32_t* rows,
                     void* k_out, void* v_out, void* stream, const specmoe_kv4_desc* desc,
                     const specmoe_paged_kv* paged) {
  int st = validate_rows(desc, true, block_table != nullptr, paged);
  if (st != SPECMOE_OK) return st;
  if (desc->B == 0) return SPECMOE_OK;
  if ((st = check_cache(cache)) != SPECMOE_OK) return st;
  if (!first || !rows || !k_out || !v_out || (paged && !block_table)) return SPECMOE_ERR_NULL_POINTER;
  if (!cache_aligned(cache) || !aligned(k_out, 16) || !aligned(v_out, 16)) return SPECMOE_ERR_ALIGN;

  ReadParams p;
  p.cache = cache_of(cache);
  p.paging = paging_of(paged, block_table);
  p.first = first;
  p.rows = rows;
  p.k_out = static_cast<char*>(k_out);
  p.v_out = static_cast<char*>(v_out);
  p.Hkv = desc->Hkv;
  p.N_max = desc->N_max;
  p.S_max = desc->S_max;
  p.tiles = (int)((desc->N_max + (int64_t)kReadTokens - 1) / kReadTokens);

  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned groups = (unsigned)desc->B * (unsigned)p.tiles;
  (void)hipGetLastError();
  if (desc->dtype == SPECMOE_BF16) launch_read<kBF16>(desc->D, p, groups, s);
  else if (desc->dtype == SPECMOE_F16) launch_read<kF16>(desc->D, p, groups, s);
  else launch_read<kF32>(desc->D, p, groups, s);
  return hipGetLastError() == hipSuccess ? SPECMOE_OK : SPECMOE_ERR_LAUNCH;
}

int specmoe_compact_accepted_kv4(const specmoe_kv4* cache, const int32_t* block_table, const int32_t* ctx_lens,
                                 const uint64_t* path, void* stream, const specmoe_kv4_desc* desc,
                                 const specmoe_paged_kv* paged) {
  int st = validate_rows(desc, false, block_table != nullptr, paged);
  if (st != SPECMOE_OK) return st;
  if (desc->B == 0) return SPECMOE_OK;
  if ((st = check_cache(cache)) != SPECMOE_OK) return st;
  if (!ctx_lens || !path || (paged && !block_table)) return SPECMOE_ERR_NULL_POINTER;
  if (!cache_aligned(cache) || !aligned(path, 8)) return SPECMOE_ERR_ALIGN;

  MoveParams p;
  p.cache = cache_of(cache);
  p.paging = paging_of(paged, block_table);
  p.ctx_lens = ctx_lens;
  p.path = path;
  p.Hkv = desc->Hkv;
  p.S_max = desc->S_max;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned units = (unsigned)desc->B * (unsigned)desc->Hkv;
  (void)hipGetLastError();
  if (desc->D == 128) hipLaunchKernelGGL((move_kv4_kernel<128>), dim3(units, 2), dim3(kMoveThreads), 0, s, p);
  else hipLaunchKernelGGL((move_kv4_kernel<64>), dim3(units, 2), dim3(kMoveThreads), 0, s, p);
  return hipGetLastError() == hipSuccess ? SPECMOE_OK : SPECMOE_ERR_LAUNCH;
}

}  // extern "C"
