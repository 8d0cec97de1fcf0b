// A chunk's queries, keys and values put in place for the verification
// attention, for MI355X (gfx950, CDNA4): head norms, the rotation by the
// position, and the append to a contiguous or paged KV cache in one pass.
//
// Every entry is read once and written once, so the step is bound by HBM for
// prompts and by its latencies for chunks of draft tokens:
//   * one workgroup per token.  Its head rows are cut into items of two 16-byte
//     chunks whose entries are rotated with each other, so a lane holds both
//     halves of every pair it turns and nothing crosses lanes but the sum of
//     squares of a norm (4 to 16 lanes);
//   * the loads of all items go out before anything else is worked out; the
//     first lanes turn the position into rot_dim / 2 sines and cosines, shared
//     through LDS, while they are under way: the angle and its reduction to
//     one turn in fp64, then one fp32 sine and cosine each.
// 10,900 tokens of 8 prompts (32 + 2 x 8 heads of 128, bf16) move their 268 MB
// in 53 us, 5.1 TB/s, near what a copy of that size reaches (5.4 TB/s).  A chunk of 5
// for 64 sequences takes 5.2 us on the GPU and one sequence's 2.5 us, of which
// most are the chain of lengths, table, angle and stores; the calls' host side
// (9 to 11 us) is longer.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "specmoe_append.h"

namespace {

constexpr int kF32 = SPECMOE_F32, kBF16 = SPECMOE_BF16, kF16 = SPECMOE_F16;
constexpr int kMaxThreads = 512;
constexpr int kMaxDraftBits = 64;
constexpr int64_t kMaxTokens = ((int64_t)1 << 32) / kMaxThreads - 1;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

struct Params {
  const char* q;
  const char* k;
  const char* v;
  const char* q_weight;
  const char* k_weight;
  const double* inv_freq;
  const int32_t* ctx_lens;
  const int32_t* chunk_lens;
  const uint64_t* draft_mask;
  const int32_t* block_table;
  char* q_out;
  char* k_cache;
  char* v_cache;
  int64_t q_stride, k_stride, v_stride;   // bytes
  int Hq, Hkv, C_max, S_max;
  int rot_dim, pairs;
  float eps;
  int page_shift, pages_per_seq, num_pages;   // (block_table != NULL)
};

// the VE entries of a 16-byte chunk as fp32, and back with one rounding each
template <int ELT, int VE>
__device__ __forceinline__ void unpack(const u32x4& x, float (&y)[VE]) {
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    if constexpr (ELT == kF32) y[e] = __uint_as_float(x[e]);
    else if constexpr (ELT == kBF16) y[e] = __uint_as_float((e & 1) ? x[e >> 1] & 0xffff0000u : x[e >> 1] << 16);
    else y[e] = (float)__builtin_bit_cast(_Float16, (uint16_t)(x[e >> 1] >> (16 * (e & 1))));
  }
}
template <int ELT, int VE>
__device__ __forceinline__ u32x4 pack(const float (&y)[VE]) {
  u32x4 x;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (ELT == kF32) {
      x[w] = __float_as_uint(y[w]);
    } else if constexpr (ELT == kBF16) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      x[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{y[2 * w], y[2 * w + 1]}), bf16x2));
    } else {
      typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
      x[w] = __builtin_bit_cast(uint32_t, (f16x2{(_Float16)y[2 * w], (_Float16)y[2 * w + 1]}));
    }
  }
  return x;
}

template <int ELT, int D>
__global__ __launch_bounds__(kMaxThreads) void append_kernel(Params p) {
  constexpr int kElt = ELT == kF32 ? 4 : 2;
  constexpr int VE = 16 / kElt;      // entries per 16-byte chunk
  constexpr int LP = D / VE / 2;     // items (chunk pairs) of a head row: 4 to 16
  constexpr int kRow = D * kElt;     // bytes of a head row
  __shared__ __attribute__((aligned(16))) float turn[2][D / 2];   // cosines, sines

  const int tid = threadIdx.x;
  const int b = blockIdx.x / p.C_max, i = blockIdx.x - b * p.C_max;
  const int c = min(p.chunk_lens[b], p.C_max);
  const int64_t l = max(p.ctx_lens[b], 0);
  if (i >= c) return;
  const size_t token = (size_t)b * p.C_max + i;
  const int half = p.rot_dim >> 1;

  // where the token's K and V rows go: the row of KV head 0, and the distance
  // from one KV head to the next
  const int64_t row = l + i;
  bool fits = row < p.S_max;
  size_t at = 0, head_step = 0;
  if (p.block_table) {
    int page = -1;
    if (fits) page = p.block_table[(size_t)b * p.pages_per_seq + (row >> p.page_shift)];
    fits = page >= 0 && page < p.num_pages;
    head_step = (size_t)kRow << p.page_shift;
    at = (size_t)(fits ? page : 0) * p.Hkv * head_step + (size_t)(row & ((1 << p.page_shift) - 1)) * kRow;
  } else {
    head_step = (size_t)p.S_max * kRow;
    at = (size_t)b * p.Hkv * head_step + (size_t)row * kRow;
  }

  const int rot_items = half / VE;   // items of a row whose entries are rotated
  const int n_q = p.Hq * LP, n_k = n_q + p.Hkv * LP, n = n_k + p.Hkv * LP;
  for (int base = 0; base < n; base += blockDim.x) {
    // item s of head row `head` of q (0), k (1) or v (2): two chunks
    const int item = base + tid;
    const bool in = item < n;
    const int which = item < n_q ? 0 : item < n_k ? 1 : 2;
    const int local = which == 0 ? item : which == 1 ? item - n_q : item - n_k;
    const int head = local / LP, s = local % LP;
    const bool turned = s < rot_items;
    const bool split = turned && !p.pairs;   // chunks half a rotation apart
    const int ca = split ? s : 2 * s, cb = split ? s + rot_items : 2 * s + 1;
    const char* src = which == 0 ? p.q + token * p.q_stride : which == 1 ? p.k + token * p.k_stride : p.v + token * p.v_stride;
    src += head * kRow;
    const char* weight = which == 0 ? p.q_weight : which == 1 ? p.k_weight : nullptr;
    u32x4 xa = {0u, 0u, 0u, 0u}, xb = xa, wa = xa, wb = xa;
    if (in) {
      xa = *reinterpret_cast<const u32x4*>(src + 16 * ca);
      xb = *reinterpret_cast<const u32x4*>(src + 16 * cb);
      if (weight) {
        wa = *reinterpret_cast<const u32x4*>(weight + 16 * ca);
        wb = *reinterpret_cast<const u32x4*>(weight + 16 * cb);
      }
    }
    if (base == 0) {
      if (tid < half) {
        int64_t pos = row;
        if (p.draft_mask) {
          const uint64_t seen = p.draft_mask[token] & (c >= kMaxDraftBits ? ~0ull : (1ull << c) - 1);
          pos = l + max((int)__popcll(seen), 1) - 1;
        }
        // the angle in turns, less its whole turns: off by at most three
        // roundings of 2^-53 of the angle (two products, the constant), so far
        // positions lose nothing in fp32
        double t = (double)pos * p.inv_freq[tid] * 0.15915494309189533577;
        t -= rint(t);
        float sn, cs;
        sincospif((float)(2.0 * t), &sn, &cs);
        turn[0][tid] = cs;
        turn[1][tid] = sn;
      }
      __syncthreads();
    }
    if (which < 2) {
      float a[VE], z[VE];
      unpack<ELT, VE>(xa, a);
      unpack<ELT, VE>(xb, z);
      if (weight) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VE; ++e) ss = fmaf(a[e], a[e], fmaf(z[e], z[e], ss));
#pragma unroll
        for (int m = 1; m < LP; m <<= 1) ss += __shfl_xor(ss, m);
        const float inv = 1.f / sqrtf(ss * (1.f / D) + p.eps);
        float g[VE], h[VE];
        unpack<ELT, VE>(wa, g);
        unpack<ELT, VE>(wb, h);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          a[e] *= inv * g[e];
          z[e] *= inv * h[e];
        }
      }
      if (turned) {
        const float* cs = turn[0] + s * VE;
        const float* sn = turn[1] + s * VE;
        if (!p.pairs) {
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float u = a[e], w = z[e];
            a[e] = u * cs[e] - w * sn[e];
            z[e] = w * cs[e] + u * sn[e];
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
      if (turned || weight) {   // (a row that is only copied keeps its bits)
        xa = pack<ELT, VE>(a);
        xb = pack<ELT, VE>(z);
      }
    }
    char* dst = which == 0 ? p.q_out + (token * p.Hq + head) * kRow
                           : (which == 1 ? p.k_cache : p.v_cache) + at + head * head_step;
    if (in && (which == 0 || fits)) {
      *reinterpret_cast<u32x4*>(dst + 16 * ca) = xa;
      *reinterpret_cast<u32x4*>(dst + 16 * cb) = xb;
    }
  }
}

// ---------------------------------------------------------------- host side

bool aligned(const void* ptr, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(ptr) & (bytes - 1)) == 0; }

int validate(const specmoe_append_desc* d, bool tree, bool table, const specmoe_paged_kv* pk) {
  if (!d) return SPECMOE_ERR_NULL_POINTER;
  if (d->dtype != SPECMOE_F32 && d->dtype != SPECMOE_BF16 && d->dtype != SPECMOE_F16) return SPECMOE_ERR_DTYPE;
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
  if (pk) {
    const int ps = pk->page_size;
    if (ps < 8 || ps > 65536 || (ps & (ps - 1)) != 0) return SPECMOE_ERR_PAGES;
    if (pk->pages_per_seq < 1 || pk->num_pages < 1) return SPECMOE_ERR_PAGES;
    if ((int64_t)ps * pk->pages_per_seq != d->S_max) return SPECMOE_ERR_PAGES;
  } else if (table) {
    return SPECMOE_ERR_NULL_POINTER;
  }
  return SPECMOE_OK;
}

template <int ELT>
void launch(int D, const Params& p, unsigned tokens, hipStream_t s) {
  const int items = (p.Hq + 2 * p.Hkv) * (D * (ELT == kF32 ? 4 : 2) / 32);
  const int rounds = (items + kMaxThreads - 1) / kMaxThreads;
  const int threads = ((items + rounds - 1) / rounds + 63) / 64 * 64;
  if (D == 128) hipLaunchKernelGGL((append_kernel<ELT, 128>), dim3(tokens), dim3(threads), 0, s, p);
  else hipLaunchKernelGGL((append_kernel<ELT, 64>), dim3(tokens), dim3(threads), 0, s, p);
}

}  // namespace

extern "C" int specmoe_append_kv(const void* q, const void* k, const void* v, const void* q_weight,
                                 const void* k_weight, const double* inv_freq, const int32_t* ctx_lens,
                                 const int32_t* chunk_lens, const uint64_t* draft_mask, const int32_t* block_table,
                                 void* q_out, void* k_cache, void* v_cache, void* stream,
                                 const specmoe_append_desc* desc, const specmoe_paged_kv* paged) {
  const int st = validate(desc, draft_mask != nullptr, block_table != nullptr, paged);
  if (st != SPECMOE_OK) return st;
  if (desc->B == 0) return SPECMOE_OK;
  if (!k || !v || !ctx_lens || !chunk_lens || !k_cache || !v_cache) return SPECMOE_ERR_NULL_POINTER;
  if (desc->Hq > 0 && (!q || !q_out)) return SPECMOE_ERR_NULL_POINTER;
  if (desc->rot_dim > 0 && !inv_freq) return SPECMOE_ERR_NULL_POINTER;
  if (paged && !block_table) return SPECMOE_ERR_NULL_POINTER;
  for (const void* ptr : {q, k, v, q_weight, k_weight, (const void*)q_out, (const void*)k_cache, (const void*)v_cache})
    if (!aligned(ptr, 16)) return SPECMOE_ERR_ALIGN;
  if (!aligned(inv_freq, 8) || !aligned(draft_mask, 8)) return SPECMOE_ERR_ALIGN;

  const int64_t elt = desc->dtype == SPECMOE_F32 ? 4 : 2;
  Params p;
  p.q = static_cast<const char*>(q);
  p.k = static_cast<const char*>(k);
  p.v = static_cast<const char*>(v);
  p.q_weight = static_cast<const char*>(q_weight);
  p.k_weight = static_cast<const char*>(k_weight);
  p.inv_freq = inv_freq;
  p.ctx_lens = ctx_lens;
  p.chunk_lens = chunk_lens;
  p.draft_mask = draft_mask;
  p.block_table = paged ? block_table : nullptr;
  p.q_out = static_cast<char*>(q_out);
  p.k_cache = static_cast<char*>(k_cache);
  p.v_cache = static_cast<char*>(v_cache);
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
  p.page_shift = paged ? __builtin_ctz((unsigned)paged->page_size) : 0;
  p.pages_per_seq = paged ? paged->pages_per_seq : 0;
  p.num_pages = paged ? paged->num_pages : 0;

  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned tokens = (unsigned)((int64_t)desc->B * desc->C_max);
  (void)hipGetLastError();
  if (desc->dtype == SPECMOE_BF16) launch<kBF16>(desc->D, p, tokens, s);
  else if (desc->dtype == SPECMOE_F16) launch<kF16>(desc->D, p, tokens, s);
  else launch<kF32>(desc->D, p, tokens, s);
  return hipGetLastError() == hipSuccess ? SPECMOE_OK : SPECMOE_ERR_LAUNCH;
}
