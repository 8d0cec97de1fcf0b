// Block tables and slot maps of a paged KV cache from the requests' lengths
// (specmoe_pages.h), for MI355X (gfx950, CDNA4).
//
// What comes back and what is taken are prefix sums over the requests, and a
// page's place on the stack follows from them, so one workgroup does a step
// without atomics: up to 1024 requests at a time, one per thread, are counted,
// summed (in a wave's registers, then over the waves through LDS), and their pages
// moved as one list, each item finding its request by a search in the sums.  Pages
// given back are written to the stack before any is taken off it.  A decode step
// moves few bytes; its time is the chain lengths, sums, stack, table: 5.6 us for 64
// requests, 4.6 for one.  512 requests of which half are new prompts move 17,000 pages
// each way in 17 us, a CU's latencies.  Slots are written by the same workgroup where
// they are few, else by a launch of their own (4.7 us for 512 prompts; 5,120 slots of
// 1024 requests 11.7 us in all, by the step's workgroup 16.5).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "specmoe_pages.h"

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kSlotThreads = 256;
// Slots up to which the step's workgroup writes them itself
constexpr int64_t kOwnSlots = 2048;

struct Params {
  const int32_t* ctx_lens;
  const int32_t* chunk_lens;
  int32_t* table;
  int32_t* held;
  int32_t* free_pages;
  int32_t* free_count;
  int32_t* missing;
  int64_t* slots;
  int B, C_max, page_shift, pages_per_seq, num_pages;
};

struct Need {
  int l, c, pages;   // clamped lengths, and the pages that they take
};
__device__ __forceinline__ Need need_of(const Params& p, int b) {
  Need n;
  const int most = p.pages_per_seq << p.page_shift;   // (< 2^31: host check)
  n.l = min(max(p.ctx_lens[b], 0), most);
  n.c = min(min(max(p.chunk_lens[b], 0), p.C_max), most - n.l);
  n.pages = (int)(((int64_t)n.l + n.c + (1 << p.page_shift) - 1) >> p.page_shift);
  return n;
}

__device__ __forceinline__ int wave_scan(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d);
    if ((int)(threadIdx.x & 63) >= d) x += y;
  }
  return x;
}

// Inclusive sums of x over the workgroup's threads, also left in sums[]; all
// threads get the total.  (Sums stay below 2^31: host check.)
__device__ int block_scan(int x, int* sums, int* waves, int& total) {
  const int tid = threadIdx.x;
  x = wave_scan(x);
  __syncthreads();   // (the last use of sums and waves)
  if ((tid & 63) == 63) waves[tid >> 6] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int s = waves[w];
    before += w < (tid >> 6) ? s : 0;
    all += s;
  }
  total = all;
  sums[tid] = x + before;
  __syncthreads();
  return x + before;
}

// Copies the first n of the pages that this lot's requests give back or take, a page to
// a thread, which searches for its request in the inclusive sums: place(r, k, i, from,
// to) is where request r's k-th page, the i-th of all, is and goes.
//
// A search is ten dependent LDS reads and the page a load behind them; kTogether of both
// are in flight (17,000 pages: 21.7 us a step with its slots, one at a time 24.8).
// (Indexes past the last page, which may be the 2^31st, stay below 2^32.)
template <int kTogether, class Place>
__device__ __forceinline__ void copy_list(const int* sums, int n, const Place& place) {
  for (uint32_t i0 = threadIdx.x; i0 < (uint32_t)n; i0 += kTogether * kThreads) {
    int at[kTogether], lo[kTogether];
#pragma unroll
    for (int u = 0; u < kTogether; ++u) at[u] = (int)min(i0 + u * kThreads, (uint32_t)n - 1), lo[u] = 0;
    // the first thread whose inclusive sum exceeds the item's index
#pragma unroll
    for (int step = kThreads / 2; step; step >>= 1)
#pragma unroll
      for (int u = 0; u < kTogether; ++u) lo[u] += sums[lo[u] + step - 1] <= at[u] ? step : 0;
    int32_t* to[kTogether];
    int32_t x[kTogether];
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
      const int32_t* from;
      place(lo[u], at[u] - (lo[u] ? sums[lo[u] - 1] : 0), at[u], from, to[u]);
      x[u] = *from;
    }
    // (past the end the last page is written again, with the same value)
#pragma unroll
    for (int u = 0; u < kTogether; ++u) *to[u] = x[u];
  }
}
template <class Place>
__device__ __forceinline__ void copy_pages(const int* sums, int n, const Place& place) {
  if (n <= kThreads) copy_list<1>(sums, n, place);
  else copy_list<4>(sums, n, place);
}

__device__ __forceinline__ int64_t slot_of(const Params& p, int b, const Need& n, int held, int i) {
  if (i >= n.c) return -1;
  const int pos = n.l + i;   // (< 2^31, as l + c is)
  if ((pos >> p.page_shift) >= held) return -1;
  const int64_t page = p.table[(size_t)b * p.pages_per_seq + (pos >> p.page_shift)];
  return (page << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
}

__global__ __launch_bounds__(kThreads) void assign_kernel(Params p, int write_slots) {
  __shared__ int sums[kThreads], first[kThreads], waves[kWaves];
  const int tid = threadIdx.x;
  const int64_t per = p.pages_per_seq;
  int count = min(max(*p.free_count, 0), p.num_pages);

  // 1. what comes back, on the stack
  for (int b0 = 0; b0 < p.B; b0 += kThreads) {
    const int b = b0 + tid;
    int back = 0;
    if (b < p.B) {
      const int need = need_of(p, b).pages;
      back = max(min(max(p.held[b], 0), p.pages_per_seq) - need, 0);
      first[tid] = need;
    }
    int total;
    block_scan(back, sums, waves, total);
    copy_pages(sums, min(total, p.num_pages - count), [&](int r, int k, int i, const int32_t*& from, int32_t*& to) {
      from = p.table + (b0 + r) * per + first[r] + k;
      to = p.free_pages + count + i;
    });
    count = (int)min((int64_t)count + total, (int64_t)p.num_pages);
    if (b0 + kThreads < p.B) __syncthreads();   // (first[])
  }
  __threadfence_block();
  __syncthreads();

  // 2. what is taken off it
  const int stack = count;
  int asked = 0;    // pages that the requests before wanted
  int taken = 0;
  for (int b0 = 0; b0 < p.B; b0 += kThreads) {
    const int b = b0 + tid;
    int want = 0, held = 0, need = 0;
    if (b < p.B) {
      need = need_of(p, b).pages;
      held = min(max(p.held[b], 0), p.pages_per_seq);
      want = max(need - held, 0);
      first[tid] = held;
    }
    int total;
    const int end = block_scan(want, sums, waves, total);
    // (in 64 bits: the sums of two lots may pass 2^31)
    const bool served = (int64_t)asked + end <= stack;
    if (b < p.B) {
      p.held[b] = served ? need : min(held, need);
      if (p.missing) p.missing[b] = served ? 0 : want;
    }
    // the requests that are served come first: theirs are the first items
    const int last = __syncthreads_count(served);
    const int items = last ? sums[last - 1] : 0;
    copy_pages(sums, items, [&](int r, int k, int i, const int32_t*& from, int32_t*& to) {
      from = p.free_pages + (stack - 1 - asked - i);
      to = p.table + (b0 + r) * per + first[r] + k;
    });
    taken += items;
    asked = (int)min((int64_t)asked + total, (int64_t)0x7fffffff);
    if (b0 + kThreads < p.B) __syncthreads();   // (first[])
  }
  if (tid == 0) *p.free_count = stack - taken;

  // 3. slots
  if (!write_slots) return;
  __threadfence_block();
  __syncthreads();
  const int n = p.B * p.C_max;
  for (int s = tid; s < n; s += kThreads) {
    const int b = s / p.C_max;
    p.slots[s] = slot_of(p, b, need_of(p, b), p.held[b], s - b * p.C_max);
  }
}

__global__ __launch_bounds__(kSlotThreads) void slots_kernel(Params p) {
  const int b = blockIdx.y;
  const int i = blockIdx.x * kSlotThreads + threadIdx.x;
  if (i < p.C_max) p.slots[(size_t)b * p.C_max + i] = slot_of(p, b, need_of(p, b), p.held[b], i);
}

// ---------------------------------------------------------------- host side

bool aligned(const void* ptr, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(ptr) & (bytes - 1)) == 0; }

int validate(const specmoe_pages_desc* d, bool slots) {
  if (!d) return SPECMOE_ERR_NULL_POINTER;
  // (a launch's second grid dimension holds less than 2^16 workgroups)
  if (d->B < 0 || d->B > 65535 || d->C_max < 1) return SPECMOE_ERR_SHAPE;
  if (slots && (int64_t)d->B * d->C_max >= ((int64_t)1 << 31)) return SPECMOE_ERR_SHAPE;
  const int ps = d->page_size;
  if (ps < 8 || ps > 65536 || (ps & (ps - 1)) != 0) return SPECMOE_ERR_PAGES;
  if (d->pages_per_seq < 1 || d->num_pages < 1) return SPECMOE_ERR_PAGES;
  if ((int64_t)ps * d->pages_per_seq >= ((int64_t)1 << 31)) return SPECMOE_ERR_PAGES;
  if ((int64_t)d->B * d->pages_per_seq >= ((int64_t)1 << 31)) return SPECMOE_ERR_PAGES;
  return SPECMOE_OK;
}

}  // namespace

extern "C" int specmoe_assign_pages(const int32_t* ctx_lens, const int32_t* chunk_lens, int32_t* block_table,
                                    int32_t* held, int32_t* free_pages, int32_t* free_count, int32_t* missing,
                                    int64_t* slots, void* stream, const specmoe_pages_desc* desc) {
  const int st = validate(desc, slots != nullptr);
  if (st != SPECMOE_OK) return st;
  if (desc->B == 0) return SPECMOE_OK;
  if (!ctx_lens || !chunk_lens || !block_table || !held || !free_pages || !free_count) return SPECMOE_ERR_NULL_POINTER;
  for (const void* ptr : {(const void*)ctx_lens, (const void*)chunk_lens, (const void*)block_table, (const void*)held,
                          (const void*)free_pages, (const void*)free_count, (const void*)missing})
    if (!aligned(ptr, 4)) return SPECMOE_ERR_ALIGN;
  if (!aligned(slots, 8)) return SPECMOE_ERR_ALIGN;

  Params p;
  p.ctx_lens = ctx_lens;
  p.chunk_lens = chunk_lens;
  p.table = block_table;
  p.held = held;
  p.free_pages = free_pages;
  p.free_count = free_count;
  p.missing = missing;
  p.slots = slots;
  p.B = desc->B;
  p.C_max = desc->C_max;
  p.page_shift = __builtin_ctz((unsigned)desc->page_size);
  p.pages_per_seq = desc->pages_per_seq;
  p.num_pages = desc->num_pages;

  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool own = slots && (int64_t)desc->B * desc->C_max <= kOwnSlots;
  (void)hipGetLastError();
  hipLaunchKernelGGL(assign_kernel, dim3(1), dim3(kThreads), 0, s, p, own ? 1 : 0);
  if (slots && !own)
    hipLaunchKernelGGL(slots_kernel, dim3((unsigned)(((int64_t)desc->C_max + kSlotThreads - 1) / kSlotThreads), desc->B),
                       dim3(kSlotThreads), 0, s, p);
  return hipGetLastError() == hipSuccess ? SPECMOE_OK : SPECMOE_ERR_LAUNCH;
}
