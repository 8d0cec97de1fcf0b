// Chunked verification attention for MI355X (gfx950, CDNA4): the entry points of
// specmoe_verify.h but for specmoe_verify_attn_scored.  The kernel is in
// verify_kernel.h.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <mutex>

#include "specmoe_verify.h"
#include "verify_kernel.h"

// Device scratch of specmoe_verify_attn_noalloc (for callers that cannot
// allocate): the workspace layout of a normal call (header, arrival
// counters, partial results) in one file-scope array per GPU, held until the
// process ends.  Host code never passes the array's name to a kernel (on the
// host it is only a stand-in for the symbol): it uses the device address
// that hipGetSymbolAddress returns for the current device.
constexpr size_t kScratchBytes = (size_t)48 << 20;
static __device__ __attribute__((aligned(256))) char scratch[kScratchBytes];

namespace {

// Zero the per-unit counters of a workspace.
__global__ void zero_counters_kernel(int* counters, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) counters[i] = 0;
}

// Host checks and launch of both entry points; draft_mask is NULL for a
// chain draft.
int run(const void* q, const void* k_cache, const void* v_cache, const int32_t* ctx_lens,
        const int32_t* chunk_lens, const uint64_t* draft_mask, bool tree, float scale, float* out, float* lse,
        void* stream, const specmoe_verify_desc* desc, const int32_t* block_table = nullptr,
        const specmoe_paged_kv* paged = nullptr, bool clear_counters = false) {
  int st = validate_call(desc, tree, paged);
  if (st != SPECMOE_OK) return st;
  if (desc->B == 0) return SPECMOE_OK;   // nothing to read or write
  Params p;
  Plan pl;
  st = make_params(q, k_cache, v_cache, ctx_lens, chunk_lens, draft_mask, tree, scale, out, lse, desc, block_table,
                   paged, p, pl);
  if (st != SPECMOE_OK) return st;

  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();  // clear a stale error from unrelated work
  if (clear_counters) {
    // the arrival counters of the units of one launch (at most kMaxSeqs
    // sequences), zeroed by a small kernel ahead of the main one
    const int n = (desc->B < kMaxSeqs ? desc->B : kMaxSeqs) * desc->Hkv;
    hipLaunchKernelGGL(zero_counters_kernel, dim3((n + 255) / 256), dim3(256), 0, s, p.counters, n);
  }
  launch_for<false>(desc->dtype, desc->D, tree, paged != nullptr, p, pl, s);
  if (hipGetLastError() != hipSuccess) return SPECMOE_ERR_LAUNCH;
  return SPECMOE_OK;
}

// Device address of `scratch` on the current device, looked up once per
// device (with that device current) and kept.
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

int scratch_for_current_device(void** ptr_out) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return SPECMOE_ERR_LAUNCH;
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* ptr = nullptr;
    if (hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)) != hipSuccess || ptr == nullptr) return SPECMOE_ERR_LAUNCH;
    g_scratch_ptr[dev] = ptr;
  }
  *ptr_out = g_scratch_ptr[dev];
  return SPECMOE_OK;
}

}  // namespace

extern "C" {

size_t specmoe_verify_attn_workspace_bytes(const specmoe_verify_desc* desc) {
  if (validate_desc(desc) != SPECMOE_OK) return 0;
  return make_plan(desc).ws_bytes;
}

int specmoe_verify_attn_workspace_init(void* workspace, size_t workspace_bytes, void* stream,
                                       const specmoe_verify_desc* desc) {
  const int st = validate_desc(desc);
  if (st != SPECMOE_OK) return st;
  if (!workspace) return SPECMOE_ERR_NULL_POINTER;
  if (!aligned16(workspace)) return SPECMOE_ERR_ALIGN;
  const Plan pl = make_plan(desc);
  if (workspace_bytes < pl.ws_bytes) return SPECMOE_ERR_WORKSPACE;
  const int n = (int)(pl.zero_bytes / sizeof(int));
  (void)hipGetLastError();
  hipLaunchKernelGGL(zero_counters_kernel, dim3((n + 255) / 256), dim3(256), 0, static_cast<hipStream_t>(stream),
                     static_cast<int*>(workspace), n);
  return hipGetLastError() == hipSuccess ? SPECMOE_OK : SPECMOE_ERR_LAUNCH;
}

int specmoe_verify_attn_status(const void* workspace, size_t workspace_bytes, void* stream) {
  if (!workspace && workspace_bytes == 0) {   // the current device's static scratch
    void* ptr = nullptr;
    const int st = scratch_for_current_device(&ptr);
    if (st != SPECMOE_OK) return st;
    workspace = ptr;
    workspace_bytes = kScratchBytes;
  }
  if (!workspace) return SPECMOE_ERR_NULL_POINTER;
  if (!aligned16(workspace)) return SPECMOE_ERR_ALIGN;
  if (workspace_bytes < kHeaderBytes) return SPECMOE_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  int word = 0;
  (void)hipGetLastError();
  if (hipMemcpyAsync(&word, workspace, sizeof(word), hipMemcpyDeviceToHost, s) != hipSuccess)
    return SPECMOE_ERR_LAUNCH;
  if (hipStreamSynchronize(s) != hipSuccess) return SPECMOE_ERR_LAUNCH;
  return (word & kGaveUp) ? SPECMOE_ERR_HANDOFF : SPECMOE_OK;
}

int32_t specmoe_verify_attn_key_tile(const specmoe_verify_desc* desc) {
  if (!desc) return SPECMOE_ERR_NULL_POINTER;
  if (!known_dtype(desc->dtype)) return SPECMOE_ERR_DTYPE;
  if (desc->D != 64 && desc->D != 128) return SPECMOE_ERR_HEAD_DIM;
  return key_tile(desc->dtype, desc->D);
}

const char* specmoe_status_str(int status) {
  switch (status) {
    case SPECMOE_OK: return "ok";
    case SPECMOE_ERR_NULL_POINTER: return "null pointer argument";
    case SPECMOE_ERR_SHAPE: return "invalid shape (B, Hq, Hkv, C_max, S_max) or sizes too large";
    case SPECMOE_ERR_GQA: return "Hq is not a multiple of Hkv";
    case SPECMOE_ERR_HEAD_DIM: return "unsupported head dimension (must be 64 or 128)";
    case SPECMOE_ERR_DTYPE: return "unsupported dtype";
    case SPECMOE_ERR_ROWS: return "C_max * (Hq / Hkv) exceeds 128 query rows per KV head";
    case SPECMOE_ERR_GRID: return "grid_blocks must be 0 (default) or in [1, 2048], with partial results under 2 GB";
    case SPECMOE_ERR_FLAGS: return "flags may only hold SPECMOE_FLAG_NO_WAIT";
    case SPECMOE_ERR_WORKSPACE: return "workspace too small";
    case SPECMOE_ERR_ALIGN: return "q, k_cache, v_cache, out and workspace must be 16-byte aligned";
    case SPECMOE_ERR_SCALE: return "scale must be finite and positive";
    case SPECMOE_ERR_LAUNCH: return "HIP kernel launch failed";
    case SPECMOE_ERR_MASK: return "draft masks hold at most 64 draft tokens: C_max must be <= 64";
    case SPECMOE_ERR_HANDOFF: return "an in-kernel wait for another wave gave up: results of a call are unspecified";
    case SPECMOE_ERR_ROPE: return "rot_dim must be a multiple of 16 in [0, D], rope_style and norm_eps valid";
    case SPECMOE_ERR_SCORE: return "softcap and scale / softcap must be finite, softcap and window not negative";
    case SPECMOE_ERR_PAGES:
      return "page_size must be a power of two in [8, 65536], pages_per_seq and num_pages positive, "
             "S_max = page_size * pages_per_seq";
    default: return "unknown status";
  }
}

int specmoe_verify_attn(const void* q, const void* k_cache, const void* v_cache, const int32_t* ctx_lens,
                        const int32_t* chunk_lens, float scale, float* out, float* lse, void* stream,
                        const specmoe_verify_desc* desc) {
  return run(q, k_cache, v_cache, ctx_lens, chunk_lens, nullptr, false, scale, out, lse, stream, desc);
}

int specmoe_verify_attn_noalloc(const void* q, const void* k_cache, const void* v_cache, const int32_t* ctx_lens,
                                const int32_t* chunk_lens, float scale, float* out, float* lse, void* stream,
                                const specmoe_verify_desc* desc) {
  const int st = validate_desc(desc);
  if (st != SPECMOE_OK) return st;
  if (make_plan(desc).ws_bytes > kScratchBytes) return SPECMOE_ERR_WORKSPACE;
  if (desc->B == 0) return SPECMOE_OK;
  void* ws = nullptr;
  const int ss = scratch_for_current_device(&ws);
  if (ss != SPECMOE_OK) return ss;
  specmoe_verify_desc d = *desc;
  d.workspace = ws;
  d.workspace_bytes = kScratchBytes;
  return run(q, k_cache, v_cache, ctx_lens, chunk_lens, nullptr, false, scale, out, lse, stream, &d, nullptr, nullptr,
             true);
}

int specmoe_verify_attn_tree(const void* q, const void* k_cache, const void* v_cache, const int32_t* ctx_lens,
                             const int32_t* chunk_lens, const uint64_t* draft_mask, float scale, float* out,
                             float* lse, void* stream, const specmoe_verify_desc* desc) {
  return run(q, k_cache, v_cache, ctx_lens, chunk_lens, draft_mask, true, scale, out, lse, stream, desc);
}

int specmoe_verify_attn_paged(const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                              const int32_t* ctx_lens, const int32_t* chunk_lens, const uint64_t* draft_mask,
                              float scale, float* out, float* lse, void* stream, const specmoe_verify_desc* desc,
                              const specmoe_paged_kv* paged) {
  if (!paged) return SPECMOE_ERR_NULL_POINTER;
  return run(q, k_pages, v_pages, ctx_lens, chunk_lens, draft_mask, draft_mask != nullptr, scale, out, lse, stream,
             desc, block_table, paged);
}

}  // extern "C"
