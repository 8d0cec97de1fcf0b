"""Thin Python binding of the chunked verification-attention C-ABI.

Argument marshalling only: every step of the computation runs in the HIP
kernels of ``libspecmoe_verify.so``; PyTorch supplies device memory and the
stream.  There is no fallback path: if the shared library is missing, every
entry point raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

LIB_NAME = "libspecmoe_verify.so"
LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), LIB_NAME)

SPECMOE_F32 = 0
SPECMOE_BF16 = 1
SPECMOE_F16 = 2

STATUS = {
    0: "SPECMOE_OK", -1: "SPECMOE_ERR_NULL_POINTER", -2: "SPECMOE_ERR_SHAPE", -3: "SPECMOE_ERR_GQA",
    -4: "SPECMOE_ERR_HEAD_DIM", -5: "SPECMOE_ERR_DTYPE", -6: "SPECMOE_ERR_ROWS", -7: "SPECMOE_ERR_GRID",
    -8: "SPECMOE_ERR_WORKSPACE", -9: "SPECMOE_ERR_ALIGN", -10: "SPECMOE_ERR_SCALE", -11: "SPECMOE_ERR_LAUNCH",
    -12: "SPECMOE_ERR_FLAGS", -13: "SPECMOE_ERR_MASK", -14: "SPECMOE_ERR_PAGES", -15: "SPECMOE_ERR_HANDOFF",
    -16: "SPECMOE_ERR_ROPE", -17: "SPECMOE_ERR_SCORE",
}
ROPE_STYLES = {"halves": 0, "pairs": 1}   # specmoe_rope_style
SPECMOE_FLAG_NO_WAIT = 1


class Desc(ctypes.Structure):
    """Mirror of ``specmoe_verify_desc``."""
    _fields_ = [
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
        ("C_max", ctypes.c_int32), ("S_max", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("grid_blocks", ctypes.c_int32), ("flags", ctypes.c_int32),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class AcceptDesc(ctypes.Structure):
    """Mirror of ``specmoe_accept_desc``."""
    _fields_ = [
        ("B", ctypes.c_int32), ("C_max", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("split", ctypes.c_int32), ("flags", ctypes.c_int32),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class PagedKV(ctypes.Structure):
    """Mirror of ``specmoe_paged_kv``."""
    _fields_ = [("page_size", ctypes.c_int32), ("pages_per_seq", ctypes.c_int32), ("num_pages", ctypes.c_int32)]


class AppendDesc(ctypes.Structure):
    """Mirror of ``specmoe_append_desc``."""
    _fields_ = [
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
        ("C_max", ctypes.c_int32), ("S_max", ctypes.c_int32), ("dtype", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
        ("rope_style", ctypes.c_int32), ("norm_eps", ctypes.c_float),
        ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
    ]


class Score(ctypes.Structure):
    """Mirror of ``specmoe_score``."""
    _fields_ = [("softcap", ctypes.c_float), ("window", ctypes.c_int32), ("slopes", ctypes.c_void_p),
                ("starts", ctypes.c_void_p)]


class SampleDesc(ctypes.Structure):
    """Mirror of ``specmoe_sample_desc``."""
    _fields_ = [("N", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("stride", ctypes.c_int64)]


class Sampling(ctypes.Structure):
    """Mirror of ``specmoe_sampling``."""
    _fields_ = [("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("min_p", ctypes.c_void_p)]


class SpecMoEError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"{STATUS.get(status, status)}: {text}")
        self.status = status


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load the HIP library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(
            f"{p} is missing: build the HIP library first (python paper_2508_21706_amd/build.py)")
    lib = ctypes.CDLL(p)
    lib.specmoe_verify_attn.restype = ctypes.c_int
    lib.specmoe_verify_attn.argtypes = [
        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
        ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(Desc)]
    lib.specmoe_verify_attn_noalloc.restype = ctypes.c_int
    lib.specmoe_verify_attn_noalloc.argtypes = lib.specmoe_verify_attn.argtypes
    lib.specmoe_verify_attn_tree.restype = ctypes.c_int
    lib.specmoe_verify_attn_tree.argtypes = [
        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
        ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(Desc)]
    lib.specmoe_verify_attn_paged.restype = ctypes.c_int
    lib.specmoe_verify_attn_paged.argtypes = [ctypes.c_void_p] * 7 + [
        ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(Desc), ctypes.POINTER(PagedKV)]
    lib.specmoe_verify_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.specmoe_verify_attn_workspace_bytes.argtypes = [ctypes.POINTER(Desc)]
    lib.specmoe_verify_attn_workspace_init.restype = ctypes.c_int
    lib.specmoe_verify_attn_workspace_init.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                                       ctypes.POINTER(Desc)]
    lib.specmoe_verify_attn_status.restype = ctypes.c_int
    lib.specmoe_verify_attn_status.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    lib.specmoe_verify_attn_key_tile.restype = ctypes.c_int32
    lib.specmoe_verify_attn_key_tile.argtypes = [ctypes.POINTER(Desc)]
    lib.specmoe_accept_greedy.restype = ctypes.c_int
    lib.specmoe_accept_greedy.argtypes = [ctypes.c_void_p] * 9 + [ctypes.POINTER(AcceptDesc)]
    lib.specmoe_accept_greedy_tree.restype = ctypes.c_int
    lib.specmoe_accept_greedy_tree.argtypes = [ctypes.c_void_p] * 11 + [ctypes.POINTER(AcceptDesc)]
    lib.specmoe_compact_accepted_kv.restype = ctypes.c_int
    lib.specmoe_compact_accepted_kv.argtypes = [ctypes.c_void_p] * 5 + [ctypes.POINTER(Desc)]
    lib.specmoe_accept_workspace_bytes.restype = ctypes.c_size_t
    lib.specmoe_accept_workspace_bytes.argtypes = [ctypes.POINTER(AcceptDesc)]
    lib.specmoe_accept_workspace_init.restype = ctypes.c_int
    lib.specmoe_accept_workspace_init.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                                  ctypes.POINTER(AcceptDesc)]
    lib.specmoe_verify_attn_scored.restype = ctypes.c_int
    lib.specmoe_verify_attn_scored.argtypes = [ctypes.c_void_p] * 7 + [
        ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(Desc),
        ctypes.POINTER(PagedKV), ctypes.POINTER(Score)]
    lib.specmoe_append_kv.restype = ctypes.c_int
    lib.specmoe_append_kv.argtypes = [ctypes.c_void_p] * 14 + [ctypes.POINTER(AppendDesc), ctypes.POINTER(PagedKV)]
    lib.specmoe_sample.restype = ctypes.c_int
    lib.specmoe_sample.argtypes = [ctypes.c_void_p] * 2 + [ctypes.POINTER(Sampling)] + [ctypes.c_void_p] * 3 + [
        ctypes.POINTER(SampleDesc)]
    lib.specmoe_accept_sample.restype = ctypes.c_int
    lib.specmoe_accept_sample.argtypes = [ctypes.c_void_p] * 5 + [ctypes.POINTER(Sampling)] + [ctypes.c_void_p] * 6 + [
        ctypes.POINTER(AcceptDesc)]
    lib.specmoe_accept_sample_tree.restype = ctypes.c_int
    lib.specmoe_accept_sample_tree.argtypes = [ctypes.c_void_p] * 6 + [ctypes.POINTER(Sampling)] + [
        ctypes.c_void_p] * 7 + [ctypes.POINTER(AcceptDesc)]
    lib.specmoe_status_str.restype = ctypes.c_char_p
    lib.specmoe_status_str.argtypes = [ctypes.c_int]
    if path is None:
        _lib = lib
    return lib


def status_str(status: int) -> str:
    return load_library().specmoe_status_str(status).decode()


def make_desc(B, Hq, Hkv, D, C_max, S_max, dtype: int, grid_blocks: int = 0, flags: int = 0,
              workspace: Optional[torch.Tensor] = None) -> Desc:
    d = Desc(B, Hq, Hkv, D, C_max, S_max, dtype, grid_blocks, flags, None, 0)
    if workspace is not None:
        d.workspace = workspace.data_ptr()
        d.workspace_bytes = workspace.numel() * workspace.element_size()
    return d


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return SPECMOE_BF16
    if t.dtype == torch.float16:
        return SPECMOE_F16
    if t.dtype == torch.float32:
        return SPECMOE_F32
    raise TypeError(f"unsupported dtype {t.dtype}; expected torch.bfloat16, torch.float16 or torch.float32")


def desc_for(q: torch.Tensor, k_cache: torch.Tensor, grid_blocks: int = 0) -> Desc:
    B, C_max, Hq, D = q.shape
    _, Hkv, S_max, _ = k_cache.shape
    return make_desc(B, Hq, Hkv, D, C_max, S_max, _dtype_code(q), grid_blocks)


def workspace_bytes(desc: Desc) -> int:
    return int(load_library().specmoe_verify_attn_workspace_bytes(ctypes.byref(desc)))


def key_tile(desc: Desc) -> int:
    return int(load_library().specmoe_verify_attn_key_tile(ctypes.byref(desc)))


_current_gpu = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _status_on(gpu: int, call, *args) -> int:
    """The status of a library call made with GPU ``gpu`` (a tensor's get_device())
    current: handle 0 is the null stream of the current GPU, whichever that is."""
    if gpu == _current_gpu():
        return call(*args)
    with torch.cuda.device(gpu):
        return call(*args)


def _launch(gpu: int, call, *args):
    """A library call with GPU ``gpu`` current; raises on an error status."""
    st = _status_on(gpu, call, *args)
    if st != 0:
        raise SpecMoEError(st, status_str(st))


def _use_workspace(desc, workspace: torch.Tensor, gpu: int):
    """Put ``workspace`` into ``desc``; the kernels write it, so it has to be
    memory of GPU ``gpu``."""
    if workspace.get_device() != gpu or gpu < 0:
        raise ValueError(f"workspace is on {workspace.device}, expected cuda:{gpu}")
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    desc.workspace = workspace.data_ptr()
    desc.workspace_bytes = workspace.nbytes


def alloc_workspace(desc: Desc, device, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Allocate a workspace for ``desc`` and zero its status word and counters
    on the stream.  The memory comes from the stream's own pool of the caching
    allocator, so that when the tensor is dropped, the block is only reused by
    work ordered after what was enqueued on that stream."""
    n = workspace_bytes(desc)
    if n == 0:
        raise SpecMoEError(-2, "invalid descriptor")
    s = stream if stream is not None else torch.cuda.current_stream(device)
    with torch.cuda.stream(s):
        ws = torch.empty(n, dtype=torch.uint8, device=device)
    _launch(ws.get_device(), load_library().specmoe_verify_attn_workspace_init, ws.data_ptr(), n, s.cuda_stream,
            ctypes.byref(desc))
    return ws


def workspace_status(workspace: Optional[torch.Tensor], stream: Optional[torch.cuda.Stream] = None) -> int:
    """``specmoe_verify_attn_status``: synchronises with the stream and returns
    0 (SPECMOE_OK) or -15 (SPECMOE_ERR_HANDOFF: an in-kernel wait gave up in a
    call since the workspace was initialised).  ``workspace=None``: the
    current device's static scratch of ``verify_attn_noalloc``."""
    if workspace is None:
        s = stream if stream is not None else torch.cuda.current_stream()
        st = load_library().specmoe_verify_attn_status(None, 0, s.cuda_stream)
    else:
        if not workspace.is_cuda:
            raise ValueError(f"workspace is on {workspace.device}, expected a GPU")
        s = stream if stream is not None else torch.cuda.current_stream(workspace.device)
        st = _status_on(workspace.get_device(), load_library().specmoe_verify_attn_status, workspace.data_ptr(),
                        workspace.numel() * workspace.element_size(), s.cuda_stream)
    if st not in (0, -15):
        raise SpecMoEError(st, status_str(st))
    return st


# The raw handle of a device's current stream, without the Stream object that
# torch.cuda.current_stream builds (1.3 us a call).
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _raw_stream(t: torch.Tensor, stream: Optional[torch.cuda.Stream]) -> int:
    """Handle of ``stream``, or of the current stream of ``t``'s GPU."""
    if stream is not None:
        return stream.cuda_stream
    if _current_raw_stream is not None:
        return _current_raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _empty(shape, dtype, device, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """An output buffer from the launch stream's pool."""
    if stream is None:   # the current stream's, as it is
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _check(t: torch.Tensor, name: str, shape, dtype):
    # the common case in one expression: a call checks up to nine tensors
    if t.is_cuda and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def verify_attn(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                ctx_lens: torch.Tensor, chunk_lens: torch.Tensor, scale: float,
                out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, grid_blocks: int = 0,
                stream: Optional[torch.cuda.Stream] = None, flags: int = 0,
                check_lengths: bool = False):
    """Chunked verification attention; see ``include/specmoe_verify.h``.

    q [B, C_max, Hq, D], k_cache / v_cache [B, Hkv, S_max, D] (bf16, f16 or f32),
    ctx_lens / chunk_lens int32 [B], all on the GPU.  Returns (out, lse) as
    float32 [B, C_max, Hq, D] and [B, C_max, Hq].  ``workspace`` (from
    ``alloc_workspace``) is reused across calls; without one, a fresh
    workspace is allocated and zeroed.  ``check_lengths`` copies the
    lengths to the host (a synchronisation) and checks the kernel's
    preconditions; off by default.  Repeated calls with the same inputs and
    grid give bitwise-identical results.
    """
    return _call(q, k_cache, v_cache, ctx_lens, chunk_lens, None, scale, out, lse, workspace, grid_blocks,
                 stream, flags, check_lengths)


def verify_attn_noalloc(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                        ctx_lens: torch.Tensor, chunk_lens: torch.Tensor, scale: float,
                        out: torch.Tensor, lse: torch.Tensor, grid_blocks: int = 0,
                        stream: Optional[torch.cuda.Stream] = None):
    """``specmoe_verify_attn_noalloc``: chain drafts like ``verify_attn``,
    with the library's static per-GPU scratch instead of a workspace.  The
    caller passes ``out`` and ``lse``; nothing is allocated.  Calls that may
    overlap on one GPU race (they share the scratch)."""
    lib = load_library()
    B, C_max, Hq, D = q.shape
    if k_cache.dim() != 4:
        raise ValueError("k_cache must be [B, Hkv, S_max, D]")
    _, Hkv, S_max, _ = k_cache.shape
    dt = q.dtype
    _check(q, "q", (B, C_max, Hq, D), dt)
    _check(k_cache, "k_cache", (B, Hkv, S_max, D), dt)
    _check(v_cache, "v_cache", (B, Hkv, S_max, D), dt)
    _check(ctx_lens, "ctx_lens", (B,), torch.int32)
    _check(chunk_lens, "chunk_lens", (B,), torch.int32)
    _check(out, "out", (B, C_max, Hq, D), torch.float32)
    _check(lse, "lse", (B, C_max, Hq), torch.float32)
    desc = make_desc(B, Hq, Hkv, D, C_max, S_max, _dtype_code(q), grid_blocks)
    _launch(q.get_device(), lib.specmoe_verify_attn_noalloc, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
            ctx_lens.data_ptr(), chunk_lens.data_ptr(), float(scale), out.data_ptr(), lse.data_ptr(),
            _raw_stream(q, stream), ctypes.byref(desc))
    return out, lse


def verify_attn_tree(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     ctx_lens: torch.Tensor, chunk_lens: torch.Tensor, draft_mask: torch.Tensor, scale: float,
                     out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, grid_blocks: int = 0,
                     stream: Optional[torch.cuda.Stream] = None, flags: int = 0,
                     check_lengths: bool = False):
    """Chunked verification attention for tree drafts; see
    ``specmoe_verify_attn_tree`` in ``include/specmoe_verify.h``.

    Arguments as ``verify_attn``, plus ``draft_mask``: int64 (or uint64)
    [B, C_max] on the GPU, the 64-bit draft-mask words (bit k of word
    [b, i] set: draft token i of sequence b attends to draft token k).
    C_max must be <= 64.
    """
    return _call(q, k_cache, v_cache, ctx_lens, chunk_lens, draft_mask, scale, out, lse, workspace,
                 grid_blocks, stream, flags, check_lengths)


def verify_attn_paged(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, block_table: torch.Tensor,
                      ctx_lens: torch.Tensor, chunk_lens: torch.Tensor, scale: float,
                      draft_mask: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, grid_blocks: int = 0,
                      stream: Optional[torch.cuda.Stream] = None, flags: int = 0,
                      check_lengths: bool = False):
    """Chunked verification attention over a paged KV cache; see
    ``specmoe_verify_attn_paged`` in ``include/specmoe_verify.h``.

    k_pages / v_pages [num_pages, Hkv, page_size, D], block_table int32
    [B, pages_per_seq] (S_max = page_size * pages_per_seq); the other
    arguments as ``verify_attn`` (``draft_mask``: tree drafts, as
    ``verify_attn_tree``).
    """
    if k_pages.dim() != 4:
        raise ValueError("k_pages must be [num_pages, Hkv, page_size, D]")
    num_pages, _, page_size, _ = k_pages.shape
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, pages_per_seq]")
    _check(block_table, "block_table", (q.shape[0], block_table.shape[1]), torch.int32)
    paged = PagedKV(page_size, block_table.shape[1], num_pages)
    return _call(q, k_pages, v_pages, ctx_lens, chunk_lens, draft_mask, scale, out, lse, workspace, grid_blocks,
                 stream, flags, check_lengths, paged=paged, block_table=block_table)


def _call(q, k_cache, v_cache, ctx_lens, chunk_lens, draft_mask, scale, out, lse, workspace, grid_blocks,
          stream, flags, check_lengths, paged: Optional[PagedKV] = None, block_table=None):
    lib = load_library()
    B, C_max, Hq, D = q.shape
    if k_cache.dim() != 4:
        raise ValueError("k_cache must be [B, Hkv, S_max, D]")
    dt = q.dtype
    _check(q, "q", (B, C_max, Hq, D), dt)
    if paged is None:
        _, Hkv, S_max, _ = k_cache.shape
        _check(k_cache, "k_cache", (B, Hkv, S_max, D), dt)
        _check(v_cache, "v_cache", (B, Hkv, S_max, D), dt)
    else:
        Hkv = k_cache.shape[1]
        S_max = paged.page_size * paged.pages_per_seq
        _check(k_cache, "k_pages", (paged.num_pages, Hkv, paged.page_size, D), dt)
        _check(v_cache, "v_pages", (paged.num_pages, Hkv, paged.page_size, D), dt)
    _check(ctx_lens, "ctx_lens", (B,), torch.int32)
    _check(chunk_lens, "chunk_lens", (B,), torch.int32)
    if draft_mask is not None:
        mdt = draft_mask.dtype if draft_mask.dtype in (torch.int64, torch.uint64) else torch.int64
        _check(draft_mask, "draft_mask", (B, C_max), mdt)
    if check_lengths:
        c = chunk_lens.cpu()
        l = ctx_lens.cpu()
        if (c < 0).any() or (c > C_max).any() or (l < 0).any() or (l + c > S_max).any():
            raise ValueError("lengths break 0 <= c_b <= C_max, l_b >= 0, l_b + c_b <= S_max")
    if out is None:
        out = _empty((B, C_max, Hq, D), torch.float32, q.device, stream)
    if lse is None:
        lse = _empty((B, C_max, Hq), torch.float32, q.device, stream)
    _check(out, "out", (B, C_max, Hq, D), torch.float32)
    _check(lse, "lse", (B, C_max, Hq), torch.float32)
    desc = make_desc(B, Hq, Hkv, D, C_max, S_max, _dtype_code(q), grid_blocks, flags)
    if B == 0:
        return out, lse
    if workspace is None:
        workspace = alloc_workspace(desc, q.device, stream)
    gpu, raw = q.get_device(), _raw_stream(q, stream)
    _use_workspace(desc, workspace, gpu)
    if paged is not None:
        _launch(gpu, lib.specmoe_verify_attn_paged, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                block_table.data_ptr(), ctx_lens.data_ptr(), chunk_lens.data_ptr(),
                draft_mask.data_ptr() if draft_mask is not None else None, float(scale), out.data_ptr(),
                lse.data_ptr(), raw, ctypes.byref(desc), ctypes.byref(paged))
    elif draft_mask is None:
        _launch(gpu, lib.specmoe_verify_attn, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                ctx_lens.data_ptr(), chunk_lens.data_ptr(), float(scale), out.data_ptr(), lse.data_ptr(), raw,
                ctypes.byref(desc))
    else:
        _launch(gpu, lib.specmoe_verify_attn_tree, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                ctx_lens.data_ptr(), chunk_lens.data_ptr(), draft_mask.data_ptr(), float(scale), out.data_ptr(),
                lse.data_ptr(), raw, ctypes.byref(desc))
    return out, lse


# ------------------------------------------------------------ acceptance step

def accept_desc(B, C_max, V, dtype: int, split: int = 0) -> AcceptDesc:
    return AcceptDesc(B, C_max, V, dtype, split, 0, None, 0)


def alloc_accept_workspace(desc: AcceptDesc, device, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Allocate a workspace for ``desc`` and zero its counters on the stream."""
    lib = load_library()
    n = int(lib.specmoe_accept_workspace_bytes(ctypes.byref(desc)))
    if n == 0:
        raise SpecMoEError(-2, "invalid acceptance descriptor")
    s = stream if stream is not None else torch.cuda.current_stream(device)
    with torch.cuda.stream(s):   # from the stream's pool (see alloc_workspace)
        ws = torch.empty(n, dtype=torch.uint8, device=device)
    _launch(ws.get_device(), lib.specmoe_accept_workspace_init, ws.data_ptr(), n, s.cuda_stream, ctypes.byref(desc))
    return ws


def accept_greedy_tree(logits: torch.Tensor, tokens: torch.Tensor, draft_mask: torch.Tensor, ctx_lens: torch.Tensor,
                       chunk_lens: torch.Tensor, out: Optional[dict] = None, workspace: Optional[torch.Tensor] = None,
                       split: int = 0, stream: Optional[torch.cuda.Stream] = None, in_place: bool = False):
    """Greedy acceptance of tree drafts; see ``specmoe_accept_greedy_tree``
    in ``include/specmoe_accept.h``.  As ``accept_greedy`` plus ``draft_mask``
    (int64 [B, C_max] root-path words, C_max <= 64); the result also holds
    ``path`` (int64 [B]: the accepted path's node bits).  Call
    ``compact_accepted_kv`` with the context lengths from before the step to
    move the path's K/V rows into place."""
    B, C_max = tokens.shape
    mdt = draft_mask.dtype if draft_mask.dtype in (torch.int64, torch.uint64) else torch.int64
    _check(draft_mask, "draft_mask", (B, C_max), mdt)
    if out is None:
        out = {}
    if "path" not in out:
        out["path"] = _empty((B,), torch.int64, logits.device, stream)
    _check(out["path"], "path", (B,), torch.int64)
    return accept_greedy(logits, tokens, ctx_lens, chunk_lens, out=out, workspace=workspace, split=split,
                         stream=stream, in_place=in_place, _tree=(draft_mask, out["path"]))


def compact_accepted_kv(k_cache: torch.Tensor, v_cache: torch.Tensor, ctx_lens: torch.Tensor, path: torch.Tensor,
                        stream: Optional[torch.cuda.Stream] = None):
    """Move each sequence's accepted tree path's K/V rows to the rows right
    after its context (``specmoe_compact_accepted_kv``); ``ctx_lens`` are the
    lengths from before the acceptance step."""
    lib = load_library()
    B, Hkv, S_max, D = k_cache.shape
    _check(k_cache, "k_cache", (B, Hkv, S_max, D), k_cache.dtype)
    _check(v_cache, "v_cache", (B, Hkv, S_max, D), k_cache.dtype)
    _check(ctx_lens, "ctx_lens", (B,), torch.int32)
    _check(path, "path", (B,), path.dtype if path.dtype in (torch.int64, torch.uint64) else torch.int64)
    desc = make_desc(B, Hkv, Hkv, D, 1, S_max, _dtype_code(k_cache))
    _launch(k_cache.get_device(), lib.specmoe_compact_accepted_kv, k_cache.data_ptr(), v_cache.data_ptr(),
            ctx_lens.data_ptr(), path.data_ptr(), _raw_stream(k_cache, stream), ctypes.byref(desc))


def accept_greedy(logits: torch.Tensor, tokens: torch.Tensor, ctx_lens: torch.Tensor, chunk_lens: torch.Tensor,
                  out: Optional[dict] = None, workspace: Optional[torch.Tensor] = None, split: int = 0,
                  stream: Optional[torch.cuda.Stream] = None, in_place: bool = False, _tree=None):
    """Greedy acceptance after verification; see ``include/specmoe_accept.h``.

    logits [B, C_max, V] (bf16 or f32), tokens int32 [B, C_max], ctx_lens /
    chunk_lens int32 [B], all on the GPU.  Returns a dict of int32 tensors:
    argmax [B, C_max], accepted [B], next_token [B], new_ctx_lens [B] (with
    ``in_place``, ctx_lens itself is updated and returned as new_ctx_lens).
    ``out`` may supply those tensors; missing ones come from the launch
    stream's pool, as in ``verify_attn``.
    """
    lib = load_library()
    if logits.dim() != 3:
        raise ValueError("logits must be [B, C_max, V]")
    B, C_max, V = logits.shape
    _check(logits, "logits", (B, C_max, V), logits.dtype)
    _check(tokens, "tokens", (B, C_max), torch.int32)
    _check(ctx_lens, "ctx_lens", (B,), torch.int32)
    _check(chunk_lens, "chunk_lens", (B,), torch.int32)
    dev = logits.device
    if out is None:
        out = {}
    for key in ("argmax", "accepted", "next_token", "new_ctx_lens"):
        if key not in out and not (in_place and key == "new_ctx_lens"):
            out[key] = _empty((B, C_max) if key == "argmax" else (B,), torch.int32, dev, stream)
    if in_place:
        out["new_ctx_lens"] = ctx_lens
    _check(out["argmax"], "argmax", (B, C_max), torch.int32)
    for k in ("accepted", "next_token", "new_ctx_lens"):
        _check(out[k], k, (B,), torch.int32)
    desc = accept_desc(B, C_max, V, _dtype_code(logits), split)
    if B == 0:
        return out
    if workspace is None:
        workspace = alloc_accept_workspace(desc, dev, stream)
    gpu, raw = logits.get_device(), _raw_stream(logits, stream)
    _use_workspace(desc, workspace, gpu)
    if _tree is None:
        _launch(gpu, lib.specmoe_accept_greedy, logits.data_ptr(), tokens.data_ptr(), ctx_lens.data_ptr(),
                chunk_lens.data_ptr(), out["argmax"].data_ptr(), out["accepted"].data_ptr(),
                out["next_token"].data_ptr(), out["new_ctx_lens"].data_ptr(), raw, ctypes.byref(desc))
    else:
        _launch(gpu, lib.specmoe_accept_greedy_tree, logits.data_ptr(), tokens.data_ptr(), _tree[0].data_ptr(),
                ctx_lens.data_ptr(), chunk_lens.data_ptr(), out["argmax"].data_ptr(), out["accepted"].data_ptr(),
                out["next_token"].data_ptr(), out["new_ctx_lens"].data_ptr(), _tree[1].data_ptr(), raw,
                ctypes.byref(desc))
    return out


# ------------------------------------------------------------- chunk append

def _check_on(t: torch.Tensor, name: str, shape, dtype, gpu: int):
    """``_check``, and that ``t`` is on GPU ``gpu`` (a tensor's get_device())."""
    # (one expression again: these calls check a dozen tensors)
    if t.dtype is dtype and t.get_device() == gpu and t.shape == shape and t.is_contiguous() and gpu >= 0:
        return
    _check(t, name, shape, dtype)
    raise ValueError(f"{name} is on {t.device}, expected cuda:{gpu}")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _token_stride(t: torch.Tensor, name: str, shape, dtype, gpu: int) -> int:
    """Elements from one token's row of ``t`` [B, C_max, H, D] to the next's;
    a row's heads lie side by side."""
    if t.shape != shape or t.dtype is not dtype:
        _check_on(t.contiguous(), name, shape, dtype, gpu)
    B, C, H, D = shape
    sb, sc, sh, sd = t.stride()
    if sc != H * D or sd != 1 or sh != D or sb != C * sc:
        # (one row for all tokens, as expand() makes, is at a distance of 0)
        if (D > 1 and sd != 1) or (H > 1 and sh != D) or (B > 1 and C > 1 and sb != C * sc) or \
                (C > 1 and sc == 0) or (B > 1 and sb == 0):
            raise ValueError(f"{name} must be rows of side-by-side heads at one distance from token to token")
        sc = sc if C > 1 else sb if B > 1 else H * D
    if gpu < 0 or t.get_device() != gpu:
        _check_on(t.contiguous(), name, shape, dtype, gpu)
    return sc


def append_kv(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor,
              v_cache: torch.Tensor, ctx_lens: torch.Tensor, chunk_lens: torch.Tensor,
              inv_freq: Optional[torch.Tensor] = None, rope: str = "halves",
              q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
              draft_mask: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None,
              q_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Norm and rotate a chunk's queries and keys and append its keys and
    values to the cache; see ``specmoe_append_kv`` in
    ``include/specmoe_append.h``.  The step before ``verify_attn``.

    q [B, C_max, Hq, D], k / v [B, C_max, Hkv, D] (bf16, f16 or f32), possibly
    views of one packed projection; k_cache / v_cache [B, Hkv, S_max, D], or
    with ``block_table`` the pages of ``verify_attn_paged``.  ``inv_freq``
    float64 [rot_dim / 2] (None: no rotation); ``rope`` "halves" or "pairs";
    ``q_weight`` / ``k_weight`` [D] (None: no norm); ``draft_mask`` as in
    ``verify_attn_tree``.  Returns ``q_out`` (allocated if None; rows past a
    chunk's end are left as they are).  ``q=None``: keys and values only,
    returns None.
    """
    lib = load_library()
    if k.dim() != 4 or k_cache.dim() != 4 or (q is not None and q.dim() != 4):
        raise ValueError("q, k, v, k_cache and v_cache have four dimensions")
    B, C_max, Hkv, D = k.shape
    dt, dev = k.dtype, k.get_device()
    if rope not in ROPE_STYLES:
        raise ValueError(f"rope must be one of {sorted(ROPE_STYLES)}, got {rope!r}")
    paged = None
    if block_table is None:
        S_max = k_cache.shape[2]
        shape = (B, Hkv, S_max, D)
    else:
        if block_table.dim() != 2:
            raise ValueError("block_table must be [B, pages_per_seq]")
        _check_on(block_table, "block_table", (B, block_table.shape[1]), torch.int32, dev)
        num_pages, _, page_size, _ = k_cache.shape
        paged = PagedKV(page_size, block_table.shape[1], num_pages)
        S_max = page_size * block_table.shape[1]
        shape = (num_pages, Hkv, page_size, D)
    _check_on(k_cache, "k_cache", shape, dt, dev)
    _check_on(v_cache, "v_cache", shape, dt, dev)
    _check_on(ctx_lens, "ctx_lens", (B,), torch.int32, dev)
    _check_on(chunk_lens, "chunk_lens", (B,), torch.int32, dev)
    Hq = 0 if q is None else q.shape[2]
    ks = _token_stride(k, "k", (B, C_max, Hkv, D), dt, dev)
    vs = _token_stride(v, "v", (B, C_max, Hkv, D), dt, dev)
    qs = 0
    if q is not None:
        qs = _token_stride(q, "q", (B, C_max, Hq, D), dt, dev)
        if q_out is None:
            q_out = _empty((B, C_max, Hq, D), dt, k.device, stream)
        else:
            _check_on(q_out, "q_out", (B, C_max, Hq, D), dt, dev)
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None:
            _check_on(w, name, (D,), dt, dev)
    rot_dim = 0
    if inv_freq is not None:
        _check_on(inv_freq, "inv_freq", (inv_freq.numel(),), torch.float64, dev)
        rot_dim = 2 * inv_freq.numel()
    if draft_mask is not None:
        mdt = draft_mask.dtype if draft_mask.dtype in (torch.int64, torch.uint64) else torch.int64
        _check_on(draft_mask, "draft_mask", (B, C_max), mdt, dev)
    desc = AppendDesc(B, Hq, Hkv, D, C_max, S_max, _dtype_code(k), rot_dim, ROPE_STYLES[rope], eps, qs, ks, vs)
    _launch(dev, lib.specmoe_append_kv, _ptr(q), k.data_ptr(), v.data_ptr(), _ptr(q_weight), _ptr(k_weight),
            _ptr(inv_freq), ctx_lens.data_ptr(), chunk_lens.data_ptr(), _ptr(draft_mask), _ptr(block_table),
            _ptr(q_out) if q is not None else None, k_cache.data_ptr(), v_cache.data_ptr(), _raw_stream(k, stream),
            ctypes.byref(desc), None if paged is None else ctypes.byref(paged))
    return q_out if q is not None else None


# --------------------------------------------------------- scored attention

def _scored_shape(q: torch.Tensor, k_cache: torch.Tensor, block_table: Optional[torch.Tensor]):
    """(Hkv, S_max, page geometry or None) of a contiguous or paged cache."""
    if q.dim() != 4 or k_cache.dim() != 4:
        raise ValueError("q must be [B, C_max, Hq, D], k_cache [B, Hkv, S_max, D] or [num_pages, Hkv, page_size, D]")
    if block_table is None:
        return k_cache.shape[1], k_cache.shape[2], None
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, pages_per_seq]")
    paged = PagedKV(k_cache.shape[2], block_table.shape[1], k_cache.shape[0])
    return k_cache.shape[1], paged.page_size * paged.pages_per_seq, paged


def alloc_scored_workspace(q: torch.Tensor, k_cache: torch.Tensor, block_table: Optional[torch.Tensor] = None,
                           grid_blocks: int = 0, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """A workspace for ``verify_attn_scored`` calls of these shapes (one of
    ``alloc_workspace``, which serves ``verify_attn`` too)."""
    B, C_max, Hq, D = q.shape
    Hkv, S_max, _ = _scored_shape(q, k_cache, block_table)
    return alloc_workspace(make_desc(B, Hq, Hkv, D, C_max, S_max, _dtype_code(q), grid_blocks), q.device, stream)


def verify_attn_scored(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, ctx_lens: torch.Tensor,
                       chunk_lens: torch.Tensor, scale: float, softcap: float = 0.0,
                       slopes: Optional[torch.Tensor] = None, window: int = 0,
                       starts: Optional[torch.Tensor] = None, draft_mask: Optional[torch.Tensor] = None,
                       block_table: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                       lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                       grid_blocks: int = 0, stream: Optional[torch.cuda.Stream] = None, flags: int = 0,
                       check_lengths: bool = False):
    """Verification attention with capped, biased or windowed scores; see
    ``specmoe_verify_attn_scored`` in ``include/specmoe_verify.h``.

    Arguments as ``verify_attn``, ``verify_attn_tree`` (``draft_mask``) and
    ``verify_attn_paged`` (``block_table``); ``softcap`` (0: off), ``window``
    in keys (0: off), ``slopes`` float32 [Hq] and ``starts`` int32 [B] on the
    GPU (None: off).  Returns (out, lse): ``out`` [B, C_max, Hq, D] in q's
    type, ``lse`` float32 [B, C_max, Hq].
    """
    lib = load_library()
    Hkv, S_max, paged = _scored_shape(q, k_cache, block_table)
    B, C_max, Hq, D = q.shape
    dt, dev = q.dtype, q.get_device()
    _check_on(q, "q", (B, C_max, Hq, D), dt, dev)
    cache = (B, Hkv, S_max, D) if paged is None else (paged.num_pages, Hkv, paged.page_size, D)
    _check_on(k_cache, "k_cache", cache, dt, dev)
    _check_on(v_cache, "v_cache", cache, dt, dev)
    _check_on(ctx_lens, "ctx_lens", (B,), torch.int32, dev)
    _check_on(chunk_lens, "chunk_lens", (B,), torch.int32, dev)
    if block_table is not None:
        _check_on(block_table, "block_table", (B, block_table.shape[1]), torch.int32, dev)
    if slopes is not None:
        _check_on(slopes, "slopes", (Hq,), torch.float32, dev)
    if starts is not None:
        _check_on(starts, "starts", (B,), torch.int32, dev)
    if draft_mask is not None:
        mdt = draft_mask.dtype if draft_mask.dtype in (torch.int64, torch.uint64) else torch.int64
        _check_on(draft_mask, "draft_mask", (B, C_max), mdt, dev)
    if check_lengths:
        c, l = chunk_lens.cpu(), ctx_lens.cpu()
        if (c < 0).any() or (c > C_max).any() or (l < 0).any() or (l + c > S_max).any():
            raise ValueError("lengths break 0 <= c_b <= C_max, l_b >= 0, l_b + c_b <= S_max")
    if out is None:
        out = _empty((B, C_max, Hq, D), dt, q.device, stream)
    if lse is None:
        lse = _empty((B, C_max, Hq), torch.float32, q.device, stream)
    _check_on(out, "out", (B, C_max, Hq, D), dt, dev)
    _check_on(lse, "lse", (B, C_max, Hq), torch.float32, dev)
    desc = make_desc(B, Hq, Hkv, D, C_max, S_max, _dtype_code(q), grid_blocks, flags)
    if B > 0:
        if workspace is None:
            workspace = alloc_workspace(desc, q.device, stream)
        _use_workspace(desc, workspace, dev)
    window = max(min(window, (1 << 31) - 1), -1)   # (the field has 32 bits, and so has a length)
    score = Score(softcap, window, _ptr(slopes), _ptr(starts))
    if softcap and not score.softcap:   # (0 in 32 bits, which would mean off)
        raise SpecMoEError(-17, status_str(-17))
    _launch(dev, lib.specmoe_verify_attn_scored, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
            _ptr(block_table), ctx_lens.data_ptr(), chunk_lens.data_ptr(), _ptr(draft_mask), float(scale),
            out.data_ptr(), lse.data_ptr(), _raw_stream(q, stream), ctypes.byref(desc),
            None if paged is None else ctypes.byref(paged), ctypes.byref(score))
    return out, lse


# ----------------------------------------------------------------- sampling

def _sampling(n: int, device, temperature, top_k, top_p, min_p) -> Sampling:
    for t, name, dt in ((temperature, "temperature", torch.float32), (top_k, "top_k", torch.int32),
                        (top_p, "top_p", torch.float32), (min_p, "min_p", torch.float32)):
        if t is not None:
            _check_on(t, name, (n,), dt, device)
    return Sampling(_ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p))


def sample(logits: torch.Tensor, uniforms: torch.Tensor, temperature: Optional[torch.Tensor] = None,
           top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
           min_p: Optional[torch.Tensor] = None, out=None, stream: Optional[torch.cuda.Stream] = None):
    """One token per row of logits from given random numbers; see
    ``specmoe_sample`` in ``include/specmoe_sample.h``.

    logits [N, V] (bf16 or f32; rows may lie apart), uniforms float32 [N] in
    [0, 1); the settings [N] (float32, top_k int32), None: off.  Returns
    (tokens int32 [N], logprobs float32 [N]); ``out`` may supply the pair.
    """
    lib = load_library()
    if logits.dim() != 2:
        raise ValueError("logits must be [N, V]")
    N, V = logits.shape
    dev = logits.get_device()
    if V > 1 and logits.stride(1) != 1:
        raise ValueError("the entries of a row of logits must lie side by side")
    stride = logits.stride(0) if N > 1 else V
    if stride == 0 and V > 0:   # (one row for all, as expand() makes: a stride of 0 is the library's word for V)
        raise ValueError("every row of logits must have memory of its own")
    if dev < 0:
        raise ValueError("logits must be a GPU tensor")
    _check_on(uniforms, "uniforms", (N,), torch.float32, dev)
    settings = _sampling(N, dev, temperature, top_k, top_p, min_p)
    if out is None:
        out = (_empty((N,), torch.int32, logits.device, stream), _empty((N,), torch.float32, logits.device, stream))
    _check_on(out[0], "tokens", (N,), torch.int32, dev)
    _check_on(out[1], "logprobs", (N,), torch.float32, dev)
    desc = SampleDesc(N, V, _dtype_code(logits), 0, stride)
    _launch(dev, lib.specmoe_sample, logits.data_ptr(), uniforms.data_ptr(), ctypes.byref(settings),
            out[0].data_ptr(), out[1].data_ptr(), _raw_stream(logits, stream), ctypes.byref(desc))
    return out[0], out[1]


def accept_sample(logits: torch.Tensor, tokens: torch.Tensor, ctx_lens: torch.Tensor, chunk_lens: torch.Tensor,
                  uniforms: torch.Tensor, temperature: Optional[torch.Tensor] = None,
                  top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
                  min_p: Optional[torch.Tensor] = None, out: Optional[dict] = None,
                  workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                  in_place: bool = False, _tree=None):
    """Acceptance of draft tokens by sampling; see ``specmoe_accept_sample`` in
    ``include/specmoe_sample.h``.

    As ``accept_greedy`` (whose workspace it takes), plus uniforms float32
    [B, C_max] and each sequence's settings [B] (None: off).  Returns a dict:
    sampled int32 [B, C_max], logprobs float32 [B, C_max], accepted,
    next_token and new_ctx_lens int32 [B].
    """
    lib = load_library()
    if logits.dim() != 3:
        raise ValueError("logits must be [B, C_max, V]")
    B, C_max, V = logits.shape
    dev = logits.get_device()
    _check_on(logits, "logits", (B, C_max, V), logits.dtype, dev)
    _check_on(tokens, "tokens", (B, C_max), torch.int32, dev)
    _check_on(ctx_lens, "ctx_lens", (B,), torch.int32, dev)
    _check_on(chunk_lens, "chunk_lens", (B,), torch.int32, dev)
    _check_on(uniforms, "uniforms", (B, C_max), torch.float32, dev)
    settings = _sampling(B, dev, temperature, top_k, top_p, min_p)
    out = {} if out is None else out
    if in_place:
        out["new_ctx_lens"] = ctx_lens
    kinds = {"sampled": ((B, C_max), torch.int32), "logprobs": ((B, C_max), torch.float32),
             "accepted": ((B,), torch.int32), "next_token": ((B,), torch.int32), "new_ctx_lens": ((B,), torch.int32)}
    if _tree is not None:
        kinds["path"] = ((B,), torch.int64)
    for key, (shape, dt) in kinds.items():
        if key not in out:
            out[key] = _empty(shape, dt, logits.device, stream)
        _check_on(out[key], key, shape, dt, dev)
    desc = accept_desc(B, C_max, V, _dtype_code(logits))
    if B == 0:
        return out
    if workspace is None:
        workspace = alloc_accept_workspace(desc, logits.device, stream)
    _use_workspace(desc, workspace, dev)
    head = (logits.data_ptr(), tokens.data_ptr())
    lens = (ctx_lens.data_ptr(), chunk_lens.data_ptr(), uniforms.data_ptr(), ctypes.byref(settings),
            out["sampled"].data_ptr(), out["logprobs"].data_ptr(), out["accepted"].data_ptr(),
            out["next_token"].data_ptr(), out["new_ctx_lens"].data_ptr())
    tail = (_raw_stream(logits, stream), ctypes.byref(desc))
    if _tree is None:
        _launch(dev, lib.specmoe_accept_sample, *head, *lens, *tail)
    else:
        _launch(dev, lib.specmoe_accept_sample_tree, *head, _tree.data_ptr(), *lens, out["path"].data_ptr(), *tail)
    return out


def accept_sample_tree(logits: torch.Tensor, tokens: torch.Tensor, draft_mask: torch.Tensor, ctx_lens: torch.Tensor,
                       chunk_lens: torch.Tensor, uniforms: torch.Tensor, temperature: Optional[torch.Tensor] = None,
                       top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
                       min_p: Optional[torch.Tensor] = None, out: Optional[dict] = None,
                       workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                       in_place: bool = False):
    """Acceptance of tree drafts by sampling; see ``specmoe_accept_sample_tree``
    in ``include/specmoe_sample.h``.  As ``accept_sample`` plus ``draft_mask``
    (int64 [B, C_max] root-path words, C_max <= 64); the result also holds
    ``path`` (int64 [B]) for ``compact_accepted_kv``."""
    mdt = draft_mask.dtype if draft_mask.dtype in (torch.int64, torch.uint64) else torch.int64
    _check_on(draft_mask, "draft_mask", tuple(tokens.shape), mdt, logits.get_device())
    return accept_sample(logits, tokens, ctx_lens, chunk_lens, uniforms, temperature, top_k, top_p, min_p, out=out,
                         workspace=workspace, stream=stream, in_place=in_place, _tree=draft_mask)
