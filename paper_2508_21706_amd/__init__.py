"""Chunked verification attention (SpecMoEOff's verify step) for MI355X.

``verify_attn`` (chain drafts), ``verify_attn_tree`` (tree drafts),
``verify_attn_paged`` (a paged KV cache), ``verify_attn_scored`` (capped,
biased or windowed scores) and ``accept_greedy`` (the acceptance step after verification), ``append_kv``
(the chunk's rotation and KV append before it), ``sample`` and
``accept_sample`` (tokens and acceptance from given random numbers), and for a
KV cache held in 4 bits ``append_kv4``, ``verify_attn_kv4``, ``read_kv4`` and
``compact_accepted_kv4``, with ``assign_pages`` for the pages, run the HIP kernels
of ``libspecmoe_verify.so`` through its C-ABI; ``workloads`` draws
the seeded synthetic inputs.
"""
from .binding import (AcceptDesc, Desc, KV4Cache, PageState, SpecMoEError, accept_desc, accept_greedy, accept_greedy_tree,  # noqa: F401
                      accept_sample, accept_sample_tree, alloc_scored_workspace, append_kv,
                      compact_accepted_kv, sample,
                      alloc_accept_workspace, alloc_workspace, desc_for, key_tile, load_library, make_desc,
                      status_str, verify_attn, verify_attn_noalloc, verify_attn_paged, verify_attn_scored, verify_attn_tree,
                      workspace_bytes,
                      workspace_status,
                      alloc_kv4_cache, alloc_kv4_workspace, alloc_page_state, append_kv4, assign_pages,
                      compact_accepted_kv4, read_kv4, verify_attn_kv4)
from . import binding  # noqa: F401
