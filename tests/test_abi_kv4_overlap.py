"""verify_attn_kv4 refuses results that share memory with the queries or with each other,
at the C entry point (before any HIP call) and in the binding."""
import pytest
import torch

import paper_2508_21706_amd as pkg
from paper_2508_21706_amd import binding as bd
from test_abi_kv4 import attn, attn_desc, lib  # noqa: F401

Q = 1 << 24
BYTES = 2 * 5 * 32 * 128 * 2   # q and out of attn_desc()
LSE = 2 * 5 * 32 * 4


@pytest.mark.parametrize("out,lse", [
    (Q, 2 * Q), (Q + 16, 2 * Q), (Q - 16, 2 * Q), (Q + BYTES - 16, 2 * Q), (Q - BYTES + 16, 2 * Q),
    (2 * Q, Q), (2 * Q, Q + BYTES - 4), (2 * Q, Q - LSE + 4),
    (2 * Q, 2 * Q), (2 * Q, 2 * Q + BYTES - 4), (2 * Q, 2 * Q - LSE + 4),
])
def test_shared_memory_is_refused(lib, out, lse):  # noqa: F811
    assert attn(lib, attn_desc(), q=Q, out=out, lse=lse) == -18
    assert attn(lib, attn_desc(), bd.PagedKV(16, 144, 9), q=Q, out=out, lse=lse) == -18
    assert attn(lib, attn_desc(), q=Q, out=out, lse=lse, scale=0.0) == -10      # (the last of the checks)
    assert attn(lib, attn_desc(B=0), q=Q, out=out, lse=lse) == 0


@pytest.mark.gpu
def test_neighbouring_memory_is_taken():
    """q, out and lse one behind the other in one buffer; a row's shift is refused."""
    from test_gpu_kv4_attn import call, make, on_gpu
    from test_gpu_parity import dev

    x = make(24, "f32", [40, 7], [2, 2], C=2)
    ref = call(x)
    cache, _ = on_gpu(x)
    B, C, Hq, D = x["q"].shape
    n = x["q"].numel()
    flat = torch.zeros(2 * n + B * C * Hq, device=dev())
    q, out, lse = flat[:n].view_as(x["q"]), flat[n:2 * n].view_as(x["q"]), flat[2 * n:].view(B, C, Hq)
    q.copy_(x["q"])
    lens = [torch.tensor(a, dtype=torch.int32, device=dev()) for a in (x["ctx"], x["chunk"])]
    pkg.verify_attn_kv4(q, cache, *lens, x["scale"], out=out, lse=lse)
    torch.cuda.synchronize()
    assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
    for shift in (4, D, n - 4):
        for other in (flat[shift:shift + n].view_as(q), flat[:n].view_as(q)):
            first = flat[:n].view_as(q) if other.data_ptr() != flat.data_ptr() else flat[shift:shift + n].view_as(q)
            with pytest.raises(ValueError, match="q's memory"):
                pkg.verify_attn_kv4(first, cache, *lens, x["scale"], out=other)
    with pytest.raises(pkg.SpecMoEError, match="OVERLAP"):
        pkg.verify_attn_kv4(q, cache, *lens, x["scale"], out=out, lse=flat[2 * n - 4:2 * n - 4 + B * C * Hq].view(B, C, Hq))
