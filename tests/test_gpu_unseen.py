"""A draft token that sees no key gets out = 0 and lse = -inf whatever the hidden
keys and values of its sequence hold: tree drafts without context, and scored
calls whose context a first key or a window hides, over types, pages and one to
five 16-row blocks (of which one and two are split over the waves by keys)."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
from paper_2508_21706_amd import workloads as wl
from test_gpu_parity import dev, note

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.mark.parametrize("dtype,D", [("f32", 128), ("f32", 64), ("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("g,C", [(1, 3), (4, 6), (4, 12), (2, 33)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("page", [0, 16])
def test_unseen_values_leave_empty_rows_alone(dtype, D, g, C, bad, page):
    d, Hkv, S = dev(), 2, 96
    gen = torch.Generator().manual_seed(C)
    rand = lambda *shape: torch.randn(shape, generator=gen).to(TYPES[dtype])   # noqa: E731
    chunk = [C, C - 1, 2]
    B = len(chunk)
    q, k, v = rand(B, C, g * Hkv, D), rand(B, Hkv, S, D), rand(B, Hkv, S, D)
    words = wl.tree_draft_masks(C, np.int32(chunk), C)
    empty = [[0, C - 1], [1], [0]]   # draft tokens whose word has no bit
    for b, rows in enumerate(empty):
        for i in rows:
            words[b, i] = 0
    for l in ([0, 0, 0], [40, 7, 17]):
        kk, vv = k.clone(), v.clone()
        for b in range(B):
            kk[b, :, l[b] + chunk[b] - 1], vv[b, :, l[b]:l[b] + chunk[b]] = bad, bad
        table = None
        if page:
            n = S // page
            table = torch.arange(B * n, dtype=torch.int32).reshape(B, n).to(d)
            kk, vv = (x.reshape(B, Hkv, n, page, D).transpose(1, 2).reshape(B * n, Hkv, page, D) for x in (kk, vv))
        t = lambda a: torch.tensor(a, dtype=torch.int32, device=d)   # noqa: E731
        head = (q.to(d), kk.contiguous().to(d), vv.contiguous().to(d))
        mask = torch.from_numpy(words.view(np.int64)).to(d)
        calls = {}
        if not any(l):
            if page:
                calls["plain"] = pkg.verify_attn_paged(*head, table, t(l), t(chunk), D ** -0.5, draft_mask=mask)
            else:
                calls["plain"] = pkg.verify_attn_tree(*head, t(l), t(chunk), mask, D ** -0.5)
        for name, kw in (("starts", dict(starts=t(l), softcap=5.0)), ("window", dict(window=1))):
            calls[name] = pkg.verify_attn_scored(*head, t(l), t(chunk), D ** -0.5, draft_mask=mask, block_table=table, **kw)
        torch.cuda.synchronize()
        for name, (out, lse) in calls.items():
            for b, rows in enumerate(empty):
                for i in rows:
                    assert (lse[b, i] == -np.inf).all(), f"{name} contexts {l}: lse of row {b, i}"
                    assert (out[b, i] == 0).all(), f"{name} contexts {l}: out of row {b, i}"
                assert (out[b, chunk[b]:] == 0).all() and (lse[b, chunk[b]:] == -np.inf).all()
    note(f"[unseen {dtype} {D} g={g} C={C} {bad} page={page}]")
