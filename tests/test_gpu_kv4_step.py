"""The 4-bit cache's and the pages' calls together, as a serving loop makes them: pages
for the chunk, the append, the attention over tree drafts, acceptance, the path's move.
Eager against the oracles step by step, in a captured graph against the eager run, on
streams of their own side by side, and with another GPU current."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
from oracle import accept_tree_ref
from oracle.kv4 import assign_pages_ref, cache_append_ref, cache_move_ref, cache_rows_ref
from oracle.step import scored_row_ref
from paper_2508_21706_amd import binding as bd
from paper_2508_21706_amd import workloads as wl
import test_gpu_devices as devices
from test_gpu_append import f64, inv_freq_of
from test_gpu_devices import calls  # noqa: F401
from test_gpu_parity import dev

pytestmark = pytest.mark.gpu

B, C, HQ, HKV, D, V, PAGE, PER = 4, 8, 8, 2, 128, 64, 16, 8


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).to(dev())


class Loop:
    """Buffers of a serving loop over one layer, and its step."""

    def __init__(self, seed, ctx):
        d, gen = dev(), torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=gen)   # noqa: E731
        n = B * PER
        self.cache = pkg.alloc_kv4_cache(n, HKV, PAGE, D, d)
        self.pages = pkg.alloc_page_state(B, PER, n, d)
        self.ctx, self.chunk = i32(ctx), i32([0] * B)
        self.inv = torch.from_numpy(inv_freq_of(D)).to(d)
        self.wq, self.wk = ((1 + 0.1 * rand(D)).to(torch.bfloat16).to(d) for _ in range(2))
        self.qkv = torch.zeros((B, C, HQ + 2 * HKV, D), dtype=torch.bfloat16, device=d)
        self.q_out = torch.zeros((B, C, HQ, D), dtype=torch.bfloat16, device=d)
        self.mask = torch.zeros((B, C), dtype=torch.int64, device=d)
        self.logits = torch.zeros((B, C, V), dtype=torch.bfloat16, device=d)
        self.tokens = torch.zeros((B, C), dtype=torch.int32, device=d)
        self.slots = torch.zeros((B, C), dtype=torch.int64, device=d)
        self.missing = i32([0] * B)
        self.out = torch.zeros_like(self.q_out)
        self.lse = torch.zeros((B, C, HQ), device=d)
        self.ws = pkg.alloc_kv4_workspace(self.q_out, self.cache, self.pages.block_table)
        self.aws = pkg.alloc_accept_workspace(pkg.accept_desc(B, C, V, bd.SPECMOE_BF16), d)
        self.acc = {k: i32(np.zeros((B, C) if k == "argmax" else B)) for k in ("argmax", "accepted", "next_token")}
        self.acc["path"] = torch.zeros((B,), dtype=torch.int64, device=d)

    def feed(self, seed, chunk):
        """New projections, drafts and logits; drafts that often match."""
        rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        self.chunk.copy_(i32(chunk))
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=gen).to(torch.bfloat16))
        words = wl.tree_draft_masks(seed, np.int32(chunk), C)
        self.mask.copy_(torch.from_numpy(words.view(np.int64)))
        logits = rng.standard_normal((B, C, V)).astype(np.float32)
        best = logits.argmax(-1)
        tokens = rng.integers(0, V, size=(B, C))
        for b in range(B):
            for i in range(1, chunk[b]):
                up = int(words[b, i]) & ~(1 << i)
                if rng.random() < 0.8:
                    tokens[b, i] = best[b, up.bit_length() - 1]
        self.logits.copy_(torch.from_numpy(logits).to(torch.bfloat16))
        self.tokens.copy_(torch.from_numpy(tokens.astype(np.int32)))

    def step(self, stream=None):
        q, k, v = self.qkv[:, :, :HQ], self.qkv[:, :, HQ:HQ + HKV], self.qkv[:, :, HQ + HKV:]
        table = self.pages.block_table
        pkg.assign_pages(self.ctx, self.chunk, self.pages, PAGE, missing=self.missing, slots=self.slots, stream=stream)
        pkg.append_kv4(q, k, v, self.cache, self.ctx, self.chunk, self.inv, q_weight=self.wq, k_weight=self.wk,
                       draft_mask=self.mask, block_table=table, q_out=self.q_out, stream=stream)
        pkg.verify_attn_kv4(self.q_out, self.cache, self.ctx, self.chunk, D ** -0.5, draft_mask=self.mask,
                            block_table=table, out=self.out, lse=self.lse, workspace=self.ws, stream=stream)
        before = self.ctx.clone()
        pkg.accept_greedy_tree(self.logits, self.tokens, self.mask, self.ctx, self.chunk, out=self.acc,
                               workspace=self.aws, stream=stream, in_place=True)
        pkg.compact_accepted_kv4(self.cache, before, self.acc["path"], block_table=table, stream=stream)

    def state(self):
        return [t.clone() for t in (*self.cache, *self.pages, self.ctx, self.slots, self.missing, self.out, self.lse,
                                    self.q_out, *self.acc.values())]


def test_steps_of_a_serving_loop():
    loop = Loop(1, [0, 0, 0, 0])
    cache = [t.cpu().numpy() for t in loop.cache]
    table, held, free, count = (t.cpu().numpy() for t in loop.pages)
    count, ctx, q_out = int(count[0]), np.zeros(B, np.int64), f64(loop.q_out)
    accepted = 0
    for step, chunk in enumerate([[8, 3, 1, 5], [8, 8, 8, 8], [2, 0, 8, 7], [8, 8, 5, 1]] * 2):
        loop.feed(100 + step, chunk)
        loop.step()
        torch.cuda.synchronize()
        ref = assign_pages_ref(ctx, np.array(chunk), table, held, free, count, PAGE, C)
        table, held, free, count = ref["table"], ref["held"], ref["free_pages"], ref["free_count"]
        for name, got in zip(("table", "held", "free_pages"), loop.pages):
            assert np.array_equal(got.cpu().numpy(), ref[name]), (step, name)
        assert np.array_equal(loop.slots.cpu().numpy(), ref["slots"]) and not ref["missing"].any()
        x, words = f64(loop.qkv), loop.mask.cpu().numpy().view(np.uint64)
        q_out, cache, near = cache_append_ref(
            x[:, :, :HQ], x[:, :, HQ:HQ + HKV], x[:, :, HQ + HKV:], cache, q_out, ctx, chunk, inv_freq_of(D), "halves",
            f64(loop.wq), f64(loop.wk), float(np.float32(1e-6)), words, table)
        assert (near > 2.0 ** -36).all()
        # attention on the queries as the call before left them
        q = f64(loop.q_out)
        for b in range(B):
            k, v = cache_rows_ref(cache, b, 0, int(ctx[b]) + chunk[b], table)
            for i in range(chunk[b]):
                sees = np.arange(len(k)) < ctx[b]
                sees[int(ctx[b]):] = [(int(words[b, i]) >> n) & 1 for n in range(chunk[b])]
                for h in range(HQ):
                    o, s = scored_row_ref(q[b, i, h], k[:, h // 4], v[:, h // 4], D ** -0.5, sees)
                    # (probabilities and the result are rounded to bfloat16, 2^-8 each at most)
                    w = np.abs(v[sees][:, h // 4]).max(0)
                    assert (np.abs(f64(loop.out)[b, i, h] - o) <= 2.0 ** -8 * (w + np.abs(o)) * 1.01).all(), (step, b, i, h)
                    assert abs(float(loop.lse[b, i, h]) - s) < 1e-4
        acc = accept_tree_ref(loop.logits.view(torch.int16).cpu().numpy().view(np.uint16), loop.tokens.cpu().numpy(), words,
                              ctx.astype(np.int32), np.int32(chunk), "bf16")
        path = loop.acc["path"].cpu().numpy()
        assert np.array_equal(path.view(np.uint64), np.asarray(acc["path"], np.uint64))
        cache = cache_move_ref(cache, ctx, path.view(np.uint64), PAGE * PER, table)
        accepted += int((acc["accepted"] > 0).sum())
        ctx = np.asarray(acc["new_ctx_lens"], np.int64)
        assert np.array_equal(loop.ctx.cpu().numpy(), ctx)
        for name, got, want in zip(pkg.KV4Cache._fields, loop.cache, cache):
            assert np.array_equal(got.cpu().numpy(), want), (step, name)
    assert accepted > 8 and ctx.max() > 16


def test_a_captured_step_replays():
    """Every replay against the eager step, with eager work and synchronizations between."""
    loop = Loop(2, [30, 0, 64, 17])
    loop.feed(7, [8, 5, 1, 8])
    start = [t.clone() for t in (*loop.cache, *loop.pages, loop.ctx)]

    def reset():
        for t, s in zip((*loop.cache, *loop.pages, loop.ctx), start):
            t.copy_(s)

    reset()
    loop.step()
    torch.cuda.synchronize()
    eager = loop.state()
    side = torch.cuda.Stream(dev())
    side.wait_stream(torch.cuda.current_stream(dev()))
    with torch.cuda.stream(side):
        reset()
        loop.step()
    torch.cuda.current_stream(dev()).wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        reset()
        loop.step()
    for rep in range(4):
        for t in (loop.out, loop.lse, loop.q_out, loop.slots, loop.missing):
            t.fill_(-5)
        reset()
        loop.q_out.zero_()
        loop.step()          # eager work on the same buffers
        torch.cuda.synchronize()
        loop.out.fill_(-5)
        loop.slots.fill_(-5)
        loop.q_out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n, (a, b) in enumerate(zip(loop.state(), eager)):
            assert torch.equal(a, b), f"replay {rep}: tensor {n}"
    assert int(loop.ws[:256 + 1024 * HKV * 4].view(torch.int32).abs().sum()) == 0


def test_two_loops_on_streams_of_their_own():
    alone, together = [], []
    for seed in (3, 4):
        loop = Loop(seed, [40, 9, 100, 0])
        loop.feed(seed, [8, 8, 3, 6])
        loop.step()
        torch.cuda.synchronize()
        alone.append(loop.state())
    loops = [Loop(seed, [40, 9, 100, 0]) for seed in (3, 4)]
    for seed, loop in zip((3, 4), loops):
        loop.feed(seed, [8, 8, 3, 6])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(dev()) for _ in loops]
    for loop, s in zip(loops, streams):
        with torch.cuda.stream(s):
            loop.step()
    torch.cuda.synchronize()
    together = [loop.state() for loop in loops]
    for a, b in zip(alone, together):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_an_explicit_stream_is_the_one_used():
    """Outputs that a call allocates come from the launch stream's pool, and the work is
    ordered after what that stream holds."""
    loop = Loop(5, [40, 9, 100, 0])
    loop.feed(5, [8, 8, 3, 6])
    loop.step()
    torch.cuda.synchronize()
    ref, cache, ctx = loop.out.clone(), loop.cache, i32([40, 9, 100, 0])
    s = torch.cuda.Stream(dev())
    q = loop.q_out.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        late = torch.zeros_like(q)
        torch.cuda._sleep(2_000_000)
        late.copy_(q)
    # (the table after the step: the chunk's pages are still held)
    out, lse = pkg.verify_attn_kv4(late, cache, ctx, loop.chunk, D ** -0.5, draft_mask=loop.mask,
                                   block_table=loop.pages.block_table, stream=s)
    k, v = pkg.read_kv4(cache, ctx, loop.chunk, max_rows=C, block_table=loop.pages.block_table, stream=s)
    s.synchronize()
    # rows that the move left alone: those of sequences whose path is a prefix
    path = loop.acc["path"].tolist()
    for b in range(B):
        if path[b] & (path[b] + 1) == 0:
            assert torch.equal(out[b], ref[b])
    assert k.shape == (B, C, HKV, D) and bool((k[2, 3:] == 0).all()) and bool((v[0] != 0).any())


def test_calls_with_another_gpu_current(calls, monkeypatch):  # noqa: F811
    monkeypatch.setattr(devices, "HOST_ONLY", devices.HOST_ONLY | {"specmoe_verify_attn_kv4_workspace_bytes"})
    loop = Loop(6, [5, 0, 3, 9])
    loop.feed(6, [2, 3, 1, 0])
    q, k, v = loop.qkv[:, :, :HQ], loop.qkv[:, :, HQ:HQ + HKV], loop.qkv[:, :, HQ + HKV:]
    table = loop.pages.block_table
    del calls[:]
    pkg.assign_pages(loop.ctx, loop.chunk, loop.pages, PAGE, max_chunk=C)
    pkg.append_kv4(q, k, v, loop.cache, loop.ctx, loop.chunk, loop.inv, block_table=table)
    pkg.verify_attn_kv4(loop.q_out, loop.cache, loop.ctx, loop.chunk, 0.1, block_table=table)
    pkg.read_kv4(loop.cache, loop.ctx, loop.chunk, C, block_table=table)
    pkg.compact_accepted_kv4(loop.cache, loop.ctx, loop.acc["path"], block_table=table)
    assert [n for n in calls if n not in devices.HOST_ONLY] == [
        "specmoe_assign_pages", "specmoe_append_kv4", "specmoe_verify_attn_workspace_init", "specmoe_verify_attn_kv4",
        "specmoe_read_kv4", "specmoe_compact_accepted_kv4"]


def test_tensors_elsewhere_are_refused():
    """A member of the cache, or of the page state, in host memory or of another shape."""
    loop = Loop(7, [5, 0, 3, 9])
    q = loop.q_out
    for n in range(4):
        host = loop.cache._replace(**{pkg.KV4Cache._fields[n]: loop.cache[n].cpu()})
        short = loop.cache._replace(**{pkg.KV4Cache._fields[n]: loop.cache[n][:, :, :, :-1].contiguous()})
        for bad in (host, short):
            with pytest.raises(ValueError):
                pkg.verify_attn_kv4(q, bad, loop.ctx, loop.chunk, 0.1, block_table=loop.pages.block_table)
        with pytest.raises(ValueError):
            pkg.assign_pages(loop.ctx, loop.chunk, pkg.PageState(*(t.cpu() if i == n else t for i, t in enumerate(loop.pages))), PAGE)
    with pytest.raises(ValueError, match="slabs"):
        pkg.verify_attn_kv4(q, loop.cache, loop.ctx, loop.chunk, 0.1)
    with pytest.raises(ValueError, match="heads of"):
        pkg.verify_attn_kv4(q[..., :64].contiguous(), loop.cache, loop.ctx, loop.chunk, 0.1,
                            block_table=loop.pages.block_table)
    with pytest.raises(ValueError, match="contiguous"):
        pkg.verify_attn_kv4(q, loop.cache, loop.ctx, loop.chunk, 0.1, block_table=loop.pages.block_table,
                            workspace=loop.ws[::2])
    with pytest.raises(pkg.SpecMoEError, match="WORKSPACE"):
        pkg.verify_attn_kv4(q, loop.cache, loop.ctx, loop.chunk, 0.1, block_table=loop.pages.block_table,
                            workspace=loop.ws[:4096])
