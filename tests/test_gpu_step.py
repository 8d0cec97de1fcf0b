"""The operators together, as a serving loop calls them: a chunk's append, the
scored verification attention over the cache it made, logits, and acceptance by
sampling -- step after step, over slabs and pages, for chains and trees; then
captured into graphs, replayed between eager work, and on two streams at once.

The attention and the acceptance are compared with the oracle on the very
cache, queries and logits that the step before them left (each operator's own
tests bound its errors); the cache itself with the append's oracle."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
from oracle.step import accept_sample_ref, append_ref, scored_attn_ref
from paper_2508_21706_amd import workloads as wl
from test_gpu_parity import dev, note

pytestmark = pytest.mark.gpu

B, C, Hq, Hkv, D, S, V, PAGE = 4, 6, 8, 2, 64, 128, 256, 16
SCORE = dict(softcap=8.0, window=40)


def f64(t):
    return t.detach().cpu().double().numpy()


class Loop:
    """One model layer's serving state."""

    def __init__(self, seed, dtype, paged, tree):
        d = dev()
        self.gen = torch.Generator().manual_seed(seed)
        self.dtype, self.tree, self.seed = dtype, tree, seed
        self.k, self.v = (torch.zeros((B, Hkv, S, D), dtype=dtype, device=d) for _ in range(2))
        self.table = None
        if paged:
            n = B * S // PAGE
            self.k, self.v = (torch.zeros((n + 2, Hkv, PAGE, D), dtype=dtype, device=d) for _ in range(2))
            self.table = torch.randperm(n + 2, generator=self.gen)[:n].reshape(B, -1).int().to(d)
        self.ctx = torch.zeros((B,), dtype=torch.int32, device=d)
        self.inv = torch.from_numpy(1.0 / 1e4 ** (np.arange(0, D, 2) / D)).to(d)
        self.wq, self.wk = (torch.rand((D,), generator=self.gen).add(0.5).to(dtype).to(d) for _ in range(2))
        self.slopes = (2.0 ** -torch.arange(1, Hq + 1)).to(d)
        self.proj = torch.randn((Hq * D, V), generator=self.gen).to(d)
        self.settings = dict(temperature=torch.tensor([0.7, 1.0, 0.0, 1.3], device=d),
                             top_k=torch.tensor([0, 20, 0, 0], dtype=torch.int32, device=d),
                             top_p=torch.tensor([0.9, 1.0, 1.0, 0.95], device=d))
        self.x = dict(qkv=torch.empty((B, C, Hq + 2 * Hkv, D), dtype=dtype, device=d),
                      chunk=torch.empty((B,), dtype=torch.int32, device=d),
                      tokens=torch.empty((B, C), dtype=torch.int32, device=d), u=torch.empty((B, C), device=d),
                      mask=torch.empty((B, C), dtype=torch.int64, device=d) if tree else None)
        self.q = torch.zeros((B, C, Hq, D), dtype=dtype, device=d)
        self.out, self.lse = torch.empty_like(self.q), torch.empty((B, C, Hq), device=d)
        self.logits = torch.empty((B, C, V), device=d)
        self.ws = pkg.alloc_scored_workspace(self.q, self.k, self.table, grid_blocks=24)
        self.aws = pkg.alloc_accept_workspace(pkg.accept_desc(B, C, V, 0), d)
        self.res = {n: torch.empty(s, dtype=t, device=d) for n, s, t in (
            ("sampled", (B, C), torch.int32), ("logprobs", (B, C), torch.float32), ("accepted", (B,), torch.int32),
            ("next_token", (B,), torch.int32), ("new_ctx_lens", (B,), torch.int32))}
        if tree:
            self.res["path"] = torch.empty((B,), dtype=torch.int64, device=d)

    def inputs(self, step, chunk):
        """New inputs of a step, into the buffers that the calls read."""
        rand = lambda *s: torch.randn(s, generator=self.gen)   # noqa: E731
        self.x["qkv"].copy_(rand(B, C, Hq + 2 * Hkv, D))
        self.x["chunk"].copy_(torch.tensor(chunk))
        self.x["tokens"].copy_(torch.randint(0, V, (B, C), generator=self.gen))
        self.x["u"].copy_(torch.rand((B, C), generator=self.gen))
        self.words = None
        if self.tree:
            self.words = wl.tree_draft_masks(self.seed + step, np.int32(chunk), C)
            self.x["mask"].copy_(torch.from_numpy(self.words.view(np.int64)))

    def step(self, stream=None):
        x, q = self.x, self.x["qkv"]
        pkg.append_kv(q[:, :, :Hq], q[:, :, Hq:Hq + Hkv], q[:, :, Hq + Hkv:], self.k, self.v, self.ctx, x["chunk"],
                      inv_freq=self.inv, q_weight=self.wq, k_weight=self.wk, draft_mask=x["mask"],
                      block_table=self.table, q_out=self.q, stream=stream)
        pkg.verify_attn_scored(self.q, self.k, self.v, self.ctx, x["chunk"], D ** -0.5, slopes=self.slopes,
                               draft_mask=x["mask"], block_table=self.table, out=self.out, lse=self.lse,
                               workspace=self.ws, grid_blocks=24, stream=stream, **SCORE)
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            torch.matmul(self.out.view(B * C, Hq * D).float(), self.proj, out=self.logits.view(B * C, V))
        args = dict(out=self.res, workspace=self.aws, stream=stream, **self.settings)
        if self.tree:
            pkg.accept_sample_tree(self.logits, x["tokens"], x["mask"], self.ctx, x["chunk"], x["u"], **args)
        else:
            pkg.accept_sample(self.logits, x["tokens"], self.ctx, x["chunk"], x["u"], **args)

    def state(self):
        return {**{n: t.clone() for n, t in self.res.items()}, "out": self.out.clone(), "lse": self.lse.clone(),
                "q": self.q.clone(), "k": self.k.clone(), "v": self.v.clone()}

    def slab(self, cache):
        if self.table is None:
            return cache
        return cache[self.table.long()].transpose(1, 2).reshape(B, Hkv, S, D)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("tree", [False, True])
def test_steps_follow_each_other(dtype, paged, tree):
    m = Loop(1, dtype, paged, tree)
    eps = torch.finfo(dtype).eps
    for step, chunk in enumerate([[6, 6, 6, 6], [5, 0, 6, 1], [6, 6, 1, 4], [3, 6, 6, 6]]):
        m.inputs(step, chunk)
        ctx = m.ctx.tolist()
        before = [f64(t) for t in (m.k, m.v, m.q)]
        m.step()
        torch.cuda.synchronize()
        q = f64(m.x["qkv"])
        want = append_ref(q[:, :, :Hq], q[:, :, Hq:Hq + Hkv], q[:, :, Hq + Hkv:], before[0], before[1], before[2], ctx,
                          chunk, f64(m.inv), "halves", f64(m.wq), f64(m.wk), 1e-6, m.words,
                          None if m.table is None else m.table.cpu().numpy())
        for name, got, ref in zip(("q", "k", "v"), (m.q, m.k, m.v), want):
            # (half a step of the type, and fp32's part: |x_a| + |x_b| < 12 here)
            err = np.abs(f64(got) - ref)
            assert (err <= eps / 2 * np.abs(ref) * (1 + eps) + 24 * 2.0 ** -24 * 12).all(), f"step {step}: {name}"
        ref_o, ref_l = scored_attn_ref(f64(m.q), f64(m.slab(m.k)), f64(m.slab(m.v)), ctx, chunk, D ** -0.5,
                                       slopes=f64(m.slopes), words=m.words, **SCORE)
        seen = np.isfinite(ref_l)
        assert np.array_equal(seen, np.isfinite(f64(m.lse)))
        # (values below 5: two roundings of 16 bits, the probabilities' and the result's)
        tol = 1e-4 if dtype == torch.float32 else 2 * eps / 2 * 5 + 1e-4
        assert np.abs(f64(m.out) - ref_o).max() <= tol and np.abs(f64(m.lse)[seen] - ref_l[seen]).max() <= 1e-4
        settings = [{n: float(f64(t)[b]) for n, t in m.settings.items()} for b in range(B)]
        ref = accept_sample_ref(f64(m.logits), m.x["tokens"].cpu().numpy(), ctx, chunk, f64(m.x["u"]), settings, m.words)
        for name in ("sampled", "accepted", "next_token", "new_ctx_lens"):
            assert m.res[name].cpu().tolist() == ref[name].tolist(), f"step {step}: {name}"
        if tree:
            assert m.res["path"].cpu().tolist() == ref["path"].tolist()
            if not paged:
                pkg.compact_accepted_kv(m.k, m.v, m.ctx, m.res["path"])
        m.ctx.copy_(m.res["new_ctx_lens"])
    assert pkg.workspace_status(m.ws) == 0
    note(f"[step {dtype} paged={paged} tree={tree}] contexts {m.ctx.tolist()}")


@pytest.mark.parametrize("tree", [False, True])
def test_steps_replayed_from_graphs(tree):
    """Two captured steps share one loop's workspaces; replays in turn, with
    eager steps and other inputs between them, equal eager results."""
    m = Loop(2, torch.bfloat16, True, tree)
    m.ctx.copy_(torch.tensor([60, 3, 90, 0]))
    m.inputs(0, [6, 5, 6, 2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.step(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.step()
        graphs.append(g)
    for k in range(6):
        m.inputs(k + 1, [[6, 5, 6, 2], [1, 0, 6, 6], [6, 6, 6, 6]][k % 3])
        m.step()
        torch.cuda.synchronize()
        want = m.state()
        for t in (m.out, m.lse, *m.res.values()):
            t.zero_()
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        for n, t in m.state().items():
            assert torch.equal(t, want[n]), f"replay {k}: {n}"
    assert pkg.workspace_status(m.ws) == 0


def test_two_loops_at_once():
    """Two loops with their own workspaces on two streams give what each gives
    alone."""
    loops = [Loop(3 + i, torch.bfloat16, bool(i), bool(i)) for i in range(2)]
    want = []
    for m in loops:
        m.ctx.copy_(torch.tensor([50, 70, 10, 0]))
        m.inputs(0, [6, 6, 3, 6])
        m.step()
        torch.cuda.synchronize()
        want.append(m.state())
    streams = [torch.cuda.Stream() for _ in loops]
    torch.cuda.synchronize()
    for _ in range(10):
        for m, s in zip(loops, streams):
            m.step(s)
    torch.cuda.synchronize()
    for m, w in zip(loops, want):
        for n, t in m.state().items():
            assert torch.equal(t, w[n]), n


def test_outputs_on_the_launch_stream():
    """Outputs that a call allocates come from the launch stream's pool: they
    hold their values though the current stream allocates meanwhile."""
    m = Loop(6, torch.bfloat16, False, False)
    m.inputs(0, [6, 6, 6, 6])
    m.step()
    torch.cuda.synchronize()
    want = m.state()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q = m.x["qkv"]
    for _ in range(5):
        got_q = pkg.append_kv(q[:, :, :Hq], q[:, :, Hq:Hq + Hkv], q[:, :, Hq + Hkv:], m.k, m.v, m.ctx, m.x["chunk"],
                              inv_freq=m.inv, q_weight=m.wq, k_weight=m.wk, stream=s)
        out, lse = pkg.verify_attn_scored(got_q, m.k, m.v, m.ctx, m.x["chunk"], D ** -0.5, slopes=m.slopes,
                                          grid_blocks=24, stream=s, **SCORE)
        tokens, logp = pkg.sample(m.logits.view(B * C, V), m.x["u"].view(-1), stream=s)
        res = pkg.accept_sample(m.logits, m.x["tokens"], m.ctx, m.x["chunk"], m.x["u"], stream=s, **m.settings)
        junk = [torch.full((1 << 16,), float("nan"), device=dev()) for _ in range(8)]
        s.synchronize()
        assert torch.equal(got_q, want["q"]) and torch.equal(out, want["out"]) and torch.equal(lse, want["lse"])
        assert torch.equal(res["sampled"], want["sampled"]) and int((tokens < 0).sum()) == 0
        del junk
