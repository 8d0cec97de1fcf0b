"""append_kv on the GPU against the float64 oracle: types, head layouts, both
rotations, partial rotations, norms, packed and strided inputs, slabs and
pages, chains, trees and prompts, empty chunks, far positions.

Tolerance: the result is rounded once to its type (half a step, eps / 2 of the
value); before that fp32 leaves at most 24 x 2^-24 of |x_a| + |x_b| of the
rotated pair: the norm's sum of up to 128 squares, root, quotient and two
products at most 16 half-steps, sine and cosine at most 4 (one for the angle,
rounded after its reduction to a turn, times pi), two products, a sum.
Values that are copied are equal bit for bit, and rows outside the chunk keep
their bits."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
from oracle.step import append_ref
from test_gpu_parity import dev, note
from paper_2508_21706_amd import workloads as wl

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def inv_freq_of(rot, theta=10000.0):
    return 1.0 / theta ** (np.arange(0, rot, 2) / rot) if rot else None


def make(seed, dtype, B, Hq, Hkv, D, C, S, page=0, packed=False):
    d = dev()
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen).to(TYPES[dtype])   # noqa: E731
    x = {}
    if packed:
        qkv = rand(B, C, Hq + 2 * Hkv, D).to(d)
        x["q"], x["k"], x["v"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    else:
        x["q"], x["k"], x["v"] = (rand(B, C, h, D).to(d) for h in (Hq, Hkv, Hkv))
    shape, x["table"] = (B, Hkv, S, D), None
    if page:
        n = B * (S // page) + 3
        shape = (n, Hkv, page, D)
        x["table"] = torch.randperm(n, generator=gen)[:n - 3].reshape(B, -1).int().to(d)
    x["k_cache"], x["v_cache"] = rand(*shape).to(d), rand(*shape).to(d)
    x["q_out"] = rand(B, C, Hq, D).to(d)
    x["wq"], x["wk"] = rand(D).to(d), rand(D).to(d)
    return x


def f64(t):
    return t.detach().cpu().double().numpy()


def check(x, ctx, chunk, rot, rope="halves", norm=False, words=None, label=""):
    d = dev()
    inv = inv_freq_of(rot)
    before = {n: x[n].clone() for n in ("q_out", "k_cache", "v_cache")}
    to = lambda a: torch.from_numpy(np.asarray(a)).to(d)   # noqa: E731
    args = dict(inv_freq=None if inv is None else to(inv), rope=rope,
                q_weight=x["wq"] if norm else None, k_weight=x["wk"] if norm else None, eps=1e-6,
                draft_mask=None if words is None else to(words.view(np.int64)), block_table=x["table"])
    got = pkg.append_kv(x["q"], x["k"], x["v"], x["k_cache"], x["v_cache"], to(np.int32(ctx)), to(np.int32(chunk)),
                        q_out=x["q_out"], **args)
    torch.cuda.synchronize()
    assert got is x["q_out"]
    ref = append_ref(f64(x["q"]), f64(x["k"]), f64(x["v"]), f64(before["k_cache"]), f64(before["v_cache"]),
                     f64(before["q_out"]), ctx, chunk, inv, rope, f64(x["wq"]) if norm else None,
                     f64(x["wk"]) if norm else None, 1e-6, words, None if x["table"] is None else x["table"].cpu().numpy())
    eps = torch.finfo(x["q"].dtype).eps
    worst = 0.0
    for name, r in zip(("q_out", "k_cache", "v_cache"), ref):
        g, old = f64(x[name]), f64(before[name])
        same = r == old
        assert np.array_equal(g[same], old[same]), f"{label} {name}: a value that stays changed"
        if name == "v_cache" or (rot == 0 and not norm):
            assert np.array_equal(g, r), f"{label} {name}: a copied value changed"
            continue
        half = rot // 2
        mag = np.abs(r)
        if rot:
            a, b = ((slice(0, half), slice(half, rot)) if rope == "halves" else (slice(0, rot, 2), slice(1, rot, 2)))
            pair = np.hypot(r[..., a], r[..., b]) * np.sqrt(2.0)   # >= |x_a| + |x_b| before the rotation
            mag[..., a], mag[..., b] = pair, pair
        tol = eps / 2 * np.abs(r) * (1 + eps) + 24 * 2.0 ** -24 * mag + 2.0 ** -24 * (TYPES["f16"] == x["q"].dtype)
        err = np.abs(g - r)
        worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
        assert (err <= tol).all(), f"{label} {name}: {float((err / tol).max()):.2f} of the tolerance"
    note(f"[append {label}] worst {worst:.2f} of the tolerance")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,rot,rope", [(128, 128, "halves"), (128, 128, "pairs"), (64, 64, "halves"), (64, 32, "pairs"),
                                        (128, 48, "halves"), (128, 16, "pairs"), (64, 0, "halves")])
@pytest.mark.parametrize("norm", [False, True])
def test_types_and_rotations(dtype, D, rot, rope, norm):
    x = make(1, dtype, 3, 6, 2, D, 5, 64)
    check(x, [0, 7, 59], [5, 0, 3], rot, rope, norm, label=f"{dtype} {D} {rot} {rope} {norm}")


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (28, 4), (32, 8), (80, 16)])
@pytest.mark.parametrize("page", [0, 8, 16, 64])
def test_heads_and_pages(Hq, Hkv, page):
    x = make(2, "bf16", 2, Hq, Hkv, 128, 4, 128, page=page, packed=True)
    check(x, [13, 124], [4, 4], 128, norm=True, label=f"{Hq}/{Hkv} page {page}")   # 13..16 crosses 16-token pages


@pytest.mark.parametrize("page", [0, 16])
def test_trees_take_their_depth(page):
    chunk = [16, 1, 0, 9]
    words = wl.tree_draft_masks(5, np.int32(chunk), 16)
    words[3, 4] = 0   # a token that sees nothing stands like a root
    x = make(3, "f16", 4, 8, 2, 64, 16, 64, page=page, packed=True)
    check(x, [40, 0, 5, 33], chunk, 64, norm=True, words=words, label="tree")


def test_a_prompt():
    x = make(4, "bf16", 2, 4, 2, 64, 300, 320, packed=True)
    check(x, [0, 20], [299, 300], 64, label="prompt")


def test_far_positions():
    S = 1 << 20
    x = make(5, "f32", 1, 2, 1, 64, 3, S)
    check(x, [S - 3], [3], 64, label="far")
    x = make(6, "f32", 1, 2, 1, 64, 3, S, page=1 << 16)
    check(x, [S - 5], [3], 64, "pairs", label="far, pages")


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes: the last sequence's rows."""
    d = dev()
    B, Hkv, S, D = 5, 4, 1 << 20, 128
    k_cache = torch.zeros((B, Hkv, S, D), dtype=torch.bfloat16, device=d)
    v_cache = torch.zeros_like(k_cache)
    k = torch.randn((B, 1, Hkv, D), device=d).bfloat16()
    lens = torch.tensor([3, 0, 1, 2, S - 1], dtype=torch.int32, device=d)
    one = torch.ones((B,), dtype=torch.int32, device=d)
    assert pkg.append_kv(None, k, -k, k_cache, v_cache, lens, one) is None
    torch.cuda.synchronize()
    for b, l in enumerate(lens.tolist()):
        assert torch.equal(k_cache[b, :, l], k[b, 0]) and torch.equal(v_cache[b, :, l], -k[b, 0])
    for h in range(Hkv):
        assert int((k_cache[:, h] != 0).any(-1).sum()) == B


def test_rows_and_pages_out_of_range_are_not_written():
    d = dev()
    B, Hkv, D, page, C = 3, 2, 64, 8, 4
    k = torch.randn((B, C, Hkv, D), device=d)
    chunk = torch.full((B,), C, dtype=torch.int32, device=d)
    cache = torch.zeros((4, Hkv, page, D), device=d)
    v_cache = torch.zeros_like(cache)
    # sequence 0 runs past its table, 1 names pages outside the pool, 2 fits
    table = torch.tensor([[0, 1], [-1, 4], [2, 3]], dtype=torch.int32, device=d)
    ctx = torch.tensor([14, 6, 7], dtype=torch.int32, device=d)
    pkg.append_kv(None, k, k, cache, v_cache, ctx, chunk, block_table=table)
    want = torch.zeros_like(cache)
    want[1, :, 6:8] = k[0, :2].transpose(0, 1)
    want[2, :, 7] = k[2, 0]
    want[3, :, 0:3] = k[2, 1:].transpose(0, 1)
    assert torch.equal(cache, want) and torch.equal(v_cache, want)
    slab = torch.zeros((B, Hkv, 16, D), device=d)
    v_slab = torch.zeros_like(slab)
    pkg.append_kv(None, k, k, slab, v_slab, torch.tensor([14, -3, 40], dtype=torch.int32, device=d),
                  torch.tensor([9, 2, 4], dtype=torch.int32, device=d))
    want = torch.zeros_like(slab)
    want[0, :, 14:16] = k[0, :2].transpose(0, 1)
    want[1, :, 0:2] = k[1, :2].transpose(0, 1)   # a negative length counts as 0
    assert torch.equal(slab, want) and torch.equal(v_slab, want)


def test_in_place_queries_and_strides():
    d = dev()
    x = make(7, "bf16", 2, 8, 2, 128, 5, 64)
    inv = torch.from_numpy(inv_freq_of(128)).to(d)
    ctx = torch.tensor([3, 17], dtype=torch.int32, device=d)
    chunk = torch.tensor([5, 4], dtype=torch.int32, device=d)
    want = pkg.append_kv(x["q"], x["k"], x["v"], x["k_cache"], x["v_cache"], ctx, chunk, inv_freq=inv,
                         q_weight=x["wq"])
    q = x["q"].clone()
    pkg.append_kv(q, x["k"], x["v"], x["k_cache"], x["v_cache"], ctx, chunk, inv_freq=inv, q_weight=x["wq"], q_out=q)
    assert torch.equal(q[0], want[0]) and torch.equal(q[1, :4], want[1, :4]) and torch.equal(q[1, 4], x["q"][1, 4])
    # one token per sequence out of longer rows: the batch's distance counts
    wide = torch.randn((2, 9, 12, 128), device=d).bfloat16()
    part = wide[:, 4:5]
    one = torch.ones((2,), dtype=torch.int32, device=d)
    got = pkg.append_kv(part[:, :, :8], part[:, :, 8:10], part[:, :, 10:], x["k_cache"], x["v_cache"], ctx, one,
                        inv_freq=inv)
    torch.testing.assert_close(got, pkg.append_kv(part[:, :, :8].contiguous(), part[:, :, 8:10].contiguous(),
                                                  part[:, :, 10:].contiguous(), x["k_cache"], x["v_cache"], ctx, one,
                                                  inv_freq=inv), rtol=0, atol=0)
    assert torch.equal(x["v_cache"][1, :, 17], part[1, 0, 10:])


def test_another_stream_and_empty_batch():
    d = dev()
    x = make(8, "f16", 2, 4, 2, 64, 3, 32)
    s = torch.cuda.Stream(device=d)
    ctx, chunk = (torch.tensor(n, dtype=torch.int32, device=d) for n in ([1, 2], [3, 3]))
    inv = torch.from_numpy(inv_freq_of(64)).to(d)
    want = pkg.append_kv(x["q"], x["k"], x["v"], x["k_cache"], x["v_cache"], ctx, chunk, inv_freq=inv)
    s.wait_stream(torch.cuda.current_stream(d))
    got = pkg.append_kv(x["q"], x["k"], x["v"], x["k_cache"], x["v_cache"], ctx, chunk, inv_freq=inv, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    none = torch.empty((0,), dtype=torch.int32, device=d)
    out = pkg.append_kv(x["q"][:0], x["k"][:0], x["v"][:0], x["k_cache"][:0], x["v_cache"][:0], none, none, inv_freq=inv)
    assert out.shape == (0, 3, 4, 64)


def test_positions_past_two_to_the_thirty():
    """A table of 2^31 - 65536 positions over two pages.  (The angle's own three
    roundings, 2^-53 of 2^30 each, are six of the half-steps that the norm
    would take.)"""
    d = dev()
    page, pos = 1 << 16, (1 << 30) + 3 * (1 << 16) + 77
    table = torch.zeros((1, (1 << 15) - 1), dtype=torch.int32, device=d)
    table[0, pos // page] = 1
    gen = torch.Generator().manual_seed(9)
    rand = lambda *shape: torch.randn(shape, generator=gen).to(d)   # noqa: E731
    x = dict(q=rand(1, 2, 2, 64), k=rand(1, 2, 1, 64), v=rand(1, 2, 1, 64), k_cache=rand(2, 1, page, 64),
             v_cache=rand(2, 1, page, 64), q_out=rand(1, 2, 2, 64), table=table)
    check(x, [pos], [2], 64, label="past 2^30")
