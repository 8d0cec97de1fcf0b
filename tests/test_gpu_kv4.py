"""append_kv4, read_kv4 and compact_accepted_kv4 on the GPU against the oracle: types,
head layouts, rotations, norms, packed and strided inputs, slabs and pages, chains,
trees and prompts, blocks on borders, empty and without a value, bad page numbers,
large offsets.

Codes and scales are equal: the kernel works a key out in fp64, off by less than 2^-40
of the pair's magnitude, so it can differ from the oracle only where a value lies as
near to a border between two codes but not on it, and no input here has such a value.  Queries have append_kv's tolerance: half a step of the type and
24 x 2^-24 of |x_a| + |x_b|.  Rows that are read come back exactly, but for float16's
one rounding.  Everything outside the rows that a call writes keeps its bits."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
from oracle.kv4 import cache_append_ref, cache_move_ref, cache_rows_ref, decode_ref, encode_ref
from paper_2508_21706_amd import workloads as wl
from test_gpu_append import f64, inv_freq_of
from test_gpu_parity import dev, note

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def make_cache(seed, B, Hkv, D, S, page=0):
    """A cache of arbitrary bytes (NaN blocks among them) and its table."""
    d, gen = dev(), torch.Generator().manual_seed(seed)
    shape, table = (B, Hkv, S), None
    if page:
        n = B * (S // page) + 3
        shape = (n, Hkv, page)
        table = torch.randperm(n, generator=gen)[:n - 3].reshape(B, -1).int().to(d)
    new = lambda n: torch.randint(0, 256, (*shape, n), generator=gen).to(torch.uint8).to(d)   # noqa: E731
    return pkg.KV4Cache(new(D // 2), new(D // 32), new(D // 2), new(D // 32)), table


def host(cache):
    return [x.cpu().numpy() for x in cache]


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).to(dev())


def check_append(x, cache, table, ctx, chunk, rot, rope="halves", norm=False, words=None, label=""):
    d = dev()
    inv = inv_freq_of(rot)
    to = lambda a: torch.from_numpy(np.asarray(a)).to(d)   # noqa: E731
    before, old_q = host(cache), x["q_out"].clone()
    got = pkg.append_kv4(x["q"], x["k"], x["v"], cache, i32(ctx), i32(chunk), inv_freq=None if inv is None else to(inv),
                         rope=rope, q_weight=x["wq"] if norm else None, k_weight=x["wk"] if norm else None, eps=1e-6,
                         draft_mask=None if words is None else to(words.view(np.int64)), block_table=table,
                         q_out=x["q_out"])
    torch.cuda.synchronize()
    assert got is x["q_out"]
    host_table = None if table is None else table.cpu().numpy()
    ref_q, ref, near = cache_append_ref(
        f64(x["q"]), f64(x["k"]), f64(x["v"]), before, f64(old_q), ctx, chunk, inv, rope, f64(x["wq"]) if norm else None,
        f64(x["wk"]) if norm else None, float(np.float32(1e-6)), words, host_table)
    # (on a border exactly: entries that are copied, as at position 0)
    assert ((near == 0) | (near > 2.0 ** -36)).all(), f"{label}: a block next to a border"
    for name, g, r in zip(pkg.KV4Cache._fields, host(cache), ref):
        assert np.array_equal(g, r), f"{label} {name}: {int((g != r).sum())} of {g.size} bytes differ"
    half, eps = rot // 2, torch.finfo(x["q"].dtype).eps
    g, mag = f64(x["q_out"]), np.abs(ref_q)
    if rot:
        a, b = ((slice(0, half), slice(half, rot)) if rope == "halves" else (slice(0, rot, 2), slice(1, rot, 2)))
        pair = np.hypot(ref_q[..., a], ref_q[..., b]) * np.sqrt(2.0)
        mag[..., a], mag[..., b] = pair, pair
    tol = eps / 2 * np.abs(ref_q) * (1 + eps) + 24 * 2.0 ** -24 * mag + 2.0 ** -24 * (x["q"].dtype == torch.float16)
    err = np.abs(g - ref_q)
    assert (err <= tol).all(), f"{label} q_out: {float((err / np.maximum(tol, 1e-300)).max()):.2f} of the tolerance"
    for b, c in enumerate(chunk):
        assert torch.equal(x["q_out"][b, c:], old_q[b, c:]), f"{label}: padding rows of sequence {b}"


def make(seed, dtype, B, Hq, Hkv, D, C, packed=False):
    d, gen = dev(), torch.Generator().manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen).to(TYPES[dtype])   # noqa: E731
    x = {}
    if packed:
        qkv = rand(B, C, Hq + 2 * Hkv, D).to(d)
        x["q"], x["k"], x["v"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    else:
        x["q"], x["k"], x["v"] = (rand(B, C, h, D).to(d) for h in (Hq, Hkv, Hkv))
    x["q_out"], x["wq"], x["wk"] = rand(B, C, Hq, D).to(d), rand(D).to(d), rand(D).to(d)
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,rot,rope", [(128, 128, "halves"), (128, 128, "pairs"), (64, 64, "halves"), (64, 32, "pairs"),
                                        (128, 48, "halves"), (128, 16, "pairs"), (64, 16, "halves"), (64, 0, "halves")])
@pytest.mark.parametrize("norm", [False, True])
def test_append_types_and_rotations(dtype, D, rot, rope, norm):
    x = make(1, dtype, 3, 6, 2, D, 5)
    cache, table = make_cache(2, 3, 2, D, 64)
    check_append(x, cache, table, [0, 7, 59], [5, 0, 3], rot, rope, norm, label=f"{dtype} {D} {rot} {rope} {norm}")


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (28, 4), (32, 8), (3, 3), (80, 16)])
@pytest.mark.parametrize("page", [0, 8, 16, 64])
def test_append_heads_and_pages(Hq, Hkv, page):
    x = make(3, "bf16", 2, Hq, Hkv, 128, 4, packed=True)
    cache, table = make_cache(4, 2, Hkv, 128, 128, page)
    check_append(x, cache, table, [13, 124], [4, 4], 128, norm=True, label=f"{Hq}/{Hkv} page {page}")


@pytest.mark.parametrize("page", [0, 16])
def test_append_trees_take_their_depth(page):
    chunk = [16, 1, 0, 9]
    words = wl.tree_draft_masks(5, np.int32(chunk), 16)
    words[3, 4] = 0   # a token that sees nothing stands like a root
    x = make(5, "f16", 4, 8, 2, 64, 16, packed=True)
    cache, table = make_cache(6, 4, 2, 64, 64, page)
    check_append(x, cache, table, [40, 0, 5, 33], chunk, 64, norm=True, words=words, label="tree")


def test_append_a_prompt_and_far_positions():
    x = make(7, "bf16", 2, 4, 2, 64, 70, packed=True)
    cache, table = make_cache(8, 2, 2, 64, 1 << 17, 64)
    check_append(x, cache, table, [0, (1 << 17) - 60], [70, 60], 64, label="prompt")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_append_values_on_borders_and_without_a_value(dtype):
    """Without norm and rotation, keys and values are encoded as they are: ties, units
    that change at 7, tiny and huge blocks, zeros, infinities and NaN."""
    x = make(9, dtype, 1, 2, 2, 64, 6)
    ties = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0] * 4)
    unit = torch.tensor([1.0, 2.0 ** -10, 1024.0])
    for n in ("k", "v"):
        t = torch.zeros((1, 6, 2, 64))
        for i in range(3):
            t[0, i] = torch.cat([ties, -ties]) * unit[i]
        t[0, 3, 0], t[0, 3, 1] = 7.0, -6.96875
        t[0, 4, 0, 3], t[0, 4, 0, 40], t[0, 4, 1, 0] = float("inf"), float("nan"), -0.0
        t[0, 5] = torch.randn((2, 64)) * (2.0 ** -130 if dtype != "f16" else 2.0 ** -22)
        t[0, 5, 1, 32:] = torch.finfo(TYPES[dtype]).max
        x[n] = t.to(TYPES[dtype]).to(dev())
    cache, table = make_cache(10, 1, 2, 64, 32)
    check_append(x, cache, table, [3], [6], 0, label=f"borders {dtype}")
    assert (cache.k_scales[0, 0, 7] == 255).all() and (cache.k_scales[0, 1, 7] == 1).all()


def test_append_rows_outside_the_cache_are_dropped():
    x = make(11, "bf16", 2, 2, 2, 64, 4)
    cache, table = make_cache(12, 2, 2, 64, 32, 8)
    table[1, 1], table[1, 2] = -1, 10 ** 6
    before = host(cache)
    pkg.append_kv4(x["q"], x["k"], x["v"], cache, i32([30, 14]), i32([4, 4]), block_table=table)
    torch.cuda.synchronize()
    keep = np.ones(before[0].shape[0], bool)
    keep[int(table[0, 3])] = False
    for g, r in zip(host(cache), before):
        assert np.array_equal(g[keep], r[keep])
        assert not np.array_equal(g[~keep][0, :, 6:], r[~keep][0, :, 6:]) and np.array_equal(g[~keep][0, :, :6], r[~keep][0, :, :6])


def test_append_keys_and_values_only_and_past_the_slab():
    x = make(13, "f32", 1, 1, 2, 128, 3)
    cache, _ = make_cache(14, 1, 2, 128, 16)
    before = host(cache)
    assert pkg.append_kv4(None, x["k"], x["v"], cache, i32([15]), i32([3])) is None
    torch.cuda.synchronize()
    for g, r, t in zip(host(cache), before, (x["k"], x["k"], x["v"], x["v"])):
        assert np.array_equal(g[:, :, :15], r[:, :, :15])
    codes, scales, _ = encode_ref(f64(x["v"])[0, 0])
    assert np.array_equal(host(cache)[2][0, :, 15], codes) and np.array_equal(host(cache)[3][0, :, 15], scales)


# --------------------------------------------------------------------- read

def check_read(cache, table, first, rows, N, dtype, label=""):
    d = dev()
    Hkv, D = cache.k_codes.shape[1], 2 * cache.k_codes.shape[3]
    out = tuple(torch.randn((len(first), N, Hkv, D)).to(TYPES[dtype]).to(d) for _ in range(2))
    before = [t.clone() for t in out]
    got = pkg.read_kv4(cache, i32(first), i32(rows), out=out, block_table=table)
    torch.cuda.synchronize()
    assert got[0] is out[0] and got[1] is out[1]
    ref_cache, ref_table = host(cache), None if table is None else table.cpu().numpy()
    for b, (f, n) in enumerate(zip(first, rows)):
        for g, old, r in zip(out, before, cache_rows_ref(ref_cache, b, f, n, ref_table)):
            r = torch.from_numpy(r).to(TYPES[dtype]).to(d)   # (one rounding, for float16)
            assert torch.equal(torch.nan_to_num(g[b, :n].float(), nan=7e30), torch.nan_to_num(r.float(), nan=7e30)), f"{label} {b}"
            assert torch.equal(g[b, n:], old[b, n:]), f"{label} {b}: rows that stay"


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [0, 8, 32])
def test_read(dtype, D, page):
    cache, table = make_cache(20, 3, 3, D, 96, page)
    check_read(cache, table, [0, 90, 13], [96, 0, 37], 96, dtype, label=f"{dtype} {D} {page}")


def test_read_every_byte():
    d = dev()
    codes = torch.arange(256, device=d).repeat(256)[:256 * 256].reshape(1, 1, 2048, 32).to(torch.uint8)
    scales = torch.arange(256, device=d).repeat_interleave(16).reshape(1, 1, 2048, 2).to(torch.uint8)
    check_read(pkg.KV4Cache(codes, scales, codes.flip(2).contiguous(), scales), None, [0], [2048], 2048, "f32")


def test_read_leaves_rows_without_a_place():
    cache, table = make_cache(21, 1, 2, 64, 32, 8)
    table[0, 1] = 10 ** 6
    k, v = pkg.read_kv4(cache, i32([5]), i32([40]), max_rows=40, block_table=table)
    torch.cuda.synchronize()
    assert (k[0, 3:11] == 0).all() and (v[0, 27:] == 0).all()   # rows 8..15 have no page, rows from 32 on no place
    assert torch.equal(torch.nan_to_num(k[0, 11:27].float()),
                       torch.nan_to_num(pkg.read_kv4(cache, i32([16]), i32([16]), 16, block_table=table)[0][0].float()))


# --------------------------------------------------------------------- move

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [0, 8, 16])
def test_move(D, page):
    path = np.array([0b1, 0b1101, 0, (1 << 63) | 1, 0xAAAAAAAAAAAAAAAA, 0xFFFFFFFFFFFFFFFE, 0b110], np.uint64)
    ctx = [5, 0, 9, 60, 3, 64, 126]      # the last one's second row is past the cache
    cache, table = make_cache(30, len(ctx), 3, D, 128, page)
    before = host(cache)
    pkg.compact_accepted_kv4(cache, i32(ctx), torch.from_numpy(path.view(np.int64)).to(dev()), block_table=table)
    torch.cuda.synchronize()
    ref = cache_move_ref(before, ctx, path, 128, None if table is None else table.cpu().numpy())
    for name, g, r in zip(pkg.KV4Cache._fields, host(cache), ref):
        assert np.array_equal(g, r), f"{name} D {D} page {page}"


def test_move_skips_pages_outside_the_pool():
    cache, table = make_cache(31, 1, 2, 64, 32, 8)
    table[0, 1] = -5
    before = host(cache)
    pkg.compact_accepted_kv4(cache, i32([6]), torch.tensor([0b10000000110], device=dev()), block_table=table)
    torch.cuda.synchronize()
    # nodes 1, 2, 10: rows 7 and 8 (no page), 16 to 6, 7, 8 (no page)
    ref = [np.array(x) for x in before]
    at = int(table[0, 0])
    for x in ref:
        x[at, :, 6] = x[at, :, 7]
    for g, r in zip(host(cache), ref):
        assert np.array_equal(g, r)


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes of codes: the append, the read and the move reach
    its last page."""
    d, page, Hkv, D = dev(), 64, 8, 128
    n = (1 << 32) // (page * Hkv * D // 2) + 2
    cache = pkg.alloc_kv4_cache(n, Hkv, page, D, d)
    assert cache.k_codes.numel() > 1 << 32
    table = torch.tensor([[n - 1, n - 2]], dtype=torch.int32, device=d)
    x = make(40, "bf16", 1, 8, Hkv, D, 6)
    pkg.append_kv4(x["q"], x["k"], x["v"], cache, i32([61]), i32([6]), block_table=table)
    pkg.compact_accepted_kv4(cache, i32([61]), torch.tensor([0b101001], device=d), block_table=table)
    k, v = pkg.read_kv4(cache, i32([61]), i32([6]), 6, block_table=table)
    torch.cuda.synchronize()
    for got, src in ((k, x["k"]), (v, x["v"])):
        ref = decode_ref(*encode_ref(f64(src)[0])[:2])[[0, 3, 5, 3, 4, 5]]
        assert np.array_equal(f64(got)[0], ref)
    note(f"pool of {cache.k_codes.numel() / 2 ** 30:.1f} GiB of key codes")
