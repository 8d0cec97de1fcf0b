"""verify_attn_kv4 on the GPU against the float64 oracle on the values that the codes
stand for: types, head dims, head layouts, chains, trees, single tokens, slabs and
pages, ragged and empty chunks, cut units, tokens that see nothing, long contexts.

Rows past a sequence's last key hold NaN blocks, and table entries past its pages name
a page of them, so what must not be read shows.

Tolerances, per row, with h = eps / 2 of the type: a score is off by at most
ds = 2^-24 (D + 8) A + dq, A the largest scale sum |q k| of the row (the dot product's
roundings; codes are exact) and dq what the queries' 8-bit parts leave (of bfloat16
and float16 with D = 128): at most half a step, 2^-10, of the last part's unit, which
is 2^-5 per part under the first's, of which the block's largest entry is at least 2^7.
That is 2^-22 (two parts) and 2^-27 (three) of the largest |q| of the block, times the
sum of the block's |k|.  A probability is off by ds + 2^-21 more (the
exponential and its argument) and by hp, its rounding for the product with the values:
2^-8 of bfloat16's, cut to 16 bits for float16 (2^-15) and to 24 for float32 (2^-23);
sums add (T / 4 + 64) 2^-24.  So with W = sum p |v|
  |out - ref| <= (2 (ds + 2^-21 + (T / 4 + 64) 2^-24) + hp) W + h |ref|,
  |lse - ref| <= ds + 2^-21 + (T / 4 + 64) 2^-24 + 2^-23 |ref|."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
from oracle.kv4 import decode_ref, encode_ref
from oracle.step import scored_row_ref
from paper_2508_21706_amd import workloads as wl
from test_gpu_append import f64
from test_gpu_parity import dev, note

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DQ = {"f32": 0.0, "bf16": 2.0 ** -22, "f16": 2.0 ** -27}
HP = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -15}
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def random_rows(rng, *shape):
    """Codes and scales of rows of about unit size [.., D]."""
    D = shape[-1]
    codes = rng.integers(0, 256, size=(*shape[:-1], D // 2)).astype(np.uint8)
    scales = (127 + rng.integers(-3, 0, size=(*shape[:-1], D // 32))).astype(np.uint8)
    return codes, scales


def make(seed, dtype, ctx, chunk, Hq=8, Hkv=2, D=128, C=None, page=0, tree=False, q_scale=1.0, S=None):
    rng, B = np.random.default_rng(seed), len(ctx)
    C = C or max(max(chunk), 1)
    unit = max(64, page)
    S = S or -(-(max(l + c for l, c in zip(ctx, chunk)) + C) // unit) * unit
    gen = torch.Generator().manual_seed(seed)
    x = dict(ctx=ctx, chunk=chunk, C=C, dtype=dtype, scale=D ** -0.5, D=D)
    x["q"] = (torch.randn((B, C, Hq, D), generator=gen) * q_scale).to(TYPES[dtype])
    for b in range(B):
        x["q"][b, chunk[b]:] = float("nan")
    x["words"] = wl.tree_draft_masks(seed, np.int32(chunk), C) if tree else None
    x["slab"] = [*random_rows(rng, B, Hkv, S, D), *random_rows(rng, B, Hkv, S, D)]
    for b in range(B):
        for n in (1, 3):
            x["slab"][n][b, :, ctx[b] + chunk[b]:] = 255
    x["page"] = page
    x["perm"] = rng.permutation(B * (S // page) + 3) if page else None
    return x


def on_gpu(x):
    """(cache, table) on the GPU."""
    d = dev()
    if not x["page"]:
        return pkg.KV4Cache(*(torch.from_numpy(t).to(d) for t in x["slab"])), None
    page, perm = x["page"], x["perm"]
    B, Hkv, S = x["slab"][0].shape[:3]
    n = B * (S // page)
    table = perm[:n].reshape(B, -1).astype(np.int32)
    pools = []
    for t in x["slab"]:
        pool = np.full((n + 3, Hkv, page, t.shape[3]), 255, np.uint8)
        pool[table.reshape(-1)] = t.reshape(B, Hkv, S // page, page, -1).swapaxes(1, 2).reshape(n, Hkv, page, -1)
        pools.append(torch.from_numpy(pool).to(d))
    for b in range(B):   # entries that nothing may be read through
        table[b, -(-(x["ctx"][b] + x["chunk"][b]) // page):] = perm[-1]
    return pkg.KV4Cache(*pools), torch.from_numpy(table).to(d)


def call(x, cache=None, table=None, **kw):
    d = dev()
    if cache is None:
        cache, table = on_gpu(x)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=d)   # noqa: E731
    B, C, Hq, D = x["q"].shape
    out = torch.full((B, C, Hq, D), float("nan"), dtype=x["q"].dtype, device=d)
    lse = torch.full((B, C, Hq), float("nan"), device=d)
    got = pkg.verify_attn_kv4(x["q"].to(d), cache, i32(x["ctx"]), i32(x["chunk"]), x["scale"],
                              draft_mask=None if x["words"] is None else torch.from_numpy(x["words"].view(np.int64)).to(d),
                              block_table=table, out=out, lse=lse, check_lengths=True, **kw)
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is lse
    return out, lse


def sees_of(x, b, i):
    l, c = x["ctx"][b], x["chunk"][b]
    sees = np.arange(l + c) <= l + i
    if x["words"] is not None:
        sees[l:] = [(int(x["words"][b, i]) >> n) & 1 for n in range(c)]
    return sees


def check(x, out, lse, label="", rows=None, skip=()):
    o, s, q = f64(out), f64(lse), f64(x["q"])
    B, C, Hq, D = o.shape
    g = Hq // x["slab"][0].shape[1]
    h, hp = torch.finfo(TYPES[x["dtype"]]).eps / 2, HP[x["dtype"]]
    worst_o = worst_l = 0.0
    for b in range(B):
        l, c = x["ctx"][b], x["chunk"][b]
        assert (o[b, c:] == 0).all() and (s[b, c:] == -np.inf).all(), f"{label}: padding rows of sequence {b}"
        if rows is not None and b not in rows:
            continue
        T = l + c
        k, v = (decode_ref(x["slab"][n][b, :, :T], x["slab"][n + 1][b, :, :T]) for n in (0, 2))
        for i in range(c):
            sees = sees_of(x, b, i)
            for head in range(Hq):
                if (b, i, head) in skip:
                    continue
                kk, vv = k[head // g], v[head // g]
                ref_o, ref_l = scored_row_ref(q[b, i, head], np.where(sees[:, None], kk, 0), np.where(sees[:, None], vv, 0),
                                              x["scale"], sees)
                if not sees.any():
                    assert (o[b, i, head] == 0).all() and s[b, i, head] == -np.inf, f"{label}: {b} {i}"
                    continue
                A = float((np.abs(kk[sees]) @ np.abs(q[b, i, head])).max()) * x["scale"]
                sc = (kk[sees] @ q[b, i, head]) * x["scale"]
                p = np.exp(sc - ref_l)
                W = p @ np.abs(vv[sees])
                ds = 2.0 ** -24 * (D + 8) * A
                if D == 128:
                    per_block = np.abs(kk[sees]).reshape(-1, 4, 32).sum(-1) @ np.abs(q[b, i, head]).reshape(4, 32).max(-1)
                    ds += DQ[x["dtype"]] * float(per_block.max()) * x["scale"]
                rel = ds + 2.0 ** -21 + (T / 4 + 64) * 2.0 ** -24
                tol_o = (2 * rel + hp) * W + h * np.abs(ref_o) * (1 + h) + 2.0 ** -24 * (x["dtype"] == "f16")
                tol_l = rel + 2.0 ** -23 * abs(ref_l)
                eo, el = np.abs(o[b, i, head] - ref_o), abs(s[b, i, head] - ref_l)
                worst_o, worst_l = max(worst_o, float((eo / np.maximum(tol_o, 1e-300)).max())), max(worst_l, el / tol_l)
                assert (eo <= tol_o).all(), f"{label} out {b} {i} {head}: {float((eo / tol_o).max()):.2f} of the tolerance"
                assert el <= tol_l, f"{label} lse {b} {i} {head}: {el / tol_l:.2f} of the tolerance"
    note(f"[kv4 {label}] worst out {worst_o:.2f}, lse {worst_l:.2f} of the tolerance")


LENS = dict(ctx=[0, 1, 31, 32, 127, 128, 129, 300], chunk=[1, 3, 2, 0, 3, 1, 3, 2])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [0, 8, 16, 64])
def test_types_dims_pages(dtype, D, page):
    x = make(1, dtype, LENS["ctx"], LENS["chunk"], D=D, page=page)
    check(x, *call(x), label=f"{dtype} {D} page {page}")


@pytest.mark.parametrize("Hq,Hkv,C", [(1, 1, 1), (4, 4, 1), (7, 1, 2), (28, 4, 5), (32, 8, 5), (8, 1, 16), (16, 2, 7),
                                      (2, 1, 64), (64, 1, 2), (5, 5, 33)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_and_row_blocks(Hq, Hkv, C, dtype):
    """1 to 8 row blocks of 16, whole and partial."""
    x = make(2, dtype, [70, 5, 200], [C, max(1, C // 2), 1], Hq=Hq, Hkv=Hkv, C=C)
    check(x, *call(x), label=f"{Hq}/{Hkv} chunk {C} {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page", [0, 16])
def test_trees(dtype, page):
    x = make(3, dtype, [0, 100, 17, 250, 64], [16, 16, 9, 1, 0], C=16, page=page, tree=True)
    check(x, *call(x), label=f"tree {dtype} page {page}")


def test_tree_of_64_and_words_that_hide_everything():
    x = make(4, "bf16", [0, 40, 0], [64, 33, 3], Hq=2, Hkv=1, C=64, tree=True)
    x["words"][2] = 0            # no context, no bit: these tokens see nothing
    x["words"][1, 5] = 0         # sees the context alone
    x["words"][0, 7] = 1 << 63   # one key
    x["words"][1, 6] |= np.uint64(1) << np.uint64(60)   # (a bit past the chunk is ignored)
    check(x, *call(x), label="tree 64")


@pytest.mark.parametrize("grid", [1, 2, 3, 7, 100, 511, 2048])
def test_any_number_of_workgroups(grid):
    """Units whole, cut once and cut many times; one tile, 1 to 17 tiles."""
    x = make(5, "bf16", [2000, 1, 500, 0, 900], [4, 1, 0, 3, 2], C=4)
    check(x, *call(x, grid_blocks=grid), label=f"grid {grid}")


@pytest.mark.parametrize("grid", [1, 3, 17, 0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_units_of_unlike_rows_in_one_range(grid, dtype):
    """Chunks that need one, two and all four groups of waves, one after the other."""
    x = make(22, dtype, [300, 9, 700, 1, 128, 260], [16, 1, 5, 12, 2, 9], Hq=16, Hkv=2, C=16, page=16)
    check(x, *call(x, grid_blocks=grid), label=f"unlike rows {dtype} grid {grid}")


@pytest.mark.parametrize("Hq,dtype", [(4, "bf16"), (12, "f16"), (12, "f32"), (40, "bf16")])
def test_few_units_of_many_pieces(Hq, dtype):
    x = make(23, dtype, [9000, 0, 6001], [1, 1, 2], Hq=Hq, Hkv=1, C=2, D=128)
    check(x, *call(x), label=f"few units {Hq} {dtype}")


def test_results_do_not_depend_on_timing():
    x = make(6, "f16", [3000, 700, 15], [5, 5, 5], page=16)
    first = call(x)
    for _ in range(5):
        again = call(x)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_large_scores():
    x = make(7, "bf16", [200, 33], [2, 3], C=3, q_scale=30.0)
    check(x, *call(x), label="large scores")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_of_very_unlike_entries(dtype, D):
    """A large entry in every block, against keys that are 0 there: the small ones, down
    to 2^-20 of it, make the scores."""
    x = make(17, dtype, [150, 40], [3, 2], C=3, D=D, Hq=4, q_scale=2.0 ** -3)
    gen = torch.Generator().manual_seed(17)
    q = x["q"].float() * torch.exp2(-torch.randint(0, 8, x["q"].shape, generator=gen).float())
    for at, size in ((3, 2.0 ** 9), (16, 1.5 * 2.0 ** 8), (31, 448.0)):
        q[..., at::32] = q[..., at::32].sign() * size
        x["slab"][0][..., at // 2::16] &= 0x0F if at % 2 else 0xF0
    x["q"] = q.to(TYPES[dtype])
    check(x, *call(x), label=f"unlike entries {dtype} {D}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_queries_at_their_types_ends(dtype):
    """Entries up to the largest finite one, and subnormal ones, in rows of their own.

    Dot products are summed in float32: of bfloat16 entries up to 2^128, 128 products
    with keys up to 3 pass its largest, 2^128, so those rows (head 0 and 1 of the first
    tokens) are not compared; a 2^-10th of them sums to 2^128 2^-10 128 3 at most, and is."""
    x = make(18, dtype, [150, 40], [3, 2], C=3, Hq=4)
    info = torch.finfo(TYPES[dtype])
    x["q"][:, 0, :2] = (x["q"][:, 0, :2].float().clamp(-1, 1) * info.max).to(TYPES[dtype])
    x["q"][:, 0, 2:] = (x["q"][:, 0, 2:].float().clamp(-1, 1) * info.max * 2.0 ** -10).to(TYPES[dtype])
    x["q"][:, 1, 1] = (x["q"][:, 1, 1].float() * info.tiny / 4).to(TYPES[dtype])
    # (scores within float32, and not all of them past a softmax's reach)
    x["scale"] = 2.0 ** -120 if dtype == "bf16" else 2.0 ** -12
    check(x, *call(x), label=f"ends {dtype}", skip=[(b, 0, h) for b in (0, 1) for h in (0, 1)] if dtype == "bf16" else ())


def test_exponents_at_their_ends():
    """Units from the least to 2^100, in blocks side by side; a key that outweighs all."""
    x = make(8, "f32", [64], [1], Hq=2, Hkv=1, D=64, q_scale=1e-3)
    scales = x["slab"][1][0, 0, :65]
    scales[:32], scales[32:64] = 1, 0
    scales[10], scales[40, 1] = 130, 134
    x["slab"][3][0, 0, :65] = np.random.default_rng(8).integers(100, 140, size=(65, 2))
    check(x, *call(x), label="exponents")


def test_a_long_context():
    x = make(9, "bf16", [40000, 33000], [2, 1], Hq=4, Hkv=1, C=2, page=64)
    check(x, *call(x), label="long")


def test_many_sequences():
    """More than one launch's 1024, and more than one length per thread of the schedule."""
    rng = np.random.default_rng(10)
    n = 1300
    x = make(10, "bf16", rng.integers(0, 40, size=n).tolist(), rng.integers(0, 3, size=n).tolist(), Hq=2, Hkv=1, D=64, C=2)
    check(x, *call(x), label="1300 sequences", rows=list(range(0, n, 37)) + [1023, 1024, 1299])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_nan_blocks_reach_only_the_rows_that_see_them(D, tree):
    """A NaN block among the values (or keys) of a draft token: rows that see the token
    are NaN there (there: a key's NaN makes the whole row NaN), all others as without it."""
    x = make(11, "bf16", [45, 3], [6, 6], Hq=4, Hkv=2, D=D, C=6, tree=tree)
    if tree:   # 0 - 1 - 2, 0 - 3 - 4, 5 alone
        x["words"][:] = np.array([1, 3, 7, 9, 25, 32], np.uint64)
    clean = [t.copy() for t in x["slab"]]
    x["slab"][3][0, 0, 45 + 3, 1] = 255       # values of token 3 of sequence 0, KV head 0, block 1
    x["slab"][1][1, 1, 3 + 2, 0] = 255        # keys of token 2 of sequence 1, KV head 1
    out, lse = call(x)
    x["slab"] = clean
    ref, ref_lse = call(x)
    for i in range(6):
        for head in range(4):
            for b in range(2):
                sees = sees_of(x, b, i)
                v_hit = b == 0 and head < 2 and sees[45 + 3]
                k_hit = b == 1 and head >= 2 and sees[3 + 2]
                nan = torch.isnan(out[b, i, head])
                if k_hit:
                    assert nan.all() and torch.isnan(lse[b, i, head]), (b, i, head)
                    continue
                assert bool(nan[32:64].all()) == bool(v_hit) and not nan[:32].any() and not nan[64:].any(), (b, i, head)
                keep = ~nan
                assert torch.equal(out[b, i, head][keep], ref[b, i, head][keep]) and lse[b, i, head] == ref_lse[b, i, head]


def test_infinite_and_nan_queries_stay_in_their_rows():
    x = make(12, "f16", [50], [4], Hq=4, Hkv=2, C=4)
    ref = call(x)
    x["q"][0, 1, 2, 5], x["q"][0, 2, 0, 0] = float("inf"), float("nan")
    out, lse = call(x)
    hit = torch.zeros((4, 4), dtype=torch.bool, device=out.device)
    hit[1, 2] = hit[2, 0] = True
    assert torch.equal(out[0][~hit], ref[0][0][~hit]) and torch.equal(lse[0][~hit], ref[1][0][~hit])
    assert torch.isnan(lse[0][hit]).all()


def test_lengths_out_of_range_and_bad_pages_stay_in_bounds():
    """Clamped before any access; other sequences are as they would be."""
    x = make(13, "bf16", [30, 20, 40], [2, 2, 2], page=8, S=64)
    cache, table = on_gpu(x)
    good = call(x, cache, table)
    d = dev()
    table[1] = torch.tensor([10 ** 6, -1, 5, 0, 0, 0, 0, 0], device=d)
    out, lse = pkg.verify_attn_kv4(x["q"].to(d), cache, torch.tensor([30, 10 ** 9, 40], dtype=torch.int32, device=d),
                                   torch.tensor([2, 99, 2], dtype=torch.int32, device=d), x["scale"], block_table=table)
    torch.cuda.synchronize()
    for b in (0, 2):
        assert torch.equal(out[b], good[0][b]) and torch.equal(lse[b], good[1][b])


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 64), ("f32", 64)])
@pytest.mark.parametrize("S", [1, 5, 37, 143])
def test_full_slabs_of_odd_capacities(dtype, D, S):
    """Every row of the slabs is a key, and the cache's tensors end with the last one."""
    c = min(S, 3)
    x = make(19, dtype, [S - c, S - 1, 0], [c, 1, c], C=c, D=D, S=S)
    check(x, *call(x), label=f"S {S} {dtype} {D}")


def test_sequences_that_share_their_first_pages():
    x = make(20, "bf16", [70, 64, 40], [2, 2, 2], C=2, page=16)
    for t in x["slab"]:
        t[1, :, :64], t[2, :, :32] = t[0, :, :64], t[0, :, :32]
    cache, table = on_gpu(x)
    ref = call(x, cache, table)
    table[1, :4], table[2, :2] = table[0, :4].clone(), table[0, :2].clone()
    got = call(x, cache, table)
    assert torch.equal(ref[0], got[0]) and torch.equal(ref[1], got[1])


def test_results_in_the_queries_memory_are_refused():
    x = make(21, "bf16", [40], [2])
    cache, _ = on_gpu(x)
    q, n = x["q"].to(dev()), torch.tensor([2], dtype=torch.int32, device=dev())
    with pytest.raises(ValueError, match="q's memory"):
        pkg.verify_attn_kv4(q, cache, n, n, x["scale"], out=q)


def test_agrees_with_the_16_bit_path_on_rows_that_are_read_back():
    """The same call of verify_attn on the cache that read_kv4 makes."""
    x = make(14, "bf16", [600, 31], [5, 4], Hq=32, Hkv=8, C=5)
    cache, _ = on_gpu(x)
    d = dev()
    T = torch.tensor([605, 35], dtype=torch.int32, device=d)
    k, v = pkg.read_kv4(cache, torch.zeros_like(T), T, 605)
    k, v = (t.transpose(1, 2).contiguous() for t in (k, v))
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=d)   # noqa: E731
    ref, ref_lse = pkg.verify_attn(x["q"].to(d).nan_to_num(), k, v, i32(x["ctx"]), i32(x["chunk"]), x["scale"])
    out, lse = call(x, cache)
    fin = torch.isfinite(ref_lse)
    assert torch.equal(fin, torch.isfinite(lse)) and (lse[fin] - ref_lse[fin]).abs().max() < 1e-4
    # both round probabilities to bfloat16 (2^-8 of W, about 1 here), and one its result (2^-8)
    assert (out.float() - ref).abs().max() <= 3 * 2.0 ** -8


def test_a_workspace_serves_both_attentions():
    x = make(15, "bf16", [900, 80], [3, 3], C=3)
    cache, _ = on_gpu(x)
    ws = pkg.alloc_kv4_workspace(x["q"].to(dev()), cache)
    ref = call(x, cache)
    B, C, Hq, D = x["q"].shape
    k = torch.randn((B, 2, 1024, D), device=dev()).to(torch.bfloat16)
    for _ in range(3):
        got = call(x, cache, workspace=ws)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
        a = torch.tensor(x["ctx"], dtype=torch.int32, device=dev())
        c = torch.tensor(x["chunk"], dtype=torch.int32, device=dev())
        pkg.verify_attn(x["q"].to(dev()).nan_to_num(), k, k, a, c, x["scale"], workspace=ws)
    assert pkg.workspace_status(ws) == 0
    assert int(ws[:256 + 1024 * 2 * 4].view(torch.int32).abs().sum()) == 0


def test_offsets_past_32_bits():
    d, page, Hkv, D = dev(), 64, 8, 128
    n = (1 << 32) // (page * Hkv * D // 2) + 2
    cache = pkg.alloc_kv4_cache(n, Hkv, page, D, d)
    rng = np.random.default_rng(16)
    x = dict(ctx=[70], chunk=[2], C=2, dtype="bf16", scale=D ** -0.5, D=D, words=None, page=0)
    x["q"] = torch.randn((1, 2, 8, D)).to(torch.bfloat16)
    x["slab"] = [*random_rows(rng, 1, Hkv, 2 * page, D), *random_rows(rng, 1, Hkv, 2 * page, D)]
    table = torch.tensor([[n - 1, n - 2]], dtype=torch.int32, device=d)
    for pool, slab in zip(cache, x["slab"]):
        for j, at in enumerate((n - 1, n - 2)):
            pool[at] = torch.from_numpy(slab[0, :, j * page:(j + 1) * page]).to(d)
    check(x, *call(x, cache, table), label="large pool")
