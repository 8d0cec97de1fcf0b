"""verify_attn_scored on the GPU against the float64 oracle: caps, slopes,
windows and starts, alone and together, over types, head dims, chains, trees,
slabs and pages, ragged and empty chunks, cut units and tokens that see nothing.

Rows that no token sees (before the first visible key, past the chunk) hold
NaN, and the table entries of pages that hold only such rows name a NaN page.

Tolerances, per row, with h = eps / 2 of the type: a score is off by at most
ds = 2^-24 (D A + 8 (cap + bias) + 8), A the largest scale sum |q k|, bias the
row's largest slope times distance among the keys that matter (those within 40
of the best score): the dot product's D roundings, and for cap, bias, their
difference and the maximum's at most eight more of what they are added to.  A
probability is off by ds + 2^-21 (ds and the exponential) and, in 16 bits, by h;
sums add (T / 4 + 64) 2^-24.  So with W = sum p |v|
  |out - ref| <= (2 (ds + 2^-21 + (T / 4 + 64) 2^-24) + h16) W + h |ref|,
  |lse - ref| <= ds + 2^-21 + (T / 4 + 64) 2^-24 + 2^-23 |ref|."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
from oracle.step import scored_row_ref
from paper_2508_21706_amd import workloads as wl
from test_gpu_parity import dev, note

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EVERYTHING = dict(softcap=20.0, slopes=True, window=150, starts=True)
SETTINGS = {"off": {}, "cap": dict(softcap=30.0), "tight_cap": dict(softcap=0.5), "slopes": dict(slopes=True),
            "window": dict(window=100), "starts": dict(starts=True), "all": EVERYTHING}


def f64(t):
    return t.detach().cpu().double().numpy()


def make(seed, dtype, ctx, chunk, Hq=8, Hkv=2, D=128, C=None, page=0, tree=False, q_scale=1.0, slopes=False,
         starts=None, window=0, S=None):
    """Inputs on the GPU, poisoned where nothing may be read."""
    d, rng, B = dev(), np.random.default_rng(seed), len(ctx)
    C = C or max(max(chunk), 1)
    unit = max(64, page)
    S = S or -(-(max(ctx) + C) // unit) * unit
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen).to(TYPES[dtype])   # noqa: E731
    x = dict(ctx=ctx, chunk=chunk, C=C, window=window, dtype=dtype, scale=D ** -0.5)
    x["q"] = rand(B, C, Hq, D) * q_scale
    k, v = rand(B, Hkv, S, D), rand(B, Hkv, S, D)
    x["starts"] = None
    if starts is not None:
        x["starts"] = [int(rng.integers(0, l + 1)) for l in ctx] if starts is True else starts
    x["words"] = wl.tree_draft_masks(seed, np.int32(chunk), C) if tree else None
    nan = float("nan")
    first = []
    for b in range(B):
        x["q"][b, chunk[b]:] = nan
        f = max(min(x["starts"][b], ctx[b]) if x["starts"] else 0, ctx[b] + 1 - window if window else 0, 0)
        first.append(f)
        k[b, :, :f], v[b, :, :f] = nan, nan
        k[b, :, ctx[b] + chunk[b]:], v[b, :, ctx[b] + chunk[b]:] = nan, nan
    x["k"], x["v"], x["table"] = k, v, None
    if page:
        n = B * (S // page)
        perm = torch.randperm(n + 3, generator=gen)
        table = perm[:n].reshape(B, -1).int()
        pools = []
        for cache in (k, v):
            pool = torch.full((n + 3, Hkv, page, D), nan, dtype=TYPES[dtype])
            pool[table.long().reshape(-1)] = cache.reshape(B, Hkv, S // page, page, D).transpose(1, 2).reshape(
                n, Hkv, page, D)
            pools.append(pool.to(d))
        for b in range(B):   # entries that nothing may be read through
            table[b, :first[b] // page] = int(perm[-1])
            table[b, -(-(ctx[b] + chunk[b]) // page):] = int(perm[-1])
        x["pools"], x["table"] = pools, table.to(d)
    x["slopes"] = 2.0 ** (-8.0 * torch.arange(1, Hq + 1) / Hq) if slopes else None
    return x


def call(x, softcap=0.0, **kw):
    d = dev()
    i32 = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device=d)   # noqa: E731
    k, v = x["pools"] if x["table"] is not None else (x["k"].to(d), x["v"].to(d))
    B, C, Hq, D = x["q"].shape
    out = torch.full((B, C, Hq, D), float("nan"), dtype=x["q"].dtype, device=d)
    lse = torch.full((B, C, Hq), float("nan"), device=d)
    got = pkg.verify_attn_scored(
        x["q"].to(d), k, v, i32(x["ctx"]), i32(x["chunk"]), x["scale"], softcap=softcap,
        slopes=None if x["slopes"] is None else x["slopes"].to(d), window=x["window"], starts=i32(x["starts"]),
        draft_mask=None if x["words"] is None else torch.from_numpy(x["words"].view(np.int64)).to(d),
        block_table=x["table"], out=out, lse=lse, check_lengths=True, **kw)
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is lse
    return out, lse


def check(x, out, lse, softcap=0.0, label="", rows=None):
    o, s = f64(out), f64(lse)
    B, C, Hq, D = o.shape
    g = Hq // x["k"].shape[1]
    h = torch.finfo(TYPES[x["dtype"]]).eps / 2
    h16 = h if x["dtype"] != "f32" else 0.0
    q, k, v = f64(x["q"]), x["k"].double().numpy(), x["v"].double().numpy()
    worst_o = worst_l = 0.0
    empty = 0
    for b in range(B):
        l, c = x["ctx"][b], x["chunk"][b]
        assert (o[b, c:] == 0).all() and (s[b, c:] == -np.inf).all(), f"{label}: padding rows of sequence {b}"
        if rows is not None and b not in rows:
            continue
        T = l + c
        start = min(x["starts"][b], l) if x["starts"] else 0
        for i in range(c):
            sees = np.arange(T) <= l + i
            if x["words"] is not None:
                sees[l:] = [(int(x["words"][b, i]) >> n) & 1 for n in range(c)]
            # (a token that sees no draft token stands like a root)
            extra = 1 if not sees[l:].any() else 0
            dist = sees.sum() - np.cumsum(sees) + extra
            keep = sees & (np.arange(T) >= start)
            if x["window"]:
                keep &= dist < x["window"]
            for hh in range(Hq):
                kk, vv = k[b, hh // g, :T][keep], v[b, hh // g, :T][keep]
                slope = 0.0 if x["slopes"] is None else float(x["slopes"][hh])
                if not keep.any():
                    assert (o[b, i, hh] == 0).all() and s[b, i, hh] == -np.inf, f"{label}: a row without keys"
                    empty += 1
                    continue
                # the kept keys, with their distances as a chain's (scored_row_ref
                # counts them itself when all are seen in a row)
                sc = kk @ q[b, i, hh] * x["scale"]
                sc = softcap * np.tanh(sc / softcap) if softcap else sc
                bias = slope * dist[keep]
                sc = sc - bias
                m = sc.max()
                p = np.exp(sc - m)
                z = p.sum()
                ref, ref_l = p @ vv / z, m + np.log(z)
                A = (np.abs(kk) @ np.abs(q[b, i, hh])).max() * x["scale"]
                near = bias[sc > m - 40].max()
                ds = 2.0 ** -24 * (D * A + 8 * (softcap + near) + 8)
                sums = (T / 4 + 64) * 2.0 ** -24 + 2.0 ** -21
                W = p @ np.abs(vv) / z
                tol = (2 * (ds + sums) + h16) * W + h * np.abs(ref) + (2.0 ** -24 if x["dtype"] == "f16" else 1e-30)
                tol_l = ds + sums + 2.0 ** -23 * abs(ref_l)
                worst_o = max(worst_o, (np.abs(o[b, i, hh] - ref) / tol).max())
                worst_l = max(worst_l, abs(s[b, i, hh] - ref_l) / tol_l)
                assert worst_o <= 1 and worst_l <= 1, f"{label} row {b, i, hh}: {worst_o:.2f} {worst_l:.2f} of the tolerance"
    note(f"[scored {label}] out {worst_o:.2f}, lse {worst_l:.2f} of the tolerance, {empty} rows without keys")


def run(seed, dtype, ctx, chunk, label="", softcap=0.0, slopes=False, window=0, starts=None, call_kw={}, rows=None, **kw):
    x = make(seed, dtype, ctx, chunk, slopes=slopes, window=window, starts=starts, **kw)
    out, lse = call(x, softcap, **call_kw)
    check(x, out, lse, softcap, label, rows)
    return x, out, lse


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tree,page,D", [(False, 0, 128), (True, 0, 64), (False, 16, 64), (True, 64, 128)])
@pytest.mark.parametrize("name", sorted(SETTINGS))
def test_settings(dtype, tree, page, D, name):
    run(1, dtype, [0, 37, 300, 129, 5], [6, 6, 3, 0, 1], f"{dtype} {tree} {page} {D} {name}", tree=tree, page=page, D=D,
        **SETTINGS[name])


def test_oracle_rows_agree():
    """The rows as this file computes them are the oracle's."""
    x = make(2, "f32", [40], [5], Hq=2, Hkv=1, D=64, tree=True, slopes=True, window=9, starts=[3])
    out, lse = call(x, 5.0)
    check(x, out, lse, 5.0, "one")
    for i in range(5):
        sees = np.ones(45, bool)
        sees[40:] = [(int(x["words"][0, i]) >> n) & 1 for n in range(5)]
        k, v = np.nan_to_num(f64(x["k"][0, 0, :45])), np.nan_to_num(f64(x["v"][0, 0, :45]))
        for h in range(2):
            o, l = scored_row_ref(f64(x["q"][0, i, h]), k, v, x["scale"], sees, 5.0, float(x["slopes"][h]), 9, 3)
            assert np.abs(o - f64(out[0, i, h])).max() < 1e-5 and abs(l - float(lse[0, i, h])) < 1e-5


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("window", [1, 2, 5, 16, 17, 127, 128, 129, 1 << 30])
def test_windows_at_chunk_and_tile_borders(window, tree):
    run(3, "bf16", [0, 3, 128, 250, 400, 127], [16, 9, 16, 1, 12, 5], f"window {window}", window=window, tree=tree, Hq=4,
        Hkv=2)


@pytest.mark.parametrize("page", [0, 8, 128])
def test_starts_at_every_place(page):
    ctx = [0, 1, 16, 130, 300, 300, 300]
    run(4, "f16", ctx, [3] * 7, f"starts, page {page}", starts=[0, 1, 40, 129, 300, 299, 0], page=page, window=200)


def test_tokens_that_see_nothing():
    x = make(5, "bf16", [20, 0, 9], [4, 3, 2], Hq=4, Hkv=2, tree=True, starts=[20, 0, 0], window=4)
    x["words"][0, 2] = 0   # its context is hidden, and no draft token is seen
    x["words"][1, 0] = 0
    out, lse = call(x, 10.0)
    check(x, out, lse, 10.0, "nothing")
    assert (lse[0, 2] == -np.inf).all() and (lse[1, 0] == -np.inf).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_far_past_the_cap(dtype):
    run(6, dtype, [300, 20], [5, 5], "large scores", softcap=4.0, q_scale=8.0, slopes=True)
    run(7, dtype, [300, 20], [5, 5], "scores of both kinds", softcap=15.0, q_scale=3.0)


@pytest.mark.parametrize("grid", [0, 1, 3, 40])
@pytest.mark.parametrize("tree", [False, True])
def test_cut_units(grid, tree):
    run(8, "bf16", [5000, 1700], [5, 8], f"grid {grid}", softcap=30.0, slopes=True, starts=[700, 0], tree=tree,
        call_kw=dict(grid_blocks=grid), Hq=4, Hkv=1)
    run(9, "f32", [3000], [3], f"grid {grid}, window", window=2100, tree=tree, call_kw=dict(grid_blocks=grid), Hq=2, Hkv=2,
        D=64)


@pytest.mark.parametrize("Hq,Hkv,C", [(1, 1, 1), (28, 4, 16), (32, 8, 5), (32, 32, 2), (64, 1, 2), (2, 1, 64)])
def test_head_layouts(Hq, Hkv, C):
    run(10, "bf16", [200, 90], [C, max(1, C // 2)], f"{Hq}/{Hkv} x {C}", Hq=Hq, Hkv=Hkv, tree=C > 1, **EVERYTHING)


def test_many_sequences_and_a_large_output():
    """More sequences than one launch takes, and results stored with device
    scope; a few sequences are compared."""
    rng = np.random.default_rng(11)
    B = 1100
    run(11, "bf16", rng.integers(0, 90, B).tolist(), rng.integers(0, 3, B).tolist(), "1100 sequences", Hq=2, Hkv=1, D=64,
        C=2, rows=[0, 1, 500, 1023, 1024, 1025, 1099], **dict(EVERYTHING, window=40))
    B = 260
    run(12, "bf16", rng.integers(0, 120, B).tolist(), rng.integers(9, 13, B).tolist(), "large output", Hq=32, Hkv=8, C=12,
        rows=[0, 130, 259], softcap=30.0, window=64)


def test_equals_the_plain_call_where_nothing_is_set():
    """Without settings the results are verify_attn's, but for the rounding to
    the inputs' type and the scores' scaling."""
    x = make(13, "bf16", [700, 333], [5, 4])
    out, lse = call(x)
    d = dev()
    ref, ref_l = pkg.verify_attn(x["q"].to(d), x["k"].to(d), x["v"].to(d),
                                 torch.tensor(x["ctx"], dtype=torch.int32, device=d),
                                 torch.tensor(x["chunk"], dtype=torch.int32, device=d), x["scale"])
    valid = torch.isfinite(ref_l)
    assert torch.equal(valid, torch.isfinite(lse))
    # (two roundings of the probabilities to bf16 may differ by a whole step)
    assert (out.float() - ref)[valid].abs().max() <= 2.0 ** -7 * ref[valid].abs().max()
    assert (lse - ref_l)[valid].abs().max() <= 1e-5


def test_repeats_streams_and_a_shared_workspace():
    d = dev()
    x = make(14, "bf16", [1500, 900, 40], [5, 5, 2], slopes=True)
    t = lambda a: torch.tensor(a, dtype=torch.int32, device=d)   # noqa: E731
    q, k, v, ctx, chunk, slopes = x["q"].to(d), x["k"].to(d), x["v"].to(d), t(x["ctx"]), t(x["chunk"]), x["slopes"].to(d)
    ws = pkg.alloc_scored_workspace(q, k)
    scored = lambda **kw: pkg.verify_attn_scored(q, k, v, ctx, chunk, x["scale"], softcap=9.0, slopes=slopes, window=700,   # noqa: E731
                                                 workspace=ws, **kw)
    first, first_l = scored()
    plain, plain_l = pkg.verify_attn(q, k, v, ctx, chunk, x["scale"], workspace=ws)
    for _ in range(3):
        a, b = scored()
        assert torch.equal(a, first) and torch.equal(b, first_l)
        c, e = pkg.verify_attn(q, k, v, ctx, chunk, x["scale"], workspace=ws)
        assert torch.equal(c, plain) and torch.equal(e, plain_l)
    s = torch.cuda.Stream(device=d)
    s.wait_stream(torch.cuda.current_stream(d))
    a, b = scored(stream=s)
    s.synchronize()
    assert torch.equal(a, first) and torch.equal(b, first_l)
    assert pkg.workspace_status(ws) == 0
    with pytest.raises(pkg.SpecMoEError):
        scored(flags=2)
    empty = torch.empty((0,), dtype=torch.int32, device=d)
    out, lse = pkg.verify_attn_scored(q[:0], k[:0], v[:0], empty, empty, x["scale"], softcap=1.0)
    assert out.shape == (0, 5, 8, 128) and out.dtype == torch.bfloat16


def test_nan_and_infinity_stay_in_their_sequence():
    """A NaN in one sequence's valid inputs reaches no other sequence."""
    x = make(15, "bf16", [300, 260], [4, 4], window=100)
    x["v"][0, :, 290] = float("nan")
    x["k"][0, 1, 280] = float("inf")
    out, lse = call(x, 10.0)
    x2 = dict(x, k=x["k"].clone(), v=x["v"].clone())
    x2["k"][0], x2["v"][0] = 0, 0
    out2, lse2 = call(x2, 10.0)
    assert torch.equal(out[1], out2[1]) and torch.equal(lse[1], lse2[1]) and torch.isfinite(out[1]).all()


def test_offsets_past_32_bits():
    """Caches of more than 2^32 bytes: the last sequence's rows, under a window
    that skips most of them."""
    d = dev()
    B, Hkv, S, D = 3, 8, 1 << 20, 128
    k = torch.zeros((B, Hkv, S, D), dtype=torch.bfloat16, device=d)
    v = torch.zeros_like(k)
    ctx, chunk = [40, 0, S - 3], [2, 2, 3]
    x = make(16, "bf16", [40, 0, 500], chunk, Hq=8, Hkv=8, window=100, slopes=True)
    x["ctx"] = ctx
    for b in range(B):
        n = [42, 2, 503][b]
        for big, small in ((k, x["k"]), (v, x["v"])):
            big[b, :, ctx[b] + chunk[b] - n:ctx[b] + chunk[b]] = torch.nan_to_num(small[b, :, :n].to(d))
    t = lambda a: torch.tensor(a, dtype=torch.int32, device=d)   # noqa: E731
    slopes = x["slopes"].to(d)
    out, lse = pkg.verify_attn_scored(x["q"].to(d), k, v, t(ctx), t(chunk), x["scale"], softcap=20.0, slopes=slopes,
                                      window=100, check_lengths=True)
    near, near_l = pkg.verify_attn_scored(x["q"].to(d), torch.nan_to_num(x["k"]).to(d), torch.nan_to_num(x["v"]).to(d),
                                          t([40, 0, 500]), t(chunk), x["scale"], softcap=20.0, slopes=slopes, window=100)
    torch.cuda.synchronize()
    # (the same keys at the same distances; other tiles, so other roundings of
    # the probabilities to bf16, one step each at most)
    assert torch.isfinite(out).all()
    valid = torch.isfinite(near_l)
    assert torch.equal(valid, torch.isfinite(lse)) and (lse - near_l)[valid].abs().max() <= 1e-5
    assert (out - near).abs().float().max() <= 2.0 ** -7 * torch.nan_to_num(x["v"]).abs().max().float().item()


def test_windows_past_32_bits_hide_nothing():
    x = make(17, "f32", [90, 5], [3, 2])
    want = call(x, 7.0)
    for window in (93, (1 << 31) - 1, 1 << 31, (1 << 32) + 1, 1 << 40):
        got = call(dict(x, window=window), 7.0)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for window in (-1, -(1 << 32)):
        with pytest.raises(pkg.SpecMoEError):
            call(dict(x, window=window), 7.0)
