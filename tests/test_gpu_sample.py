"""sample, accept_sample and accept_sample_tree on the GPU against the float64
oracle.

Tokens are equal.  (The kernel's sums are off by at most V 2^-43 of the best
token's weight and its weights by 2^-45; the seeds' uniforms keep clear of the
borders by far more.)  Log-probabilities are computed in fp64 from sums that
are off by at most V 2^-43 and rounded once: |error| <= 2^-24 |value| + V 2^-42
(the second term where the value is near 0), doubled for the oracle's own."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
from oracle.step import accept_sample_ref, sample_ref
from test_gpu_parity import dev, note
from paper_2508_21706_amd import workloads as wl

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def f64(t):
    return t.detach().cpu().double().numpy()


def on(a, dt=None):
    t = torch.as_tensor(np.asarray(a)) if not torch.is_tensor(a) else a
    return t.to(dev()) if dt is None else t.to(dt).to(dev())


def check_rows(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, label=""):
    """logits [N, V] on the GPU (possibly strided); settings as lists."""
    N, V = logits.shape
    arr = dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    put = {n: None if v is None else on(np.asarray(v), torch.int32 if n == "top_k" else torch.float32)
           for n, v in arr.items()}
    out = (torch.full((N,), -7, dtype=torch.int32, device=dev()), torch.full((N,), float("nan"), device=dev()))
    token, logp = pkg.sample(logits, on(np.asarray(u), torch.float32), out=out, **put)
    torch.cuda.synchronize()
    token, logp, x = token.cpu().numpy(), f64(logp), f64(logits)
    rows = np.asarray(u, np.float32).astype(np.float64)
    settings = {n: None if v is None else f64(put[n]) for n, v in arr.items()}
    for r in range(N):
        kw = {n: v[r] for n, v in settings.items() if v is not None}
        want, lp = sample_ref(x[r], rows[r], **kw)
        assert token[r] == want, f"{label} row {r}: token {token[r]}, oracle {want}, {kw}, u {rows[r]}"
        if np.isfinite(lp):
            assert abs(logp[r] - lp) <= 2 * (2.0 ** -24 * abs(lp) + V * 2.0 ** -42), f"{label} row {r}: {logp[r]} {lp}"
        else:
            assert logp[r] == lp
    note(f"[sample {label}] {N} rows of {V}")


def rows_of(seed, N, V, dtype, scale=2.0, top=None):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((N, V), generator=gen) * scale
    if top is not None:
        x[torch.arange(N), torch.randint(0, V, (N,), generator=gen)] = top
    return x.to(TYPES[dtype]).to(dev()), torch.rand((N,), generator=gen).numpy()


SETTINGS = {
    "plain": {},
    "cold": dict(temperature=0.3),
    "hot": dict(temperature=50.0),
    "k1": dict(top_k=1),
    "k40": dict(top_k=40, temperature=0.8),
    "k200": dict(top_k=200),
    "k300": dict(top_k=300),
    "k5000": dict(top_k=5000, temperature=1.5),
    "k_all": dict(top_k=1 << 30),
    "p90": dict(top_p=0.9),
    "p999": dict(top_p=0.999, temperature=1.3),
    "p01": dict(top_p=0.01),
    "m05": dict(min_p=0.05),
    "m_all": dict(min_p=1.0),
    "all": dict(temperature=0.9, top_k=50, top_p=0.9, min_p=0.02),
    "all_wide": dict(temperature=1.2, top_k=2000, top_p=0.95, min_p=0.001),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 8191, 32000, 36865])
def test_settings(dtype, V):
    for n, (name, kw) in enumerate(SETTINGS.items()):
        logits, u = rows_of(n, 6, V, dtype, top=9.0 if n % 2 else None)
        check_rows(logits, u, **{k: [v] * 6 for k, v in kw.items()}, label=f"{dtype} {name}")


@pytest.mark.parametrize("dtype,V", [("bf16", 50257), ("bf16", 73729), ("bf16", 151936), ("f32", 50257), ("f32", 262143)])
def test_long_rows(dtype, V):
    logits, u = rows_of(3, 4, V, dtype, scale=3.0)
    check_rows(logits, u, label=f"{dtype} plain")
    check_rows(logits, u, temperature=[0.7] * 4, top_k=[0, 50, 300, 1], top_p=[0.9, 1.0, 0.95, 0.5],
               min_p=[0.0, 0.01, 0.0, 0.3], label=f"{dtype} mixed")


def test_each_row_its_own_settings():
    N = 40
    logits, u = rows_of(5, N, 32000, "bf16", top=10.0)
    rng = np.random.default_rng(6)
    check_rows(logits, u, temperature=rng.choice([0.0, 0.5, 1.0, 1.4], N), top_k=rng.choice([-1, 0, 1, 20, 400], N),
               top_p=rng.choice([0.0, 0.3, 0.9, 1.0, 2.0], N), min_p=rng.choice([-1.0, 0.0, 0.1, 2.0], N), label="mix")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_and_nearly_equal_logits(dtype):
    """Ties go to the lowest index, whatever their number: one value, two
    values, a few neighbouring ones, in rows that are read again and in rows
    that stay in LDS."""
    for V in (300, 5000, 32000, 150001):
        u = np.float32([0.0, 0.2, 0.71, 0.9999])
        flat = torch.full((4, V), 1.5, dtype=TYPES[dtype], device=dev())
        check_rows(flat, u, label="flat")
        check_rows(flat, u, top_k=[200, 270, V - 1, 2], label="flat, top_k")
        check_rows(flat, u, top_p=[0.3] * 4, top_k=[0, 0, V // 2, 3], label="flat, top_p")
        two = flat.clone()
        two[:, ::3] = -1.25
        check_rows(two, u, label="two")
        check_rows(two, u, top_k=[V // 2] * 4, top_p=[0.9] * 4, temperature=[100.0] * 4, label="two, wide")
        step = torch.arange(V, device=dev()) * 7919 % 5
        near = (1024 + step * (8 if dtype == "bf16" else 2.0 ** -13)).to(TYPES[dtype]).repeat(4, 1)
        check_rows(near, u, temperature=[1e4] * 4, label="near")
        check_rows(near, u, temperature=[1e4] * 4, top_k=[V // 3 + 1] * 4, label="near, top_k")


def test_infinities_and_nan():
    inf, nan = float("inf"), float("nan")
    V = 700
    x = torch.randn((9, V), generator=torch.Generator().manual_seed(1))
    x[0, 1:] = -inf                       # one token left
    x[1, ::2] = -inf
    x[2] = -inf                           # no mass
    x[3] = nan
    x[4, 5:600] = nan
    x[5, 17] = inf                        # one infinity takes all, two share it
    x[6, [3, 650]] = inf
    x[7, :] = torch.finfo(torch.float32).min
    x[7, 30:33] = 2.0
    x[8, ::3], x[8, 1] = -0.0, 0.0
    x[8].clamp_(max=0.0)
    u = np.float32([0.3, 0.6, 0.1, 0.1, 0.7, 0.5, 0.6, 0.9, 0.02])
    for kw in ({}, dict(top_k=[5] * 9), dict(top_k=[400] * 9), dict(top_p=[0.8] * 9), dict(min_p=[0.5] * 9),
               dict(temperature=[3.0] * 9), dict(temperature=[inf] * 9), dict(temperature=[1e-38] * 9)):
        check_rows(x.to(dev()), u, **kw, label=str(kw)[:30])
    # greedy elects what accept_greedy does; NaN settings are off
    got = pkg.sample(x.to(dev()), on(u), temperature=on(np.float32([0.0] * 9)))[0].tolist()
    rows = torch.where(x.isnan(), torch.tensor(-inf), x)
    assert got == [0, int(rows[1].argmax()), 0, -1, int(rows[4].argmax()), 17, 3, 30, 0]
    a, la = pkg.sample(x.to(dev()), on(u))
    b, lb = pkg.sample(x.to(dev()), on(u), top_p=on(np.float32([nan] * 9)), min_p=on(np.float32([nan] * 9)))
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_uniforms_at_and_past_their_ends():
    logits, _ = rows_of(9, 6, 4096, "f32", scale=1.0)
    order = torch.argsort(logits, dim=1, descending=True, stable=True)
    below = np.float32(1.0) - np.float32(2.0 ** -24)
    u = np.float32([0.0, -1.0, float("nan"), below, 1.0, 5.0])
    token = pkg.sample(logits, on(u), top_k=on(np.int32([30] * 6)))[0]
    assert [int((order[r] == token[r]).nonzero()) for r in range(6)] == [0, 0, 0, 29, 29, 29]
    token = pkg.sample(logits, on(u))[0]
    assert [int((order[r] == token[r]).nonzero()) for r in range(6)][:3] == [0, 0, 0]
    assert [int((order[r] == token[r]).nonzero()) for r in (4, 5)] == [4095, 4095]


def test_strides_and_odd_starts():
    base = torch.randn((5, 3, 1003), generator=torch.Generator().manual_seed(2)).to(dev())
    u = np.float32([0.1, 0.4, 0.6, 0.8, 0.95])
    for dtype in ("f32", "bf16"):
        wide = base.to(TYPES[dtype])
        check_rows(wide[:, 2, 1:1001], u, top_p=[0.9] * 5, label=f"{dtype} strided")
        check_rows(wide[:, 1, 3:4], u, label=f"{dtype} one column")


def test_results_do_not_depend_on_timing_or_neighbours():
    logits, u = rows_of(11, 96, 32000, "bf16", scale=1.0)
    p = on(np.full(96, 0.95, np.float32))
    t0, l0 = pkg.sample(logits, on(u), top_p=p)
    for _ in range(3):
        t, l = pkg.sample(logits, on(u), top_p=p)
        assert torch.equal(t, t0) and torch.equal(l, l0)
    t, l = pkg.sample(logits[17:18], on(u[17:18]), top_p=p[:1])
    assert int(t) == int(t0[17]) and float(l) == float(l0[17])


def make_chunks(seed, dtype, B, C, V, chunk, tree):
    rng = np.random.default_rng(seed)
    gen = torch.Generator().manual_seed(seed)
    logits = torch.randn((B, C, V), generator=gen) * 1.5
    won = rng.integers(0, V, size=(B, C))
    logits.scatter_(2, torch.from_numpy(won)[..., None], 12.0)
    words = wl.tree_draft_masks(seed, np.asarray(chunk), C) if tree else None
    tokens = rng.integers(0, V, size=(B, C))
    for b in range(B):
        for i in range(1, chunk[b]):
            parent = i - 1
            if tree:
                parent = (int(words[b, i]) & ((1 << i) - 1)).bit_length() - 1
            if rng.random() < 0.7:
                tokens[b, i] = won[b, parent]
    return (logits.to(TYPES[dtype]).to(dev()), on(tokens, torch.int32), on(rng.integers(0, 100, B), torch.int32),
            on(np.asarray(chunk), torch.int32), on(rng.random((B, C)), torch.float32), words)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("C,V,chunk", [(1, 1000, [1, 0, 1]), (5, 32000, [5, 0, 3, 1, 5]), (64, 512, [64, 17, 33, 0]),
                                       (8, 40000, [8, 8])])
def test_acceptance(dtype, tree, C, V, chunk):
    B = len(chunk)
    logits, tokens, ctx, cl, u, words = make_chunks(7, dtype, B, C, V, chunk, tree)
    rng = np.random.default_rng(8)
    settings = dict(temperature=on(rng.choice([0.0, 0.4, 0.9], B), torch.float32),
                    top_k=on(rng.choice([0, 1, 30], B), torch.int32),
                    top_p=on(rng.choice([0.7, 0.95, 1.0], B), torch.float32),
                    min_p=on(rng.choice([0.0, 0.05], B), torch.float32))
    ws = pkg.alloc_accept_workspace(pkg.accept_desc(B, C, V, {"f32": 0, "bf16": 1}[dtype]), dev())
    per = [{n: float(f64(v)[b]) for n, v in settings.items()} for b in range(B)]
    want = accept_sample_ref(f64(logits), tokens.cpu().numpy(), ctx.tolist(), chunk, f64(u), per, words)
    for _ in range(3):   # the workspace serves call after call, and the greedy call between them
        if tree:
            mask = on(words.view(np.int64))
            got = pkg.accept_sample_tree(logits, tokens, mask, ctx, cl, u, workspace=ws, **settings)
            assert torch.equal(got["path"].cpu(), torch.from_numpy(want["path"]))
        else:
            got = pkg.accept_sample(logits, tokens, ctx, cl, u, workspace=ws, **settings)
            assert "path" not in got
        for key in ("sampled", "accepted", "next_token", "new_ctx_lens"):
            assert got[key].cpu().tolist() == want[key].tolist(), key
        err = np.abs(f64(got["logprobs"]) - want["logprobs"])
        assert (err <= 2 * (2.0 ** -24 * np.abs(want["logprobs"]) + V * 2.0 ** -42)).all()
        pkg.accept_greedy(logits, tokens, ctx, cl, workspace=ws)
    note(f"[accept {dtype} {'tree' if tree else 'chain'}] accepted {want['accepted'].tolist()} of {chunk}")


@pytest.mark.parametrize("tree", [False, True])
def test_temperature_zero_is_greedy_acceptance(tree):
    chunk = [6, 6, 2, 0, 5]
    logits, tokens, ctx, cl, u, words = make_chunks(9, "bf16", 5, 6, 2048, chunk, tree)
    cold = torch.zeros((5,), device=dev())
    if tree:
        mask = on(words.view(np.int64))
        a = pkg.accept_greedy_tree(logits, tokens, mask, ctx, cl)
        b = pkg.accept_sample_tree(logits, tokens, mask, ctx, cl, u, temperature=cold)
        assert torch.equal(a["path"], b["path"])
    else:
        a = pkg.accept_greedy(logits, tokens, ctx, cl)
        b = pkg.accept_sample(logits, tokens, ctx, cl, u, temperature=cold, in_place=True)
        assert b["new_ctx_lens"] is ctx
    assert torch.equal(a["argmax"], b["sampled"])
    for key in ("accepted", "next_token", "new_ctx_lens"):
        assert torch.equal(a[key], b[key]), key
    assert not b["logprobs"].any()


def test_long_chunks_and_large_batches():
    """Chunks past 64 positions, and more sequences than a grid's rows wait for."""
    chunk = [200, 130, 64, 65]
    logits, tokens, ctx, cl, u, _ = make_chunks(10, "f32", 4, 200, 64, chunk, False)
    sampled = pkg.sample(logits.view(-1, 64), u.view(-1), temperature=torch.full((800,), 0.3, device=dev()))[0]
    tokens[:, 1:] = sampled.view(4, 200)[:, :-1]   # every draft is right, but one
    tokens[1, 70] += 1
    per = [dict(temperature=float(np.float32(0.3)))] * 4
    want = accept_sample_ref(f64(logits), tokens.cpu().numpy(), ctx.tolist(), chunk, f64(u), per)
    got = pkg.accept_sample(logits, tokens, ctx, cl, u, temperature=torch.full((4,), 0.3, device=dev()))
    for key in ("sampled", "accepted", "next_token", "new_ctx_lens"):
        assert got[key].cpu().tolist() == want[key].tolist(), key
    assert want["accepted"].tolist() == [199, 69, 63, 64]
    B = 3000
    logits, tokens, ctx, cl, u, _ = make_chunks(11, "bf16", B, 2, 64, [2] * B, False)
    got = pkg.accept_sample(logits, tokens, ctx, cl, u)
    want = accept_sample_ref(f64(logits), tokens.cpu().numpy(), ctx.tolist(), [2] * B, f64(u), [{}] * B)
    for key in ("sampled", "accepted", "next_token", "new_ctx_lens"):
        assert got[key].cpu().tolist() == want[key].tolist(), key


def test_distribution_of_accepted_tokens():
    """What a sequence takes is distributed as token-by-token sampling: the
    first token of a two-token chunk over many uniforms has the target's
    probabilities, accepted or not."""
    V, N = 16, 40000
    gen = torch.Generator().manual_seed(3)
    logits = torch.randn((1, 2, V), generator=gen).repeat(N, 1, 1).to(dev())
    tokens = torch.zeros((N, 2), dtype=torch.int32, device=dev())
    tokens[:, 1] = int(logits[0, 0].argmax())
    u = torch.rand((N, 2), generator=gen).to(dev())
    zero, two = (torch.full((N,), n, dtype=torch.int32, device=dev()) for n in (0, 2))
    got = pkg.accept_sample(logits, tokens, zero, two, u)
    first = torch.where(got["accepted"] == 1, tokens[:, 1], got["next_token"]).long()
    share = torch.bincount(first, minlength=V).double() / N
    p = torch.softmax(logits[0, 0].double(), 0)
    # a share's standard deviation is at most 0.5 / sqrt(N); six of them
    assert (share - p).abs().max() < 6 * 0.5 / N ** 0.5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bins_around_zero_and_far_apart(dtype):
    """Rows whose numbers have more patterns than there are bins: many around 0,
    of one sign, of far apart sizes, and infinities beside NaN."""
    V, N = 6000, 8
    gen = torch.Generator().manual_seed(21)
    z = torch.randn((N, V), generator=gen)
    u = torch.rand((N,), generator=gen).numpy()
    rows = {"small": z * 1e-3, "tiny": z * 1e-30, "sizes": z.sign() * 10.0 ** (z.abs() * 8 - 12),
            "negative": -10.0 ** (z * 3), "positive": 10.0 ** (z * 3 - 6), "wide": z.sign() * 10.0 ** (z.abs() * 12 - 10)}
    near = z.clone()
    near[:, ::2] *= 2.0 ** -20
    rows["half near 0"] = near
    mixed = z.clone()
    mixed[:, ::5], mixed[:, 1::7] = float("inf"), float("nan")
    rows["infinities"] = mixed
    for name, x in rows.items():
        x = x.to(TYPES[dtype]).to(dev())
        for kw in ({}, dict(temperature=[30.0] * N), dict(temperature=[1e6] * N), dict(top_k=[700] * N, top_p=[0.8] * N),
                   dict(top_k=[60] * N), dict(min_p=[0.4] * N, temperature=[5.0] * N)):
            check_rows(x, u, **kw, label=f"{dtype} {name} {str(kw)[:24]}")


@pytest.mark.parametrize("V", [2000, 32000, 80001])
def test_tokens_around_zero(V):
    """bf16 logits next to 0, which share one bin: many zeros, many distinct
    numbers, with and without weight, and counts that end among them."""
    gen = torch.Generator().manual_seed(V)
    u = np.float32([0.03, 0.31, 0.62, 0.97])
    tiny = (torch.rand((4, V), generator=gen) - 0.5) * 2.0 ** -10
    zeros = torch.where(torch.rand((4, V), generator=gen) < 0.5, tiny, torch.tensor(0.0))
    few = torch.randint(0, V, (4, 200), generator=gen)
    for name, x in (("distinct", tiny), ("zeros", zeros), ("signed zeros", torch.copysign(torch.zeros(4, V), tiny))):
        x = x.to(torch.bfloat16).to(dev())
        check_rows(x, u, label=f"{name}")
        check_rows(x, u, temperature=[2.0 ** -13, 2.0 ** -12, 2.0 ** -11, 1e-6], label=f"{name}, cold")
        check_rows(x, u, top_k=[V // 2, 129, 400, V - 1], top_p=[0.9] * 4, label=f"{name}, top_k")
        for top in (8.0, 40.0):   # a few tokens far above: those around 0 weigh e^-8 and nothing
            y = x.clone().scatter_(1, few.to(dev()), (top - torch.arange(200) / 64.0).repeat(4, 1).bfloat16().to(dev()))
            check_rows(y, u, label=f"{name}, {top}")
            check_rows(y, u, top_k=[150, 199, 500, V - 1], label=f"{name}, {top}, top_k")
            check_rows(y, u, top_k=[V // 2] * 4, top_p=[0.9] * 4, min_p=[0.01] * 4, label=f"{name}, {top}, all")
            check_rows(y, u, temperature=[30.0] * 4, top_k=[0, 0, 900, V // 3], label=f"{name}, {top}, hot")


@pytest.mark.parametrize("V", [900, 32000, 80001])
def test_maxima_and_minima_at_the_ends_of_the_bins(V):
    gen = torch.Generator().manual_seed(V + 1)
    x = torch.randn((10, V), generator=gen)
    u = torch.rand((10,), generator=gen).numpy()
    at = torch.randint(0, V, (10,), generator=gen)
    for r, top in enumerate([63.5, 63.75, 64.0, 100.0, 1e4]):
        x[r] *= 8.0
        x[r, at[r]] = top
    x[5] -= 62.0          # around the lowest bins, below them, and far below
    x[6] -= 90.0
    x[7] -= 1e5
    x[8] *= 30.0          # weights that reach below the lowest bins
    x[9] = x[9] * 0.5 - 64.0
    x = x.to(torch.bfloat16).to(dev())
    for kw in ({}, dict(temperature=[4.0] * 10), dict(temperature=[60.0] * 10), dict(temperature=[0.05] * 10),
               dict(top_k=[300] * 10), dict(top_k=[10] * 10), dict(top_p=[0.97] * 10, temperature=[2.5] * 10),
               dict(min_p=[0.003] * 10, top_k=[500] * 10)):
        check_rows(x, u, **kw, label=str(kw)[:30])


def test_infinities_and_nan_in_bf16():
    inf, nan = float("inf"), float("nan")
    V = 700
    x = torch.randn((12, V), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    x[0, 1:] = -inf
    x[1, ::2] = -inf
    x[2] = -inf
    x[3] = nan
    x[4, 5:600] = nan
    x[5, 17] = inf
    x[6, [3, 650]] = inf
    x[7, :] = torch.finfo(torch.bfloat16).min
    x[7, 30:33] = 2.0
    x[8, ::3], x[8, 1] = -0.0, 0.0
    x[8].clamp_(max=0.0)
    bits = x.view(torch.int16)
    bits[9, ::5], bits[9, 1::5] = -1, 0x7f81       # NaN of both signs, quiet and signalling
    bits[10] = -1
    bits[11, ::2], bits[11, 1::2] = -64, -128      # NaN with the sign, and -inf
    u = np.float32([0.3, 0.6, 0.1, 0.1, 0.7, 0.5, 0.6, 0.9, 0.02, 0.4, 0.2, 0.8])
    for kw in ({}, dict(top_k=[5] * 12), dict(top_k=[400] * 12), dict(top_p=[0.8] * 12), dict(min_p=[0.5] * 12),
               dict(temperature=[3.0] * 12), dict(temperature=[inf] * 12), dict(temperature=[1e-38] * 12)):
        check_rows(x.to(dev()), u, **kw, label=str(kw)[:30])


def test_offsets_past_32_bits():
    """More than 2^32 bytes of logits: the rows around 2^32 and the last ones
    are drawn as they are alone."""
    N, V, d = 70000, 32000, dev()
    logits = torch.empty((N, V), dtype=torch.bfloat16, device=d)
    gen = torch.Generator(device=d).manual_seed(12)
    for r in range(0, N, 10000):
        logits[r:r + 10000].normal_(std=2.0, generator=gen)
    u = torch.rand((N,), generator=gen, device=d)
    top_p = torch.full((N,), 0.9, device=d)
    token, logp = pkg.sample(logits, u, top_p=top_p)
    torch.cuda.synchronize()
    for r in (0, 33553, 67108, 67109, 69990):   # (2^31 and 2^32 bytes: rows 33554 and 67108)
        t, l = pkg.sample(logits[r:r + 3].clone(), u[r:r + 3].clone(), top_p=top_p[:3])
        assert torch.equal(t, token[r:r + 3]) and torch.equal(l, logp[r:r + 3])
    check_rows(logits[-2:], u[-2:].cpu().numpy(), top_p=[0.9] * 2, label="past 2^32")
