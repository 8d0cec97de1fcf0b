"""Rows of large batches, which share their CU with another row and are drawn by
half as many threads, give what they give alone."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
import test_gpu_sample as sampling
from oracle.step import accept_sample_ref
from test_gpu_parity import dev, note

pytestmark = pytest.mark.gpu

# One token of logit 12 and n of another, and a u at which the mass passed lies
# next to a token's end: temperature, the other's bf16 bits, 2^24 u, n.  (One
# unit of 2^-42 more in the weight of the n moves the place of the token drawn.)
BORDERS = [(0.699999988, 0x4121, 5875205, 18194), (0.699999988, 0x4121, 8732259, 9429),
           (0.703700006, 0x4120, 11056677, 9840), (0.703700006, 0x4133, 1218151, 9282),
           (0.707399964, 0x413b, 12914719, 28245), (0.711099982, 0x4128, 652191, 12320),
           (0.711099982, 0x4128, 10296431, 14173), (0.733299971, 0x4129, 8465595, 2728),
           (0.736999989, 0x4139, 5346779, 21181), (0.762899995, 0x4139, 9927615, 30875),
           (0.818399966, 0x4122, 6323159, 746), (0.851700008, 0x4122, 8838141, 6299)]


@pytest.mark.parametrize("T,bits,u24,n", BORDERS)
def test_draws_next_to_a_border_do_not_depend_on_the_batch(T, bits, u24, n):
    d, N = dev(), 300
    row = torch.full((n + 1,), bits, dtype=torch.int16).view(torch.bfloat16)
    row[0] = 12.0
    logits = row.to(d).repeat(N, 1)
    u = torch.full((N,), u24 / 2.0 ** 24, device=d)
    t = torch.full((N,), T, device=d)
    token, logp = pkg.sample(logits, u, temperature=t)
    alone, alone_p = pkg.sample(logits[:1], u[:1], temperature=t[:1])
    torch.cuda.synchronize()
    note(f"[border {T} {bits:#x}] {int(alone)} alone, {int(token[0])} in a batch of {N}")
    assert (token == alone).all() and (logp == alone_p).all()


def copies_of(rows, least=257):
    return -(-least // len(rows))


@pytest.fixture
def in_a_large_batch(monkeypatch):
    """``check_rows`` of the sampling tests over copies of the rows in a batch of
    more than 256, each of which gives what the row gives in its own call; the
    oracle is asked once."""
    check_alone = sampling.check_rows

    def check(logits, u, label="", **settings):
        d, N, V = dev(), *logits.shape
        times = copies_of(logits)
        put = {n: torch.from_numpy(np.asarray(v, np.int32 if n == "top_k" else np.float32)).to(d)
               for n, v in settings.items() if v is not None}
        u_d = torch.from_numpy(np.asarray(u, np.float32)).to(d)
        own = pkg.sample(logits, u_d, **put)
        many = pkg.sample(logits.repeat(times, 1), u_d.repeat(times), **{n: v.repeat(times) for n, v in put.items()})
        torch.cuda.synchronize()
        for name, a, b in zip(("token", "log-probability"), own, many):
            rows = (a.repeat(times) != b).nonzero().flatten().tolist()
            assert not rows, f"{label}: {name} of row {rows[0] % N} of {N} x {V}, copy {rows[0] // N}"
        check_alone(logits, u, label=label, **settings)

    monkeypatch.setattr(sampling, "check_rows", check)


# (short rows: those of up to 64000 bytes in bf16, 56320 in fp32)
@pytest.mark.parametrize("dtype,V", [("bf16", 1), ("bf16", 7), ("bf16", 1000), ("bf16", 8191), ("bf16", 32000),
                                     ("f32", 2), ("f32", 64), ("f32", 1001), ("f32", 8191), ("f32", 14080)])
def test_settings(in_a_large_batch, dtype, V):
    sampling.test_settings(dtype, V)


def test_each_row_its_own_settings(in_a_large_batch):
    sampling.test_each_row_its_own_settings()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_and_nearly_equal_logits(in_a_large_batch, dtype):
    sampling.test_equal_and_nearly_equal_logits(dtype)


def test_infinities_and_nan(in_a_large_batch):
    sampling.test_infinities_and_nan()
    sampling.test_infinities_and_nan_in_bf16()


def test_strides_and_odd_starts(in_a_large_batch):
    sampling.test_strides_and_odd_starts()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bins_around_zero_and_far_apart(in_a_large_batch, dtype):
    sampling.test_bins_around_zero_and_far_apart(dtype)


@pytest.mark.parametrize("V", [2000, 32000])
def test_tokens_around_zero(in_a_large_batch, V):
    sampling.test_tokens_around_zero(V)


@pytest.mark.parametrize("V", [900, 32000])
def test_maxima_and_minima_at_the_ends_of_the_bins(in_a_large_batch, V):
    sampling.test_maxima_and_minima_at_the_ends_of_the_bins(V)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("B,C,V", [(40, 7, 1000), (5, 64, 512), (80, 4, 14080)])
def test_acceptance(dtype, tree, B, C, V):
    """Ragged chunks with each sequence's own settings, more than 256 positions;
    the tokens are also those that a call of one sequence draws."""
    rng = np.random.default_rng(B + C)
    chunk = rng.integers(0, C + 1, B)
    chunk[:2] = C, 0
    logits, tokens, ctx, cl, u, words = sampling.make_chunks(12, dtype, B, C, V, chunk.tolist(), tree)
    on, f64 = sampling.on, sampling.f64
    settings = dict(temperature=on(rng.choice([0.0, 0.4, 0.9, 1.5], B), torch.float32),
                    top_k=on(rng.choice([0, 1, 30, 300], B), torch.int32),
                    top_p=on(rng.choice([0.7, 0.95, 1.0], B), torch.float32),
                    min_p=on(rng.choice([0.0, 0.05], B), torch.float32))
    mask = on(words.view(np.int64)) if tree else None

    def accept(s):
        pick = {n: v[s] for n, v in settings.items()}
        if tree:
            return pkg.accept_sample_tree(logits[s], tokens[s], mask[s], ctx[s], cl[s], u[s], **pick)
        return pkg.accept_sample(logits[s], tokens[s], ctx[s], cl[s], u[s], **pick)

    got = accept(slice(0, B))
    per = [{n: float(f64(v)[b]) for n, v in settings.items()} for b in range(B)]
    want = accept_sample_ref(f64(logits), tokens.cpu().numpy(), ctx.tolist(), chunk.tolist(), f64(u), per, words)
    for key in ("sampled", "accepted", "next_token", "new_ctx_lens"):
        assert got[key].cpu().tolist() == want[key].tolist(), key
    if tree:
        assert torch.equal(got["path"].cpu(), torch.from_numpy(want["path"]))
    # (as the sampling tests derive it: one rounding to 32 bits, sums of V weights)
    err = np.abs(f64(got["logprobs"]) - want["logprobs"])
    assert (err <= 2 * (2.0 ** -24 * np.abs(want["logprobs"]) + V * 2.0 ** -42)).all()
    for b in range(0, B, 9):
        one = accept(slice(b, b + 1))
        for key, t in one.items():
            assert torch.equal(t[0], got[key][b]), f"{key} of sequence {b}"
    note(f"[accept {dtype} {B} x {C} {'tree' if tree else 'chain'}] accepted {want['accepted'].sum()} of {chunk.sum()}")
