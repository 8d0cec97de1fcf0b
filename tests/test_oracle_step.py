"""Pins of the oracle of the operators around the verification attention:
closed forms, library routines and invariants."""
import math

import numpy as np
import pytest
import torch

from oracle import (accept_greedy_ref, accept_sample_ref, accept_tree_ref, head_ref, positions_ref, sample_ref,
                    scored_attn_ref, verify_attn_ref)


def test_rotation_is_a_rotation():
    rng = np.random.default_rng(1)
    inv = 1.0 / 10000.0 ** (np.arange(0, 16, 2) / 16)
    x, y = rng.standard_normal((2, 24))
    for rope in ("halves", "pairs"):
        assert np.array_equal(head_ref(x, 0, inv, rope), x)
        r = head_ref(x, 11, inv, rope)
        assert np.array_equal(r[16:], x[16:]) and math.isclose(r @ r, x @ x)
        # a product of two rotated rows depends on the distance alone
        a = head_ref(x, 11, inv, rope) @ head_ref(y, 4, inv, rope)
        b = head_ref(x, 907, inv, rope) @ head_ref(y, 900, inv, rope)
        assert math.isclose(a, b, rel_tol=1e-9)
        # and the complex numbers of its pairs are turned
        at = (slice(0, 8), slice(8, 16)) if rope == "halves" else (slice(0, 16, 2), slice(1, 16, 2))
        z = (x[at[0]] + 1j * x[at[1]]) * np.exp(11j * inv)
        np.testing.assert_allclose(r[at[0]] + 1j * r[at[1]], z, rtol=1e-12)


def test_norm_matches_the_library():
    rng = np.random.default_rng(2)
    x, w = rng.standard_normal((2, 64))
    want = torch.nn.functional.rms_norm(torch.from_numpy(x), (64,), torch.from_numpy(w), eps=1e-3)
    np.testing.assert_allclose(head_ref(x, 5, None, weight=w, eps=1e-3), want.numpy(), rtol=1e-12)


def test_positions():
    assert positions_ref(7, 3) == [7, 8, 9]
    # root, two children, a grandchild, and a word without a bit
    assert positions_ref(7, 5, [0b1, 0b11, 0b101, 0b1011, 0]) == [7, 8, 8, 9, 7]
    assert positions_ref(7, 2, [0b1, 0b110]) == [7, 7]   # bits past the chunk do not count


def rand_attn(seed=3, B=2, C=4, Hq=4, Hkv=2, D=8, S=12):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((B, C, Hq, D)), rng.standard_normal((B, Hkv, S, D)), rng.standard_normal((B, Hkv, S, D)),
            [3, 8], [4, 2])


def test_scored_attention_without_settings_is_the_attention():
    q, k, v, ctx, chunk = rand_attn()
    words = np.uint64([[1, 3, 5, 11], [1, 3, 0, 0]])
    for w in (None, words):
        o, l = scored_attn_ref(q, k, v, ctx, chunk, 0.5, words=w)
        f = lambda x: x.astype(np.float32)   # noqa: E731
        ro, rl = verify_attn_ref(f(q), f(k), f(v), np.int32(ctx), np.int32(chunk), 0.5, "f32", draft_mask=w)
        np.testing.assert_allclose(o, ro, atol=1e-6)
        np.testing.assert_allclose(l, rl, atol=1e-6)


def test_scored_attention_against_a_written_bias():
    """One sequence as a plain softmax with the caps, the bias and the hidden
    keys written out as matrices."""
    q, k, v, ctx, chunk = rand_attn(4)
    l, c, g = ctx[0], chunk[0], 2
    T = l + c
    slopes = np.array([0.5, 0.25, 0.125, 1.0])
    o, lse = scored_attn_ref(q, k, v, ctx, chunk, 0.5, softcap=2.0, slopes=slopes, window=3, starts=[2, 0])
    i, j = np.mgrid[:c, :T]
    far = l + i - j
    hidden = (far < 0) | (far >= 3) | (j < 2)
    for h in range(4):
        s = 2.0 * np.tanh(0.5 * q[0, :, h] @ k[0, h // g, :T].T / 2.0) - slopes[h] * far
        s = torch.from_numpy(np.where(hidden, -np.inf, s))
        np.testing.assert_allclose(lse[0, :, h], torch.logsumexp(s, 1).numpy(), rtol=1e-12)
        np.testing.assert_allclose(o[0, :, h], (torch.softmax(s, 1) @ torch.from_numpy(v[0, h // g, :T])).numpy(), rtol=1e-10)


def test_scored_tree_equals_chains_over_its_paths():
    q, k, v, _, _ = rand_attn(5, B=1, C=5, S=12)
    l, c = 6, 5
    words = np.uint64([[1, 0b11, 0b101, 0b1011, 0b10101]])
    kw = dict(softcap=3.0, slopes=np.array([0.3, 0.1, 0.7, 0.2]), window=4)
    o, lse = scored_attn_ref(q, k, v, [l], [c], 0.5, words=words, **kw)
    for i in range(c):
        path = [n for n in range(c) if int(words[0, i]) >> n & 1]
        rows = list(range(l)) + [l + n for n in path]
        oc, lc = scored_attn_ref(q[:, path], k[:, :, rows], v[:, :, rows], [l], [len(path)], 0.5, **kw)
        np.testing.assert_allclose(o[0, i], oc[0, -1], rtol=1e-12)
        np.testing.assert_allclose(lse[0, i], lc[0, -1], rtol=1e-12)


def test_a_row_without_keys():
    q, k, v, _, _ = rand_attn(6)
    o, l = scored_attn_ref(q, k, v, [3, 8], [4, 2], 0.5, starts=[3, 8], words=np.uint64([[0, 1, 3, 7], [1, 0, 0, 0]]))
    assert np.all(l[0, 0] == -np.inf) and np.all(o[0, 0] == 0) and np.all(l[1, 1] == -np.inf)
    assert np.all(np.isfinite(l[0, 1:4])) and np.all(np.isfinite(l[1, 0]))


def test_sampling_by_hand():
    x = np.log([0.1, 0.4, 0.1, 0.4])   # order: 1, 3, 0, 2
    draw = lambda u, **kw: sample_ref(x, u, **kw)[0]   # noqa: E731
    assert [draw(u) for u in (0.0, 0.39, 0.41, 0.79, 0.81, 0.89, 0.91, 0.999)] == [1, 1, 3, 3, 0, 0, 2, 2]
    assert [draw(0.999, top_k=k) for k in (1, 2, 3, 4, 0, -1, 9)] == [1, 3, 0, 2, 2, 2, 2]
    assert [draw(0.999, top_p=p) for p in (0.0, 0.3, 0.41, 0.79, 0.81, 0.95, 1.0, 2.0)] == [1, 1, 3, 3, 0, 2, 2, 2]
    assert [draw(0.999, min_p=p) for p in (0.0, 0.2, 0.26, 1.0, 3.0)] == [2, 2, 3, 3, 3]
    # top_p is a share of what top_k keeps
    assert draw(0.999, top_k=3, top_p=0.85) == 3 and draw(0.999, top_p=0.85) == 0
    # half the temperature squares the weights
    lp = [sample_ref(x, u, temperature=0.5)[1] for u in (0.0, 0.9999)]
    np.testing.assert_allclose(np.exp(lp), [16 / 34, 1 / 34], rtol=1e-12)
    assert sample_ref(x, 0.9, temperature=0.0) == (1, 0.0)


def test_sampling_shares():
    rng = np.random.default_rng(7)
    x = rng.standard_normal(50) * 2
    n = 200000
    u = (np.arange(n) + 0.5) / n
    got = np.bincount([sample_ref(x, v, temperature=0.7)[0] for v in u[::50]], minlength=50) / (n // 50)
    p = torch.softmax(torch.from_numpy(x) / 0.7, 0).numpy()
    assert np.abs(got - p).max() <= 2 / (n // 50)


def test_acceptance_at_temperature_zero_is_greedy():
    rng = np.random.default_rng(8)
    logits = rng.standard_normal((3, 4, 16)).astype(np.float32)
    tokens = rng.integers(0, 16, (3, 4))
    for b in range(3):
        for i in range(1, 1 + b):
            tokens[b, i] = logits[b, i - 1].argmax()
    cold = [dict(temperature=0.0)] * 3
    got = accept_sample_ref(logits, tokens, [5, 6, 7], [4, 3, 4], rng.random((3, 4)), cold)
    want = accept_greedy_ref(logits, tokens, [5, 6, 7], [4, 3, 4], "f32")
    for a, b in (("sampled", "argmax"), ("accepted",) * 2, ("next_token",) * 2, ("new_ctx_lens",) * 2):
        assert np.array_equal(got[a], want[b])
    words = np.uint64([[1, 3, 5, 9]] * 3)
    got = accept_sample_ref(logits, tokens, [5, 6, 7], [4, 3, 4], rng.random((3, 4)), cold, words)
    want = accept_tree_ref(logits, tokens, words, [5, 6, 7], [4, 3, 4], "f32")
    for a, b in (("sampled", "argmax"), ("accepted",) * 2, ("next_token",) * 2, ("path",) * 2):
        assert np.array_equal(got[a], np.asarray(want[b], np.int64))
