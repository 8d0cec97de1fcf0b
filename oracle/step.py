"""Plain CPU oracle of the operators around the verification attention.

TEST INFRASTRUCTURE, NOT PART OF THE PRODUCT.  It shares no code with the HIP
path and imports nothing from it.  Everything is float64, one row at a time:

  * ``append_ref``: head norms, the rotation by a token's position, and the
    append of a chunk's keys and values;
  * ``scored_attn_ref``: verification attention whose scores are capped by a
    tanh, lowered with the distance, and hidden by a window and a first key;
  * ``sample_ref``, ``accept_sample_ref``: tokens from given random numbers,
    and the acceptance of drafts that equal them.
"""
from __future__ import annotations

import math

import numpy as np

from .acceptance import tree_parent


def positions_ref(l: int, c: int, words=None):
    """Position of each of a chunk's tokens: chains count on from the context,
    a tree's token stands after the context and its ancestors."""
    if words is None:
        return [l + i for i in range(c)]
    return [l + max(bin(int(w) & ((1 << c) - 1)).count("1"), 1) - 1 for w in words[:c]]


def head_ref(x, pos: int, inv_freq=None, rope="halves", weight=None, eps=1e-6):
    """One head row: norm, then rotation."""
    x = np.array(x, np.float64)
    if weight is not None:
        x = x / math.sqrt(np.mean(x * x) + eps) * np.asarray(weight, np.float64)
    if inv_freq is not None:
        half = len(inv_freq)
        for j, f in enumerate(np.asarray(inv_freq, np.float64)):
            a, b = (j, j + half) if rope == "halves" else (2 * j, 2 * j + 1)
            angle = np.longdouble(pos) * np.longdouble(f)
            cos, sin = float(np.cos(angle)), float(np.sin(angle))
            x[a], x[b] = x[a] * cos - x[b] * sin, x[b] * cos + x[a] * sin
    return x


def append_ref(q, k, v, k_cache, v_cache, q_out, ctx_lens, chunk_lens, inv_freq=None, rope="halves", q_weight=None,
               k_weight=None, eps=1e-6, words=None, table=None):
    """(q_out, k_cache, v_cache) after the append, as float64 copies."""
    q_out, k_cache, v_cache = (np.array(x, np.float64) for x in (q_out, k_cache, v_cache))
    for b, (l, c) in enumerate(zip(ctx_lens, chunk_lens)):
        l, c = int(l), int(c)
        for i, pos in enumerate(positions_ref(l, c, None if words is None else words[b])):
            for h in range(q.shape[2]):
                q_out[b, i, h] = head_ref(q[b, i, h], pos, inv_freq, rope, q_weight, eps)
            row = l + i
            if table is None:
                where = (b, slice(None), row)
            else:
                page = k_cache.shape[2]
                where = (int(table[b, row // page]), slice(None), row % page)
            k_cache[where] = [head_ref(x, pos, inv_freq, rope, k_weight, eps) for x in k[b, i]]
            v_cache[where] = v[b, i]
    return q_out, k_cache, v_cache


def scored_row_ref(q, k, v, scale, sees, softcap=0.0, slope=0.0, window=0, start=0, l=None):
    """Output and log-sum-exp of one query over T keys; ``sees`` the keys that
    the mask shows it, the first ``l`` of them cached (None: all but one)."""
    T = k.shape[0]
    dist = sees.sum() - np.cumsum(sees)   # the keys after each that it sees (for a key it does not see: unused)
    if l is not None and not sees[l:].any():
        dist = dist + 1                   # a token that sees no draft token stands like a root
    s = (k @ q) * scale
    if softcap:
        s = softcap * np.tanh(s / softcap)
    s = s - slope * dist
    keep = sees & (np.arange(T) >= start)
    if window:
        keep &= dist < window
    if not keep.any():
        return np.zeros(v.shape[1]), -np.inf
    s, v = s[keep], v[keep]
    m = s.max()
    p = np.exp(s - m)
    return p @ v / p.sum(), m + math.log(p.sum())


def scored_attn_ref(q, k_cache, v_cache, ctx_lens, chunk_lens, scale, softcap=0.0, slopes=None, window=0, starts=None,
                    words=None):
    """q [B, C, Hq, D], caches [B, Hkv, S, D] (float64); returns out and lse."""
    B, C, Hq, D = q.shape
    g = Hq // k_cache.shape[1]
    out, lse = np.zeros((B, C, Hq, D)), np.full((B, C, Hq), -np.inf)
    for b in range(B):
        l, c = int(ctx_lens[b]), int(chunk_lens[b])
        T = l + c
        for i in range(c):
            sees = np.arange(T) <= l + i
            if words is not None:
                sees[l:] = [(int(words[b, i]) >> n) & 1 for n in range(c)]
            for h in range(Hq):
                out[b, i, h], lse[b, i, h] = scored_row_ref(
                    q[b, i, h], k_cache[b, h // g, :T], v_cache[b, h // g, :T], scale, sees, softcap,
                    0.0 if slopes is None else float(slopes[h]), window, 0 if starts is None else int(starts[b]), l)
    return out, lse


def sample_ref(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row of logits (float64): (token, log-probability)."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64)) + 0.0
    top = x.max()
    if not temperature > 0:
        return (int(np.argmax(x)) if not np.all(np.isnan(x)) else -1), 0.0
    if top == -np.inf:
        return -1, -np.inf
    with np.errstate(invalid="ignore"):
        # (an infinite logit leaves nothing to finite ones, at any temperature)
        w = np.where(x == top, 1.0, np.where(np.isinf(x) | np.isinf(top), 0.0, np.exp((x - top) / float(temperature))))
    order = np.lexsort((np.arange(x.size), -x))
    w = w[order]
    n = x.size
    if 0 < top_k < n:
        n = int(top_k)
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[:n])[:-1]])
        n = max(1, int((before < max(float(top_p), 0.0) * w[:n].sum()).sum()))
    if min_p > 0:
        n = min(n, max(1, int((w >= min(float(min_p), 1.0)).sum())))
    cum = np.cumsum(w[:n])
    u = float(u) if u > 0 else 0.0
    at = min(int(np.searchsorted(cum, u * cum[-1], side="right")), int((w[:n] > 0).sum()) - 1)
    return int(order[at]), float((x[order[at]] - top) / temperature if x[order[at]] < top else 0.0) - math.log(cum[-1])


def accept_sample_ref(logits, tokens, ctx_lens, chunk_lens, uniforms, settings, words=None):
    """The acceptance rule with sampled tokens; ``settings``: per sequence a
    dict of sample_ref's keywords.  Returns a dict of arrays."""
    B, C, _ = logits.shape
    res = dict(sampled=np.full((B, C), -1, np.int64), logprobs=np.zeros((B, C)), accepted=np.zeros(B, np.int64),
               next_token=np.full(B, -1, np.int64), new_ctx_lens=np.array(ctx_lens, np.int64),
               path=np.zeros(B, np.int64))
    for b in range(B):
        c = int(chunk_lens[b])
        if c == 0:
            continue
        for i in range(c):
            res["sampled"][b, i], res["logprobs"][b, i] = sample_ref(logits[b, i], uniforms[b, i], **settings[b])
        s = res["sampled"][b]
        if words is None:
            a = 0
            while a < c - 1 and s[a] == tokens[b, a + 1]:
                a += 1
            best = a
        else:
            ok = [True] + [False] * (c - 1)
            for i in range(1, c):
                parent = tree_parent(words[b], i)
                ok[i] = ok[parent] and s[parent] == tokens[b, i]
            depth = [bin(int(w) & ((1 << c) - 1)).count("1") - 1 for w in words[b, :c]]
            best = max((i for i in range(c) if ok[i]), key=lambda i: (depth[i], -i))
            a = depth[best]
            res["path"][b] = np.uint64(int(words[b, best]) & ((1 << c) - 1)).astype(np.int64)
        res["accepted"][b], res["next_token"][b], res["new_ctx_lens"][b] = a, s[best], int(ctx_lens[b]) + a + 1
    return res
