"""Performance cases of the operators around the verification attention: what puts
a chunk's queries, keys and values in place before it (``append_kv``), the
attention of models whose scores are capped, biased or windowed
(``verify_attn_scored``), and what draws tokens from the logits after it
(``sample``, and ``accept_sample`` / ``accept_sample_tree`` for whole chunks).

A case is one call with the inputs and the output buffers that a serving loop
keeps between steps.  Where ``own`` is false, ``run`` computes the plain form in
elementary torch operations; where it is true, it calls the package.  Lengths
belong to the case (drawn from its ``lens`` number), so that its work is fixed;
their order over the batch and all values come from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELT = {"f32": 4, "bf16": 2, "f16": 2}


def _append(name, B, Hq, Hkv, D, dtype, ctx_lo, ctx_hi, chunk_lo, chunk_hi, lens, page=0, tree=False, norm=False,
            rot=128, rope="halves"):
    case = dict(op="append", B=B, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, ctx_lo=ctx_lo, ctx_hi=ctx_hi, chunk_lo=chunk_lo,
                chunk_hi=chunk_hi, lens=lens, page=page, tree=tree, norm=norm, rot=rot, rope=rope)
    return dict(case, name=name) if name else case


def _scored(name, B, Hq, Hkv, D, dtype, ctx_lo, ctx_hi, chunk_lo, chunk_hi, lens, page=0, tree=False, cap=0.0,
            slopes=False, window=0, starts=False):
    case = dict(op="scored", B=B, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, ctx_lo=ctx_lo, ctx_hi=ctx_hi, chunk_lo=chunk_lo,
                chunk_hi=chunk_hi, lens=lens, page=page, tree=tree, cap=cap, slopes=slopes, window=window,
                starts=starts)
    return dict(case, name=name) if name else case


def _sample(name, op, B, C, V, dtype, chunk_lo, lens, params):
    case = dict(op=op, B=B, C=C, V=V, dtype=dtype, chunk_lo=chunk_lo, lens=lens, params=params)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one user's decoding step of a Mixtral-8x7B-shaped layer: all latency
        _append("append_b1", 1, 32, 8, 128, "bf16", 1000, 1000, 1, 1, 1),
        # the ordinary batch, drafts of 5, head norms, an FP16 cache in 16-token pages
        _append("append_paged_b64", 64, 32, 8, 128, "f16", 512, 2048, 5, 5, 2, page=16, norm=True),
        # prompts going into the cache, half of each head rotated in pairs
        _append("append_prefill_b8", 8, 32, 8, 128, "bf16", 0, 1024, 512, 2048, 3, rot=64, rope="pairs"),
        # a toy model or a unit test's call
        _scored("scored_tiny_f32", 2, 4, 1, 64, "f32", 128, 200, 4, 4, 4, cap=50.0),
        # capped scores over the ordinary batch
        _scored("scored_cap_b64", 64, 32, 8, 128, "bf16", 512, 2048, 5, 5, 5, cap=50.0),
        # 16-token tree drafts with a bias that grows with the distance
        _scored("scored_slopes_tree_b64", 64, 32, 8, 128, "bf16", 512, 2048, 16, 16, 6, tree=True, slopes=True),
        # a sliding window over ragged contexts and chunks in pages, seven query heads per KV head
        _scored("scored_window_paged_b128", 128, 28, 4, 128, "bf16", 256, 4096, 1, 16, 7, page=16, window=1024),
        # long documents: capped scores, and keys of an earlier document hidden
        _scored("scored_long_b32", 32, 32, 8, 128, "bf16", 16384, 32768, 4, 4, 8, cap=30.0, starts=True),
        # one user's next token, everything on
        _sample("sample_b1", "sample", 1, 1, 32000, "bf16", 1, 9, "all"),
        # a batch of requests of which each has its own settings, fp32 logits
        _sample("sample_b64_f32", "sample", 64, 1, 32000, "f32", 1, 10, "mix"),
        # the acceptance after tree and large-batch verifications
        _sample("accept_sample_tree_b64", "accept_tree", 64, 16, 32000, "bf16", 16, 11, "mix"),
        _sample("accept_sample_b256", "accept", 256, 8, 32000, "bf16", 8, 12, "mix"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


# (query heads, KV heads, head dim)
SHAPES = [(32, 8, 128), (32, 8, 128), (28, 4, 128), (32, 32, 128), (8, 1, 128), (4, 1, 64), (12, 4, 64), (16, 8, 64)]
KV_BYTES = 2.2e9       # valid K and V rows of one drawn call, at most (below the largest listed case)
CACHE_BYTES = 4e9      # K and V caches of one drawn state, at most
LOGIT_BYTES = 1.3e8    # logits of one drawn call, at most
KV_BYTES_F32 = 2.5e8   # fp32 caches are for small models
APPEND_BYTES = 1.5e8   # queries, keys and values that one drawn append brings, at most


def draw(rng):
    lens = rng.randrange(1000, 1 << 30)
    op = rng.choice(["append", "append", "scored", "scored", "scored", "sample", "accept", "accept_tree"])
    if op in ("sample", "accept", "accept_tree"):
        dtype = "bf16" if rng.random() < 0.7 else "f32"
        C = 1 if op == "sample" else _log_int(rng, 1 if op == "accept" else 2, 24)
        V = rng.choice([32000, 32000, 8 * _log_int(rng, 125, 19000)])
        B = min(_log_int(rng, 1, 256), max(1, int(LOGIT_BYTES / (C * V * ELT[dtype]))))
        return _sample("", op, B, C, V, dtype, rng.choice([C, C, max(1, C // 3)]), lens,
                       rng.choice(["mix", "mix", "all", "plain", "top_k", "top_p", "min_p"]))
    Hq, Hkv, D = rng.choice(SHAPES)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    page = rng.choice([0, 0, 16, 16, 64, 128])
    if op == "append":
        tree = rng.random() < 0.3
        chunk_hi = _log_int(rng, 1, 24) if tree or rng.random() < 0.5 else _log_int(rng, 1, 2048)
        ctx_hi = _log_int(rng, 1, 32768)
        row, fresh = 2 * Hkv * D * ELT[dtype], (Hq + 2 * Hkv) * D * ELT[dtype]
        most = max(1, min(int(CACHE_BYTES / 2 / (row * _round(ctx_hi + chunk_hi, 256))),
                          int(APPEND_BYTES / (fresh * chunk_hi))))
        return _append("", min(_log_int(rng, 1, 256), most), Hq, Hkv, D, dtype, rng.choice([0, ctx_hi // 4, ctx_hi]),
                       ctx_hi, rng.choice([chunk_hi, max(1, chunk_hi // 4)]), chunk_hi, lens, page=page, tree=tree,
                       norm=rng.random() < 0.4, rot=rng.choice([D, D, D // 2, D // 4]),
                       rope=rng.choice(["halves", "halves", "pairs"]))
    tree = rng.random() < 0.3
    chunk_hi = min(_log_int(rng, 1, 32 if tree else 16), 128 // (Hq // Hkv))
    ctx_hi = _log_int(rng, 64, 32768)
    ctx_lo = max(1, int(ctx_hi * rng.uniform(0.1, 1.0)))
    row = 2 * Hkv * D * ELT[dtype]   # K and V bytes of one token
    cap_bytes = KV_BYTES_F32 if dtype == "f32" else KV_BYTES
    S = _round(ctx_hi + chunk_hi, 256)
    most = max(1, min(int(cap_bytes / (row * (ctx_hi + chunk_hi))), int(CACHE_BYTES / (row * S))))
    cap = rng.choice([0.0, 30.0, 50.0])
    slopes, window = rng.random() < 0.3, _log_int(rng, 16, 8192) if rng.random() < 0.5 else 0
    return _scored("", min(_log_int(rng, 1, 256), most), Hq, Hkv, D, dtype, ctx_lo, ctx_hi,
                   rng.choice([chunk_hi, chunk_hi, max(1, chunk_hi // 4)]), chunk_hi, lens, page=page, tree=tree,
                   cap=cap, slopes=slopes, window=window,
                   starts=rng.random() < 0.3 or not (cap or slopes or window))


def _round(x, m):
    return (x + m - 1) // m * m


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """Context and chunk lengths and first visible keys of the case, before the
    seed orders them."""
    rng = np.random.default_rng([case["lens"], 1])
    B = case["B"]
    ctx = rng.integers(case.get("ctx_lo", 512), case.get("ctx_hi", 2048) + 1, size=B)
    hi = case["chunk_hi"] if "chunk_hi" in case else case["C"]
    chunk = rng.integers(case["chunk_lo"], hi + 1, size=B)
    start = (ctx * rng.uniform(0.0, 0.5, size=B)).astype(np.int64) if case.get("starts") else np.zeros(B, np.int64)
    return ctx, chunk, start


def _ordered(case, seed):
    order = np.random.default_rng([seed, 2]).permutation(case["B"])
    return [x[order].astype(np.int32) for x in _lengths(case)]


def _tree_words(seed, chunk, C):
    """Root-path words of random recursive trees (bit k of word i: token k is i
    or an ancestor of i)."""
    words = np.zeros((len(chunk), C), np.uint64)
    for b, c in enumerate(chunk):
        parent = np.random.default_rng([seed, 3, b]).integers(0, np.maximum(np.arange(c), 1))
        for i in range(c):
            words[b, i] = (words[b, parent[i]] if i else np.uint64(0)) | np.uint64(1 << i)
    return words


def _cache(case, seed, gen, dev, st):
    """K and V caches, a slab per sequence or a shuffled pool of pages."""
    B, Hkv, D, S = case["B"], case["Hkv"], case["D"], _round(case["ctx_hi"] + case["chunk_hi"], 256)
    st["table"] = None
    shape = (B, Hkv, S, D)
    if case["page"]:
        n = B * (S // case["page"])
        shape = (n + 8, Hkv, case["page"], D)   # a pool with a few pages free
        table = np.random.default_rng([seed, 5]).permutation(n + 8)[:n].astype(np.int32)
        st["table"] = torch.from_numpy(table.reshape(B, -1)).to(dev)
    for n in ("k", "v"):
        st[n] = torch.randn(shape, generator=gen, device=dev, dtype=DTYPES[case["dtype"]])


def _append_state(case, seed, dev, gen, st):
    B, Hq, Hkv, D, C, dt = case["B"], case["Hq"], case["Hkv"], case["D"], case["chunk_hi"], DTYPES[case["dtype"]]
    _cache(case, seed, gen, dev, st)
    # the output of one projection to queries, keys and values
    qkv = torch.randn((B, C, Hq + 2 * Hkv, D), generator=gen, device=dev, dtype=dt)
    st["new"] = [qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]]
    rot = case["rot"]
    st["inv_freq"] = 1.0 / 10000.0 ** (torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
    st["rope"] = case["rope"]
    st["weights"] = [None, None]
    if case["norm"]:
        st["weights"] = [(1 + 0.1 * torch.randn((D,), generator=gen, device=dev)).to(dt) for _ in range(2)]
    st["q_out"] = torch.zeros((B, C, Hq, D), device=dev, dtype=dt)


def _scored_state(case, seed, dev, gen, st):
    B, Hq, D, C, dt = case["B"], case["Hq"], case["D"], case["chunk_hi"], DTYPES[case["dtype"]]
    _cache(case, seed, gen, dev, st)
    st["q"] = torch.randn((B, C, Hq, D), generator=gen, device=dev, dtype=dt)
    st["scale"], st["cap"], st["window"] = 1.0 / math.sqrt(D), case["cap"], case["window"]
    st["slopes"] = None
    if case["slopes"]:
        st["slopes"] = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=dev, dtype=torch.float32) / Hq)
    st["out"] = torch.empty((B, C, Hq, D), device=dev, dtype=dt)
    st["lse"] = torch.empty((B, C, Hq), device=dev, dtype=torch.float32)


def _sample_state(case, seed, dev, gen, st):
    """Logits with one likely winner per row; drafts that match it with
    probability 0.7 (a tree's: their parent's winner); each sequence's own
    sampling settings."""
    B, C, V = case["B"], case["C"], case["V"]
    rng = np.random.default_rng([seed, 4])
    won = rng.integers(0, V, size=(B, C))
    logits = torch.randn((B, C, V), generator=gen, device=dev, dtype=torch.float32) * 2
    logits.scatter_(2, torch.from_numpy(won).to(dev).unsqueeze(2), 12.0)
    st["logits"] = logits.to(DTYPES[case["dtype"]])
    st["u"] = torch.rand((B, C), generator=gen, device=dev, dtype=torch.float32)
    params = case["params"]
    on = lambda n: params in (n, "all", "mix")   # noqa: E731
    some = lambda x, off: np.where(rng.random(B) < 0.5, x, off) if params == "mix" else x   # noqa: E731
    put = lambda x, dt: torch.from_numpy(np.asarray(x).astype(dt)).to(dev)   # noqa: E731
    st["temperature"] = put(some(rng.uniform(0.6, 1.2, size=B), 1.0), np.float32)
    st["top_k"] = put(some(rng.choice([1, 20, 50, 200], size=B), 0), np.int32) if on("top_k") else None
    st["top_p"] = put(some(rng.uniform(0.5, 0.98, size=B), 1.0), np.float32) if on("top_p") else None
    st["min_p"] = put(some(rng.uniform(0.01, 0.2, size=B), 0.0), np.float32) if on("min_p") else None
    if case["op"] == "sample":
        st["logits"], st["u"] = st["logits"][:, 0], st["u"][:, 0]
        st["out"] = [torch.empty((B,), device=dev, dtype=torch.int32), torch.empty((B,), device=dev)]
        return
    chunk = st["chunk_host"]
    parent = np.broadcast_to(np.maximum(np.arange(C) - 1, 0), (B, C))
    if case["op"] == "accept_tree":
        words = _tree_words(seed, chunk, C)
        above = words & ~(np.uint64(1) << np.arange(C, dtype=np.uint64))[None, :]
        parent = np.array([[int(w).bit_length() - 1 if w else 0 for w in row] for row in above])
        st["mask"] = torch.from_numpy(words.view(np.int64)).to(dev)
    tokens = np.where(rng.random((B, C)) < 0.7, np.take_along_axis(won, parent, 1), rng.integers(0, V, size=(B, C)))
    st["tokens"] = torch.from_numpy(tokens.astype(np.int32)).to(dev)
    new = lambda shape, dt: torch.empty(shape, dtype=dt, device=dev)   # noqa: E731
    st["out"] = dict(sampled=new((B, C), torch.int32), logprobs=new((B, C), torch.float32),
                     **{n: new((B,), torch.int32) for n in ("accepted", "next_token", "new_ctx_lens")})
    if case["op"] == "accept_tree":
        st["out"]["path"] = new((B,), torch.int64)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    st = dict(op=case["op"], mask=None, chunk_host=None)
    ctx, chunk, start = _ordered(case, seed)
    st["chunk_host"] = chunk
    st["ctx"], st["chunk"] = torch.from_numpy(ctx).to(dev), torch.from_numpy(chunk).to(dev)
    st["starts"] = torch.from_numpy(start).to(dev) if case.get("starts") else None
    if case.get("tree"):
        st["mask"] = torch.from_numpy(_tree_words(seed, chunk, case["chunk_hi"]).view(np.int64)).to(dev)
    {"append": _append_state, "scored": _scored_state}.get(case["op"], _sample_state)(case, seed, dev, gen, st)
    return st


# ------------------------------------------------------------- plain forms

def _bits(words, C):
    """[B, C, C] truth values: token i sees draft token k."""
    return (words.unsqueeze(2) >> torch.arange(C, device=words.device)) & 1 > 0


def _plain_append(st):
    q, k, v = st["new"]
    B, C = q.shape[:2]
    dev = q.device
    i = torch.arange(C, device=dev)
    valid = i < st["chunk"][:, None]
    row = st["ctx"][:, None].long() + i
    pos = row
    if st["mask"] is not None:
        seen = _bits(st["mask"], C) & (i < st["chunk"][:, None])[:, None, :]
        pos = st["ctx"][:, None].long() + seen.sum(2) - 1
    angle = pos[:, :, None, None].double() * st["inv_freq"]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    half = st["inv_freq"].numel()
    rotated = []
    for x, w in zip((q, k), st["weights"]):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        if st["rope"] == "halves":
            a, b = x[..., :half], x[..., half:2 * half]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        rotated.append(torch.cat([turned, x[..., 2 * half:]], -1).to(q.dtype))
    st["q_out"].copy_(torch.where(valid[:, :, None, None], rotated[0], st["q_out"]))
    at = torch.arange(B, device=dev)[:, None]
    if st["table"] is not None:
        page = st["k"].shape[2]
        at, row = st["table"][at, row // page].long(), row % page
    for cache, new in ((st["k"], rotated[1]), (st["v"], v)):
        cache[at, :, row] = torch.where(valid[:, :, None, None], new, cache[at, :, row])
    return st["q_out"], st["k"], st["v"]


def _slab(cache, table):
    """The cache as [B, Hkv, S, D] in 32 bits."""
    if table is None:
        return cache.float()
    B, Hkv, D = table.shape[0], cache.shape[1], cache.shape[3]
    return cache[table.long()].transpose(1, 2).reshape(B, Hkv, -1, D).float()


def _plain_scored(st):
    q, k, v = st["q"].float(), _slab(st["k"], st["table"]), _slab(st["v"], st["table"])
    B, C, Hq, D = q.shape
    Hkv, S = k.shape[1:3]
    g, dev = Hq // Hkv, q.device
    i, j = torch.arange(C, device=dev), torch.arange(S, device=dev)
    ctx, chunk = st["ctx"][:, None, None].long(), st["chunk"][:, None].long()
    draft = j - ctx                     # [B, 1, S] draft token of a key, negative in the context
    if st["mask"] is None:
        dist = i[:, None] - draft       # [B, C, S] keys after j that token i sees
        seen = dist >= 0
    else:
        bits = (_bits(st["mask"], C) & (i < chunk)[:, None, :]).long()
        after = bits.flip(2).cumsum(2).flip(2) - bits      # draft tokens after k that i sees
        at = draft.clamp(0, C - 1).expand(B, C, S)
        inside = (draft >= 0) & (draft < C)
        dist = torch.where(inside, after.gather(2, at), bits.sum(2, keepdim=True) - 1 - draft)
        seen = torch.where(inside, bits.gather(2, at) > 0, draft < 0)
    seen = seen & (draft < chunk[:, None])
    if st["window"]:
        seen = seen & (dist < st["window"])
    if st["starts"] is not None:
        seen = seen & (j >= st["starts"][:, None, None])
    q = q.reshape(B, C, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, C * g, D)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * st["scale"]
    if st["cap"]:
        s = st["cap"] * torch.tanh(s / st["cap"])
    s = s.view(B, Hkv, C, g, S)
    if st["slopes"] is not None:
        s = s - st["slopes"].view(Hkv, 1, g, 1) * dist[:, None, :, None, :].float()
    s = s.masked_fill(~seen[:, None, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m.clamp(min=-3e38))
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, C * g, S), v).view(B, Hkv, C, g, D) / z.clamp(min=1e-37)
    valid = (i < chunk)[:, None, :, None]
    lse = (m + torch.log(z)).squeeze(-1).masked_fill(~valid, -math.inf)
    o = o.masked_fill(~valid[..., None], 0.0)
    out = o.permute(0, 2, 1, 3, 4).reshape(B, C, Hq, D).to(st["q"].dtype)
    return out, lse.permute(0, 2, 1, 3).reshape(B, C, Hq)


def _plain_draw(logits, u, temperature, top_k, top_p, min_p):
    """Tokens of rows of logits (the first in order of falling probability whose
    cumulative share passes u), and the logarithms of their probabilities.  In 64
    bits: a token is a comparison of sums over the whole vocabulary."""
    x = logits.double() + 0.0
    V = x.shape[1]
    d = (x.amax(1, keepdim=True) - x) / temperature[:, None].double()
    order = torch.sort(d, dim=1, stable=True)
    w = torch.exp(-order.values)
    if top_k is not None:
        k = torch.where(top_k > 0, top_k, V)[:, None]
        w = torch.where(torch.arange(V, device=x.device) < k, w, 0.0)
    if top_p is not None:
        before = w.cumsum(1) - w
        keep = (before < top_p[:, None].double() * w.sum(1, keepdim=True)) | (top_p[:, None] >= 1)
        w = torch.where(keep, w, 0.0)
    if min_p is not None:
        w = torch.where(w >= min_p[:, None].double(), w, 0.0)
    z = w.cumsum(1)
    at = (z <= u[:, None].double() * z[:, -1:]).sum(1, keepdim=True)
    p = w.gather(1, at) / z[:, -1:]
    return order.indices.gather(1, at).squeeze(1).int(), torch.log(p).squeeze(1).float()


def _plain_sample(st):
    if st["op"] == "sample":
        return _plain_draw(st["logits"], st["u"], st["temperature"], st["top_k"], st["top_p"], st["min_p"])
    B, C, V = st["logits"].shape
    rows = [None if st[n] is None else st[n].repeat_interleave(C) for n in ("temperature", "top_k", "top_p", "min_p")]
    token, logp = _plain_draw(st["logits"].view(B * C, V), st["u"].view(-1), *rows)
    i = torch.arange(C, device=token.device)
    chunk = st["chunk"][:, None]
    token = torch.where(i < chunk, token.view(B, C), -1)
    logp = torch.where(i < chunk, logp.view(B, C), 0.0)
    res = dict(sampled=token, logprobs=logp)
    if st["op"] == "accept":
        match = (st["tokens"][:, 1:] == token[:, :-1]) & (i[1:] < chunk)
        last = a = match.int().cumprod(1).sum(1)
    else:
        word = st["mask"]
        bits = _bits(word, C)
        parent = (bits & (i < i[:, None])).long().mul(i).amax(2)
        edge = st["tokens"] != token.gather(1, parent)
        wrong = edge & (i > 0) & (i < chunk)
        depth = bits.sum(2) - 1
        ok = ~(bits & wrong[:, None, :]).any(2) & (i < chunk)
        last = torch.where(ok, depth * C + (C - 1 - i), -1).argmax(1)
        a = depth.gather(1, last[:, None]).squeeze(1)
        res["path"] = word.gather(1, last[:, None]).squeeze(1)
    res["accepted"] = a.int()
    res["next_token"] = token.gather(1, last[:, None].long()).squeeze(1)
    res["new_ctx_lens"] = (st["ctx"] + a + 1).int()
    return res


# --------------------------------------------------------------- own calls

def _own_run(st):
    import paper_2508_21706_amd as sm

    op = st["op"]
    if op == "append":
        q, k, v = st["new"]
        sm.append_kv(q, k, v, st["k"], st["v"], st["ctx"], st["chunk"], inv_freq=st["inv_freq"], rope=st["rope"],
                     q_weight=st["weights"][0], k_weight=st["weights"][1], eps=1e-6, draft_mask=st["mask"],
                     block_table=st["table"], q_out=st["q_out"])
        return st["q_out"], st["k"], st["v"]
    if op == "scored":
        if "ws" not in st:   # a serving loop's, kept between its steps
            st["ws"] = sm.alloc_scored_workspace(st["q"], st["k"], block_table=st["table"])
        return sm.verify_attn_scored(st["q"], st["k"], st["v"], st["ctx"], st["chunk"], st["scale"],
                                     softcap=st["cap"], slopes=st["slopes"], window=st["window"],
                                     starts=st["starts"], draft_mask=st["mask"], block_table=st["table"],
                                     out=st["out"], lse=st["lse"], workspace=st["ws"])
    params = {n: st[n] for n in ("temperature", "top_k", "top_p", "min_p", "out")}
    if op == "sample":
        return sm.sample(st["logits"], st["u"], **params)
    if "ws" not in st:
        code = {torch.float32: sm.binding.SPECMOE_F32, torch.bfloat16: sm.binding.SPECMOE_BF16}[st["logits"].dtype]
        st["ws"] = sm.alloc_accept_workspace(sm.accept_desc(*st["logits"].shape, code), st["logits"].device)
    params["workspace"] = st["ws"]
    if op == "accept":
        return sm.accept_sample(st["logits"], st["tokens"], st["ctx"], st["chunk"], st["u"], **params)
    return sm.accept_sample_tree(st["logits"], st["tokens"], st["mask"], st["ctx"], st["chunk"], st["u"], **params)


def run(st):
    if own:
        return _own_run(st)
    return {"append": _plain_append, "scored": _plain_scored}.get(st["op"], _plain_sample)(st)


def work(case):
    ctx, chunk, start = _lengths(case)
    elt, B, tokens = ELT[case["dtype"]], case["B"], int(chunk.sum())
    if case["op"] == "append":
        # the chunk's queries, keys and values, read and written
        return {"bytes": 2 * tokens * (case["Hq"] + 2 * case["Hkv"]) * case["D"] * elt + 8 * B, "flops": 0}
    if case["op"] == "scored":
        Hq, Hkv, D, C = case["Hq"], case["Hkv"], case["D"], case["chunk_hi"]
        first = np.maximum(start, ctx - case["window"] + 1) if case["window"] else start
        T = ctx + chunk - np.maximum(first, 0)
        kv = 2 * int(T.sum()) * Hkv * D * elt
        # (the padding rows are written too)
        return {"bytes": kv + tokens * Hq * D * elt + B * C * Hq * (D * elt + 4),
                "flops": 4 * Hq * D * int((chunk * T).sum())}
    return {"bytes": tokens * case["V"] * elt + 20 * tokens + 32 * B, "flops": 0}


# ---------------------------------------------- the definitions in 64 bits

def _exact_append(st):
    q, k, v = st["new"]
    half = st["inv_freq"].numel()
    res = [st["q_out"].double(), st["k"].double(), st["v"].double()]
    ctx, chunk = st["ctx"].tolist(), st["chunk"].tolist()
    for b, (l, c) in enumerate(zip(ctx, chunk)):
        pos = torch.arange(l, l + c, device=q.device).double()
        if st["mask"] is not None:
            words = [int(w) & ((1 << c) - 1) for w in st["mask"][b, :c].tolist()]
            pos = torch.tensor([l + bin(w).count("1") - 1 for w in words], device=q.device).double()
        turn = torch.polar(torch.ones((), device=q.device).double(), pos[:, None] * st["inv_freq"])[:, None]
        new = []
        for x, w in ((q, st["weights"][0]), (k, st["weights"][1])):
            x = x[b, :c].double()
            if w is not None:
                x = w.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + 1e-6)
            x = x.clone()
            at = (slice(0, half), slice(half, 2 * half)) if st["rope"] == "halves" else (slice(0, 2 * half, 2),
                                                                                       slice(1, 2 * half, 2))
            z = torch.complex(x[..., at[0]].contiguous(), x[..., at[1]].contiguous()) * turn
            x[..., at[0]], x[..., at[1]] = z.real, z.imag
            new.append(x)
        res[0][b, :c] = new[0]
        for cache, x in ((res[1], new[1]), (res[2], v[b, :c].double())):
            if st["table"] is None:
                cache[b, :, l:l + c] = x.transpose(0, 1)
            else:
                rows = torch.arange(l, l + c, device=q.device)
                page = cache.shape[2]
                cache[st["table"][b].long()[rows // page], :, rows % page] = x
    return tuple(res)


def _exact_scored(st):
    B, C, Hq, D = st["q"].shape
    Hkv, dev = st["k"].shape[1], st["q"].device
    g = Hq // Hkv
    out = torch.zeros((B, C, Hq, D), dtype=torch.float64, device=dev)
    lse = torch.full((B, C, Hq), -math.inf, dtype=torch.float64, device=dev)
    ctx, chunk = st["ctx"].tolist(), st["chunk"].tolist()
    for b, (l, c) in enumerate(zip(ctx, chunk)):
        T = l + c
        if st["table"] is not None:
            pages = st["table"][b].long()[: -(-T // st["k"].shape[2])]
            k, v = (st[n][pages].transpose(0, 1).reshape(Hkv, -1, D)[:, :T].double() for n in ("k", "v"))
        else:
            k, v = (st[n][b, :, :T].double() for n in ("k", "v"))
        sees = torch.ones((c, T), dtype=torch.bool, device=dev).tril(l)
        if st["mask"] is not None:
            words = st["mask"][b, :c].tolist()
            sees[:, l:] = torch.tensor([[w >> n & 1 for n in range(c)] for w in words], device=dev) > 0
        dist = sees.long().flip(1).cumsum(1).flip(1) - sees.long()   # keys after each that the token sees
        if st["window"]:
            sees &= dist < st["window"]
        if st["starts"] is not None:
            sees[:, : int(st["starts"][b])] = False
        q = st["q"][b, :c].double().reshape(c, Hkv, g, D).permute(1, 2, 0, 3).reshape(Hkv, g * c, D)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()).view(Hkv, g, c, T) * st["scale"]
        if st["cap"]:
            s = st["cap"] * torch.tanh(s / st["cap"])
        if st["slopes"] is not None:
            s = s - st["slopes"].double().view(Hkv, g, 1, 1) * dist
        s = torch.where(sees, s, -math.inf)
        z = torch.logsumexp(s, -1)
        o = torch.matmul(torch.exp(s - z[..., None]).view(Hkv, g * c, T), v.contiguous()).view(Hkv, g, c, D)
        out[b, :c] = o.permute(2, 0, 1, 3).reshape(c, Hq, D)
        lse[b, :c] = z.permute(2, 0, 1).reshape(c, Hq)
    return out, lse


def _exact_draw(x, u, temperature, k, p, min_p):
    """One row, on the host: the most probable tokens first, cut down by each
    setting in turn."""
    order = np.lexsort((np.arange(x.size), -x))
    w = np.exp((x - x[order[0]]) / temperature)[order]
    n = k if k and k > 0 else x.size
    w, order = w[:n], order[:n]
    if p is not None and p < 1:
        n = 1 + int(np.searchsorted(np.cumsum(w)[:-1], p * w.sum(), side="left"))
        w, order = w[:n], order[:n]
    if min_p is not None:
        n = int((w >= min_p).sum())
        w, order = w[:n], order[:n]
    cum = np.cumsum(w)
    n = int(np.searchsorted(cum, u * cum[-1], side="right"))
    return int(order[n]), math.log(w[n] / cum[-1])


def _exact_sample(st):
    logits = st["logits"].double().cpu().numpy()
    chain = st["op"] != "sample"
    logits = logits if chain else logits[:, None]
    B, C, _ = logits.shape
    u = st["u"].double().cpu().numpy().reshape(B, C)
    settings = [[None] * B if st[n] is None else st[n].double().tolist()
                for n in ("temperature", "top_k", "top_p", "min_p")]
    token, logp = np.full((B, C), -1, np.int32), np.zeros((B, C))
    for b in range(B):
        for i in range(int(st["chunk_host"][b]) if chain else 1):
            t, k, p, m = (x[b] for x in settings)
            token[b, i], logp[b, i] = _exact_draw(logits[b, i], u[b, i], t, int(k) if k else 0, p, m)
    if not chain:
        return token[:, 0], logp[:, 0]
    res = dict(sampled=token, logprobs=logp, accepted=None, next_token=None, new_ctx_lens=None)
    return dict(res, path=None) if st["op"] == "accept_tree" else res


def exact(case, seed):
    if case["op"] not in ("append", "scored") and case["B"] * case["C"] * case["V"] > 80e6:
        return None   # sorted on the host: more than 20 seconds
    st = prepare(case, seed)
    return {"append": _exact_append, "scored": _exact_scored}.get(case["op"], _exact_sample)(st)
