"""Performance cases of the KV cache held in 4 bits and of the pages it lives in:
what appends to it (``append_kv4``), the verification and decode attention over it
(``verify_attn_kv4``), what hands rows back in 16 or 32 bits (``read_kv4``), what
moves an accepted tree path's rows (``compact_accepted_kv4``), and block tables and
slot maps made on the GPU from the requests' lengths (``assign_pages``).

A cached head row is D / 32 blocks of 32 entries: a scale 2^(e - 127), e the byte
kept, and 32 codes of 4 bits with the values 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign
bit.  The scale is the smallest power of two at which the block's largest entry lies
below 7, so that it rounds to 6 at most; codes are rounded to nearest, ties to even.

A case is one call (or the two that belong together) with the inputs and the output
buffers that a serving loop keeps between steps.  Where ``own`` is false, ``run``
computes the plain form in elementary torch operations; where it is true, it calls
the package.  Lengths belong to the case (drawn from its ``lens`` number), so that
its work is fixed; their order over the batch and all values come from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELT = {"f32": 4, "bf16": 2, "f16": 2}


def _case(name, op, B, Hq, Hkv, D, dtype, ctx_lo, ctx_hi, chunk_lo, chunk_hi, lens, page=0, tree=False, norm=False,
          rot=0, rope="halves"):
    case = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, ctx_lo=ctx_lo, ctx_hi=ctx_hi, chunk_lo=chunk_lo,
                chunk_hi=chunk_hi, lens=lens, page=page, tree=tree, norm=norm, rot=rot, rope=rope)
    return dict(case, name=name) if name else case


def _pages(name, B, page, ctx_lo, ctx_hi, chunk_lo, chunk_hi, lens, turnover):
    case = dict(op="pages", B=B, page=page, ctx_lo=ctx_lo, ctx_hi=ctx_hi, chunk_lo=chunk_lo, chunk_hi=chunk_hi,
                lens=lens, turnover=turnover)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one user's next token (a Mixtral-8x7B-shaped layer): all latency
        _case("append_b1", "append", 1, 32, 8, 128, "bf16", 1000, 1000, 1, 1, 1, rot=128),
        # prompts going into an FP16 model's paged cache, with head norms
        _case("append_prefill_b8", "append", 8, 32, 8, 128, "f16", 0, 768, 512, 2048, 2, page=16, norm=True, rot=128),
        # a small fp32 model's single tokens
        _case("attn_decode_f32_b4", "attn", 4, 8, 4, 64, "f32", 100, 400, 1, 1, 3),
        # the ordinary batch: drafts of 5 over contexts of 512 to 2048 in 16-token pages
        _case("attn_paged_b64", "attn", 64, 32, 8, 128, "bf16", 512, 2048, 5, 5, 4, page=16),
        # 16-token tree drafts
        _case("attn_tree_f16_b64", "attn", 64, 32, 8, 128, "f16", 512, 2048, 16, 16, 5, tree=True),
        # long documents
        _case("attn_long_b32", "attn", 32, 32, 8, 128, "bf16", 16384, 32768, 4, 4, 6),
        # a request's prompt handed from the 4-bit cache to a 16-bit one
        _case("read_b1", "read", 1, 32, 8, 128, "bf16", 0, 0, 1000, 1000, 7, page=16),
        # the same for ragged prompts of a batch
        _case("read_b16", "read", 16, 32, 8, 128, "bf16", 0, 500, 300, 4096, 8),
        # the accepted paths of 16-token trees put in place
        _case("compact_b64", "compact", 64, 32, 8, 128, "bf16", 512, 2048, 16, 16, 9, tree=True),
        # the same for large ragged trees of a large batch, in pages
        _case("compact_paged_b256", "compact", 256, 28, 4, 128, "bf16", 256, 4096, 8, 64, 10, page=16, tree=True),
        # two steps of a serving loop: most requests grow by some draft tokens, some end and some begin
        _pages("pages_b64", 64, 16, 512, 2048, 1, 5, 11, 0.1),
        # the same with prompts admitted and a large batch
        _pages("pages_prompts_b512", 512, 16, 0, 1024, 1, 2048, 12, 0.5),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


# (query heads, KV heads, head dim)
SHAPES = [(32, 8, 128), (32, 8, 128), (28, 4, 128), (32, 32, 128), (8, 1, 128), (4, 1, 64), (12, 4, 64), (16, 8, 64)]
KV_BYTES = 7e8         # valid K and V rows of one drawn call, at most (below the largest listed case)
CACHE_BYTES = 1.2e9    # K and V caches of one drawn state, at most
ATTN_FLOPS = 5e10      # and products: the plain form takes them in 32 bits
TOKEN_BYTES = 1.5e8    # queries, keys and values that one drawn append or read brings, at most


def draw(rng):
    lens = rng.randrange(1000, 1 << 30)
    op = rng.choice(["append", "attn", "attn", "attn", "attn", "read", "compact", "pages"])
    if op == "pages":
        prompts = rng.random() < 0.4
        chunk_hi = _log_int(rng, 1, 2048 if prompts else 24)
        B = min(_log_int(rng, 1, 1024), max(1, 1000000 // chunk_hi))
        ctx_hi = _log_int(rng, 16, 8192)
        return _pages("", B, rng.choice([8, 16, 16, 32, 64, 128]), rng.choice([0, ctx_hi // 4]), ctx_hi, 1, chunk_hi, lens,
                      rng.choice([0.0, 0.05, 0.2, 0.6]))
    Hq, Hkv, D = rng.choice(SHAPES)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    page = rng.choice([0, 0, 16, 16, 64, 128])
    row = 2 * Hkv * (D // 2 + D // 32)   # K and V bytes of one cached token
    if op in ("append", "read"):
        tree = op == "append" and rng.random() < 0.3
        chunk_hi = _log_int(rng, 1, 24) if tree or rng.random() < 0.4 else _log_int(rng, 1, 4096)
        ctx_hi = _log_int(rng, 1, 32768)
        fresh = (Hq + 2 * Hkv) * D * ELT[dtype]
        most = max(1, min(int(CACHE_BYTES / (row * _round(ctx_hi + chunk_hi, 256))), int(TOKEN_BYTES / (fresh * chunk_hi))))
        return _case("", op, min(_log_int(rng, 1, 256), most), Hq, Hkv, D, dtype, rng.choice([0, ctx_hi // 4, ctx_hi]),
                     ctx_hi, rng.choice([chunk_hi, max(1, chunk_hi // 4)]), chunk_hi, lens, page=page, tree=tree,
                     norm=rng.random() < 0.4, rot=rng.choice([D, D, D // 2, D // 4, 0]),
                     rope=rng.choice(["halves", "halves", "pairs"]))
    tree = op == "compact" or rng.random() < 0.3
    chunk_hi = _log_int(rng, 2, 64) if op == "compact" else min(_log_int(rng, 1, 32 if tree else 16), 128 // (Hq // Hkv))
    ctx_hi = _log_int(rng, 64, 32768)
    ctx_lo = max(1, int(ctx_hi * rng.uniform(0.1, 1.0)))
    most = max(1, min(int(KV_BYTES / (row * (ctx_hi + chunk_hi))), int(CACHE_BYTES / (row * _round(ctx_hi + chunk_hi, 256))),
                      int(ATTN_FLOPS / (4 * Hq * D * chunk_hi * ctx_hi)) if op == "attn" else 256))
    return _case("", op, min(_log_int(rng, 1, 256), most), Hq, Hkv, D, dtype, ctx_lo, ctx_hi,
                 rng.choice([chunk_hi, chunk_hi, max(1, chunk_hi // 4)]), chunk_hi, lens, page=page, tree=tree)


def _round(x, m):
    return (x + m - 1) // m * m


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """Context and chunk lengths of the case, before the seed orders them."""
    rng = np.random.default_rng([case["lens"], 1])
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=case["B"])
    chunk = rng.integers(case["chunk_lo"], case["chunk_hi"] + 1, size=case["B"])
    return ctx, chunk


def _tree_words(seed, chunk, C):
    """Root-path words of random recursive trees (bit k of word i: token k is i
    or an ancestor of i)."""
    words = np.zeros((len(chunk), C), np.uint64)
    for b, c in enumerate(chunk):
        parent = np.random.default_rng([seed, 3, b]).integers(0, np.maximum(np.arange(c), 1))
        for i in range(c):
            words[b, i] = (words[b, parent[i]] if i else np.uint64(0)) | np.uint64(1 << i)
    return words


def _codes(x):
    """Codes (two to a byte) and scale bytes of rows of entries."""
    x = x.unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(most)                       # most = m 2^e, m in [0.5, 1)
    e = torch.where(m >= 0.875, e - 2, e - 3)      # the smallest e with most / 2^e < 7
    e = torch.where(most > 0, e.clamp(-126, 127), torch.full_like(e, -126))
    y = torch.ldexp(x, -e)
    a = y.abs()
    # one more for each border below: the odd codes' neighbours take the ties
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() +
            (a >= 3.5).byte() + (a > 5).byte() + 8 * torch.signbit(y).byte())
    fine = torch.isfinite(most)
    code = torch.where(fine, code, 0).flatten(-2)
    scale = torch.where(fine, e + 127, 255).squeeze(-1).byte()
    return code[..., 0::2] | code[..., 1::2] << 4, scale


def _values(codes, scales, dtype=torch.float32):
    """What codes and scale bytes stand for."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device, dtype=dtype)
    grid = torch.cat([grid, -grid])
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    x = torch.ldexp(grid[n.int()].unflatten(-1, (-1, 32)), scales.int().unsqueeze(-1) - 127)
    return torch.where(scales.unsqueeze(-1) == 255, math.nan, x).flatten(-2)


def _cache(case, seed, gen, dev, st):
    """K and V codes and scales, a slab per sequence or a shuffled pool of pages.
    Keys have channels of unlike size."""
    B, Hkv, D, S = case["B"], case["Hkv"], case["D"], _round(case["ctx_hi"] + case["chunk_hi"], 256)
    st["table"] = None
    shape = (B, Hkv, S)
    if case["page"]:
        n = B * (S // case["page"])
        shape = (n + 8, Hkv, case["page"])   # a pool with a few pages free
        table = np.random.default_rng([seed, 5]).permutation(n + 8)[:n].astype(np.int32)
        st["table"] = torch.from_numpy(table.reshape(B, -1)).to(dev)
    spread = torch.exp(0.5 * torch.randn((Hkv, 1, D), generator=gen, device=dev))
    st["cache"] = []
    for of in (spread, torch.ones_like(spread)):
        codes = torch.empty((*shape, D // 2), device=dev, dtype=torch.uint8)
        scales = torch.empty((*shape, D // 32), device=dev, dtype=torch.uint8)
        step = max(1, (1 << 26) // (Hkv * shape[2] * D))
        for i in range(0, shape[0], step):
            x = torch.randn((min(step, shape[0] - i), Hkv, shape[2], D), generator=gen, device=dev) * of
            codes[i:i + step], scales[i:i + step] = _codes(x)
        st["cache"] += [codes, scales]


def _append_state(case, seed, dev, gen, st):
    B, Hq, Hkv, D, C, dt = case["B"], case["Hq"], case["Hkv"], case["D"], case["chunk_hi"], DTYPES[case["dtype"]]
    # the output of one projection to queries, keys and values
    qkv = torch.randn((B, C, Hq + 2 * Hkv, D), generator=gen, device=dev, dtype=dt)
    st["new"] = [qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]]
    rot = case["rot"]
    st["inv_freq"] = None
    if rot:
        st["inv_freq"] = 1.0 / 10000.0 ** (torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
    st["rope"] = case["rope"]
    st["weights"] = [None, None]
    if case["norm"]:
        st["weights"] = [(1 + 0.1 * torch.randn((D,), generator=gen, device=dev)).to(dt) for _ in range(2)]
    st["q_out"] = torch.zeros((B, C, Hq, D), device=dev, dtype=dt)


def _pages_state(case, seed, dev, gen, st):
    """Two steps' lengths.  At the first every request holds its context; until the
    second, each has kept some of its chunk's tokens, and the share ``turnover`` of
    them has ended or, where there was none, begun.  The pool is large enough for
    most, not for all."""
    rng = np.random.default_rng([case["lens"], 6])
    ctx, chunk = _lengths(case)
    B, page = case["B"], case["page"]
    changed = rng.random((2, B)) < case["turnover"]
    first = [np.where(changed[0], 0, ctx), np.where(changed[0], 0, chunk)]
    kept = np.where(changed[0], 0, ctx + rng.integers(1, chunk + 1))
    nxt = [np.where(changed[1], 0, kept), np.where(changed[1], 0, rng.permutation(chunk))]
    order = np.random.default_rng([seed, 2]).permutation(B)
    put = lambda x: torch.from_numpy(np.ascontiguousarray(x[order]).astype(np.int32)).to(dev)   # noqa: E731
    st["steps"] = [[put(x) for x in first], [put(x) for x in nxt]]
    per = _round(case["ctx_hi"] + 2 * case["chunk_hi"], 256) // page
    held = -(-ctx[order] // page)
    n = int(held.sum()) + max(2, int(0.9 * (-(-chunk // page)).sum()))
    ids = np.random.default_rng([seed, 7]).permutation(n).astype(np.int32)
    table = np.full((B, per), -1, np.int32)
    used = 0
    for b in range(B):
        table[b, :held[b]] = ids[used:used + held[b]]
        used += held[b]
    st["page"] = page
    st["table"], st["held"] = torch.from_numpy(table).to(dev), torch.from_numpy(held.astype(np.int32)).to(dev)
    free = np.full(n, -1, np.int32)
    free[:n - used] = ids[used:]
    st["free"], st["count"] = torch.from_numpy(free).to(dev), torch.tensor([n - used], dtype=torch.int32, device=dev)
    st["missing"] = torch.zeros((B,), device=dev, dtype=torch.int32)
    st["slots"] = torch.zeros((B, case["chunk_hi"]), device=dev, dtype=torch.int64)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    st = dict(op=case["op"], mask=None)
    if case["op"] == "pages":
        _pages_state(case, seed, dev, gen, st)
        return st
    B, Hq, Hkv, D, C, dt = case["B"], case["Hq"], case["Hkv"], case["D"], case["chunk_hi"], DTYPES[case["dtype"]]
    order = np.random.default_rng([seed, 2]).permutation(B)
    ctx, chunk = (x[order].astype(np.int32) for x in _lengths(case))
    st["ctx"], st["chunk"] = torch.from_numpy(ctx).to(dev), torch.from_numpy(chunk).to(dev)
    words = None
    if case["tree"]:
        words = _tree_words(seed, chunk, C)
        st["mask"] = torch.from_numpy(words.view(np.int64)).to(dev)
    _cache(case, seed, gen, dev, st)
    if case["op"] == "append":
        _append_state(case, seed, dev, gen, st)
    if case["op"] == "attn":
        st["q"] = torch.randn((B, C, Hq, D), generator=gen, device=dev, dtype=dt)
        st["scale"] = 1.0 / math.sqrt(D)
        st["out"] = torch.empty((B, C, Hq, D), device=dev, dtype=dt)
        st["lse"] = torch.empty((B, C, Hq), device=dev, dtype=torch.float32)
        return st
    st["rows"] = st["chunk"]             # rows read back, from the context's end on
    if case["op"] == "compact":
        # the accepted path: the word of one of the tree's deepest tokens
        rng = np.random.default_rng([seed, 8])
        depth = np.array([[bin(int(w)).count("1") for w in row] for row in words])
        last = (depth * C + rng.integers(0, C, size=depth.shape)).argmax(1)
        st["path"] = torch.from_numpy(words[np.arange(B), last].view(np.int64)).to(dev)
        st["rows"] = torch.from_numpy(depth[np.arange(B), last].astype(np.int32)).to(dev)
    st["kv_out"] = [torch.zeros((B, C, Hkv, D), device=dev, dtype=dt) for _ in range(2)]
    return st


# ------------------------------------------------------------- plain forms

def _bits(words, C):
    """[B, C, C] truth values: token i sees draft token k."""
    return (words.unsqueeze(2) >> torch.arange(C, device=words.device)) & 1 > 0


def _places(st, C):
    """Index of the cache rows ctx + 0 .. C - 1 of every sequence (clamped into
    the cache), for a cache tensor [.., Hkv, rows, ..] with the heads last."""
    row = st["ctx"][:, None].long() + torch.arange(C, device=st["ctx"].device)
    at = torch.arange(row.shape[0], device=row.device)[:, None]
    page = st["cache"][0].shape[2]
    if st["table"] is None:
        return at, row.clamp(max=page - 1)
    row = row.clamp(max=page * st["table"].shape[1] - 1)
    return st["table"][at, row // page].long(), row % page


def _plain_read(st):
    """Rows ctx .. ctx + rows - 1 of every sequence."""
    C = st["kv_out"][0].shape[1]
    at, row = _places(st, C)
    valid = (torch.arange(C, device=row.device) < st["rows"][:, None])[:, :, None, None]
    for out, codes, scales in zip(st["kv_out"], st["cache"][0::2], st["cache"][1::2]):
        out.copy_(torch.where(valid, _values(codes[at, :, row], scales[at, :, row]).to(out.dtype), out))
    return st["kv_out"]


def _plain_append(st):
    """Keys in 64 bits up to their codes: a value next to a border between two
    codes goes to the one that the definition says."""
    q, k, v = st["new"]
    C = q.shape[1]
    dev = q.device
    i = torch.arange(C, device=dev)
    valid = i < st["chunk"][:, None]
    pos = st["ctx"][:, None].long() + i
    if st["mask"] is not None:
        seen = _bits(st["mask"], C) & valid[:, None, :]
        pos = st["ctx"][:, None].long() + seen.sum(2) - 1
    rotated = []
    for x, w, kind in ((q, st["weights"][0], torch.float32), (k, st["weights"][1], torch.float64)):
        x = x.to(kind)
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.to(kind)
        if st["inv_freq"] is not None:
            half = st["inv_freq"].numel()
            angle = pos[:, :, None, None].double() * st["inv_freq"]
            cos, sin = torch.cos(angle).to(kind), torch.sin(angle).to(kind)
            if st["rope"] == "halves":
                a, b = x[..., :half], x[..., half:2 * half]
                turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
            else:
                a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
                turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
            x = torch.cat([turned, x[..., 2 * half:]], -1)
        rotated.append(x)
    st["q_out"].copy_(torch.where(valid[:, :, None, None], rotated[0].to(q.dtype), st["q_out"]))
    at, row = _places(st, C)
    for n, x in ((0, rotated[1]), (2, v.float())):
        for cache, new in zip(st["cache"][n:n + 2], _codes(x)):
            cache[at, :, row] = torch.where(valid[:, :, None, None], new, cache[at, :, row])
    return (st["q_out"], *_plain_read(st))


def _plain_compact(st):
    C = st["kv_out"][0].shape[1]
    i = torch.arange(C, device=st["path"].device)
    bit = (st["path"][:, None] >> i) & 1 > 0
    # token of the j-th set bit; from the last one on, every row stays
    order = torch.sort(torch.where(bit, i, C), dim=1).values
    order = torch.where(i < bit.sum(1, keepdim=True), order, i)
    at, row = _places(st, C)
    source, from_row = at.expand_as(row).gather(1, order), row.gather(1, order)
    for cache in st["cache"]:
        cache[at, :, row] = cache[source, :, from_row]
    return _plain_read(st)


def _slab(st, n, dtype):
    """Keys (n = 0) or values (2) as [B, Hkv, S, D]."""
    codes, scales = st["cache"][n:n + 2]
    if st["table"] is not None:
        B, Hkv = st["table"].shape[0], codes.shape[1]
        codes, scales = (x[st["table"].long()].transpose(1, 2).reshape(B, Hkv, -1, x.shape[3]) for x in (codes, scales))
    return _values(codes, scales, dtype)


def _plain_attn(st):
    q, k, v = st["q"].float(), _slab(st, 0, torch.float32), _slab(st, 2, torch.float32)
    B, C, Hq, D = q.shape
    Hkv, S = k.shape[1:3]
    g, dev = Hq // Hkv, q.device
    i, j = torch.arange(C, device=dev), torch.arange(S, device=dev)
    ctx, chunk = st["ctx"][:, None, None].long(), st["chunk"][:, None].long()
    draft = j - ctx                     # [B, 1, S] draft token of a key, negative in the context
    if st["mask"] is None:
        seen = draft <= i[:, None]
    else:
        inside = (draft >= 0) & (draft < C)
        seen = torch.where(inside, _bits(st["mask"], C).gather(2, draft.clamp(0, C - 1).expand(B, C, S)), draft < 0)
    seen = seen & (draft < chunk[:, None])
    q = q.reshape(B, C, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, C * g, D)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * st["scale"]
    s = s.view(B, Hkv, C, g, S).masked_fill(~seen[:, None, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m.clamp(min=-3e38))
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, C * g, S), v).view(B, Hkv, C, g, D) / z.clamp(min=1e-37)
    valid = (i < chunk)[:, None, :, None]
    lse = (m + torch.log(z)).squeeze(-1).masked_fill(~valid, -math.inf)
    o = o.masked_fill(~valid[..., None], 0.0)
    out = o.permute(0, 2, 1, 3, 4).reshape(B, C, Hq, D).to(st["q"].dtype)
    return out, lse.permute(0, 2, 1, 3).reshape(B, C, Hq)


def _plain_step(st, ctx, chunk):
    """Pages that a request no longer needs go on the stack of free ones, in order;
    then the requests take theirs from its top, in order, until one finds too few."""
    table, held, free, page = st["table"], st["held"].long(), st["free"], st["page"]
    B, per = table.shape
    n, C = free.numel(), st["slots"].shape[1]
    ctx, chunk = ctx.long(), chunk.long()
    need = (ctx + chunk + page - 1) // page
    count = st["count"].long()
    back, want = (held - need).clamp(min=0), (need - held).clamp(min=0)
    back_end, want_end = back.cumsum(0), want.cumsum(0)
    total = count + back_end[-1]
    j = torch.arange(per, device=table.device)
    # the stack with what comes back (entry n: a place for what does not)
    stack = torch.cat([free, free[:1]])
    going = (j >= need[:, None]) & (j < held[:, None])
    to = torch.where(going, count + (back_end - back)[:, None] + j - need[:, None], n)
    stack[to] = torch.where(going, table, stack[n])
    served = want_end <= total
    taken = torch.where(served, want_end, 0).amax()
    coming = served[:, None] & (j >= held[:, None]) & (j < need[:, None])
    source = torch.where(coming, total - 1 - (want_end - want)[:, None] - (j - held[:, None]), 0)
    st["table"].copy_(torch.where(coming, stack[source], table))
    st["held"].copy_(torch.where(served, need, torch.minimum(held, need)))
    free.copy_(stack[:n])
    st["count"].copy_(total - taken)
    st["missing"].copy_(torch.where(served, 0, want))
    i = torch.arange(C, device=table.device)
    row = ctx[:, None] + i
    there = (i < chunk[:, None]) & (row < page * st["held"][:, None])
    slot = st["table"].gather(1, (row // page).clamp(max=per - 1)).long() * page + row % page
    st["slots"].copy_(torch.where(there, slot, -1))


def _plain_pages(st):
    for ctx, chunk in st["steps"]:
        _plain_step(st, ctx, chunk)
    return {n: st[n] for n in ("table", "held", "free", "count", "missing", "slots")}


# --------------------------------------------------------------- own calls

def _own_run(st):
    import paper_2508_21706_amd as sm

    op = st["op"]
    if op == "pages":
        pages = sm.PageState(st["table"], st["held"], st["free"], st["count"])
        for ctx, chunk in st["steps"]:
            sm.assign_pages(ctx, chunk, pages, st["page"], missing=st["missing"], slots=st["slots"])
        return {n: st[n] for n in ("table", "held", "free", "count", "missing", "slots")}
    cache = sm.KV4Cache(*st["cache"])
    if op == "attn":
        if "ws" not in st:   # a serving loop's, kept between its steps
            st["ws"] = sm.alloc_kv4_workspace(st["q"], cache, block_table=st["table"])
        return sm.verify_attn_kv4(st["q"], cache, st["ctx"], st["chunk"], st["scale"], draft_mask=st["mask"],
                                  block_table=st["table"], out=st["out"], lse=st["lse"], workspace=st["ws"])
    if op == "append":
        q, k, v = st["new"]
        sm.append_kv4(q, k, v, cache, st["ctx"], st["chunk"], inv_freq=st["inv_freq"], rope=st["rope"],
                      q_weight=st["weights"][0], k_weight=st["weights"][1], eps=1e-6, draft_mask=st["mask"],
                      block_table=st["table"], q_out=st["q_out"])
    if op == "compact":
        sm.compact_accepted_kv4(cache, st["ctx"], st["path"], block_table=st["table"])
    sm.read_kv4(cache, st["ctx"], st["rows"], out=st["kv_out"], block_table=st["table"])
    return (st["q_out"], *st["kv_out"]) if op == "append" else st["kv_out"]


def run(st):
    if own:
        return _own_run(st)
    return {"append": _plain_append, "attn": _plain_attn, "read": _plain_read, "compact": _plain_compact,
            "pages": _plain_pages}[st["op"]](st)


def work(case):
    ctx, chunk = _lengths(case)
    B, tokens = case["B"], int(chunk.sum())
    if case["op"] == "pages":
        # two steps: the lengths and counts, the slots, and the pages that come and go (about)
        moved = 2 * int((chunk // case["page"]).sum()) + int(2 * case["turnover"] * (ctx // case["page"]).sum())
        return {"bytes": 2 * (8 * B * case["chunk_hi"] + 20 * B) + 8 * moved, "flops": 0}
    Hq, Hkv, D, elt = case["Hq"], case["Hkv"], case["D"], ELT[case["dtype"]]
    row, wide = 2 * Hkv * (D // 2 + D // 32), 2 * Hkv * D * elt
    if case["op"] == "append":
        # the chunk's queries, keys and values, read and written; the written rows read back
        return {"bytes": tokens * (2 * Hq * D * elt + wide + 2 * row + wide) + 8 * B, "flops": 0}
    if case["op"] == "read":
        return {"bytes": tokens * (row + wide) + 8 * B, "flops": 0}
    if case["op"] == "compact":
        # paths of about 2 ln c tokens, moved and read back
        path = int(np.ceil(2 * np.log(np.maximum(chunk, 2))).sum())
        return {"bytes": path * (3 * row + wide) + 16 * B, "flops": 0}
    T = ctx + chunk
    # (the padding rows are written too)
    return {"bytes": int(T.sum()) * row + tokens * Hq * D * elt + B * case["chunk_hi"] * Hq * (D * elt + 4),
            "flops": 4 * Hq * D * int((chunk * T).sum())}


# ---------------------------------------------- the definitions in 64 bits

def _exact_codes(x):
    """The values that rows of entries are kept as: the nearest of the grid at the
    block's scale, of two as near the one whose code is even."""
    b = x.double().reshape(*x.shape[:-1], -1, 32)
    most = b.abs().amax(-1, keepdim=True)
    power = torch.floor(torch.log2(most.clamp(min=1e-300))) - 4
    for _ in range(6):   # (the logarithm may be off by one)
        power = torch.where(most / torch.exp2(power) >= 7, power + 1, power)
    power = power.clamp(-126, 127)
    grid = torch.tensor([0, 1, 2, 4, 0.5, 1.5, 3, 6], device=x.device, dtype=torch.float64)   # even codes, then odd ones
    unit = torch.exp2(power)
    res = torch.empty_like(b)
    flat, out, per = (b / unit).abs().reshape(-1), res.view(-1), 1 << 24
    for i in range(0, flat.numel(), per):
        out[i:i + per] = grid[(flat[i:i + per, None] - grid).abs().argmin(-1)]
    return (torch.copysign(res, b) * unit).reshape(x.shape)


def _exact_cached(st, b, first, n, which):
    """Rows first .. first + n - 1 of sequence b as [Hkv, n, D] (which: 0 keys, 2 values)."""
    codes, scales = st["cache"][which:which + 2]
    rows = torch.arange(first, first + n, device=codes.device)
    if st["table"] is None:
        codes, scales = codes[b][:, rows], scales[b][:, rows]
    else:
        page = st["table"][b].long()[rows // codes.shape[2]]
        codes, scales = (x[page, :, rows % x.shape[2]].transpose(0, 1) for x in (codes, scales))
    x = torch.empty((*codes.shape[:2], 2 * codes.shape[2]), dtype=torch.float64, device=codes.device)
    for h in (0, 1):
        n = (codes.long() >> 4 * h) & 15
        m, e = n & 1, (n >> 1) & 3
        x[..., h::2] = torch.where(e > 0, (2.0 + m) * torch.exp2(e - 2.0), m / 2) * torch.where(n > 7, -1.0, 1.0)
    return x * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def _exact_append(st):
    q, k, v = st["new"]
    res = [st["q_out"].double(), st["kv_out"][0].double(), st["kv_out"][1].double()]
    for b, (l, c) in enumerate(zip(st["ctx"].tolist(), st["chunk"].tolist())):
        pos = torch.arange(l, l + c, device=q.device).double()
        if st["mask"] is not None:
            words = [int(w) & ((1 << c) - 1) for w in st["mask"][b, :c].tolist()]
            pos = torch.tensor([l + bin(w).count("1") - 1 for w in words], device=q.device).double()
        for n, x, w in ((0, q, st["weights"][0]), (1, k, st["weights"][1])):
            x = x[b, :c].double()
            if w is not None:
                x = w.double() * x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + 1e-6)
            x = x.clone()
            if st["inv_freq"] is not None:
                half = st["inv_freq"].numel()
                turn = torch.polar(torch.ones((), device=q.device).double(), pos[:, None] * st["inv_freq"])[:, None]
                at = (slice(0, half), slice(half, 2 * half)) if st["rope"] == "halves" else (
                    slice(0, 2 * half, 2), slice(1, 2 * half, 2))
                z = torch.complex(x[..., at[0]].contiguous(), x[..., at[1]].contiguous()) * turn
                x[..., at[0]], x[..., at[1]] = z.real, z.imag
            res[n][b, :c] = x if n == 0 else _exact_codes(x)
        res[2][b, :c] = _exact_codes(v[b, :c])
    return tuple(res)


def _exact_read(st):
    res = [x.double() for x in st["kv_out"]]
    paths = st["path"].tolist() if st["op"] == "compact" else [None] * len(st["ctx"])
    for b, (l, n, path) in enumerate(zip(st["ctx"].tolist(), st["rows"].tolist(), paths)):
        for out, which in zip(res, (0, 2)):
            if path is None:
                out[b, :n] = _exact_cached(st, b, l, n, which).transpose(0, 1)
            else:
                nodes = [i for i in range(64) if path >> i & 1]
                rows = _exact_cached(st, b, l, nodes[-1] + 1, which)
                out[b, :n] = rows[:, nodes].transpose(0, 1)
    return res


def _exact_attn(st):
    B, C, Hq, D = st["q"].shape
    Hkv, dev = st["cache"][0].shape[1], st["q"].device
    g = Hq // Hkv
    out = torch.zeros((B, C, Hq, D), dtype=torch.float64, device=dev)
    lse = torch.full((B, C, Hq), -math.inf, dtype=torch.float64, device=dev)
    for b, (l, c) in enumerate(zip(st["ctx"].tolist(), st["chunk"].tolist())):
        T = l + c
        k, v = _exact_cached(st, b, 0, T, 0), _exact_cached(st, b, 0, T, 2)
        sees = torch.ones((c, T), dtype=torch.bool, device=dev).tril(l)
        if st["mask"] is not None:
            words = st["mask"][b, :c].tolist()
            sees[:, l:] = torch.tensor([[w >> n & 1 for n in range(c)] for w in words], device=dev) > 0
        q = st["q"][b, :c].double().reshape(c, Hkv, g, D).permute(1, 2, 0, 3).reshape(Hkv, g * c, D)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()).view(Hkv, g, c, T) * st["scale"]
        s = torch.where(sees, s, -math.inf)
        z = torch.logsumexp(s, -1)
        o = torch.matmul(torch.exp(s - z[..., None]).view(Hkv, g * c, T), v.contiguous()).view(Hkv, g, c, D)
        out[b, :c] = o.permute(2, 0, 1, 3).reshape(c, Hq, D)
        lse[b, :c] = z.permute(2, 0, 1).reshape(c, Hq)
    return out, lse


def exact(case, seed):
    if case["op"] == "pages":
        return None   # whole numbers only
    st = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn}.get(case["op"], _exact_read)(st)
