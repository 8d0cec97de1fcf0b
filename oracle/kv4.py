"""Plain CPU oracle of the 4-bit KV cache and of pages from lengths.

TEST INFRASTRUCTURE, NOT PART OF THE PRODUCT.  It shares no code with the HIP
path and imports nothing from it.

  * ``encode_ref`` / ``decode_ref``: a block of 32 entries to its scale byte and
    codes, by search over the values that a code stands for, and back;
  * ``cache_append_ref``, ``cache_rows_ref``, ``cache_move_ref``: rows of a cache (slabs or
    pages) written, read and moved;
  * ``assign_pages_ref``: the hand-out of pages, one request after the other.
"""
from __future__ import annotations

import math

import numpy as np

from .step import head_ref, positions_ref

VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]   # of the codes 0 .. 7


def decode_ref(codes, scales):
    """float64 values of rows of packed codes [.., D / 2] and scale bytes [.., D / 32]."""
    codes, scales = np.asarray(codes, np.uint8), np.asarray(scales, np.uint8)
    n = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    x = np.array(VALUES + [-v for v in VALUES])[n]
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.int64) - 127.0))
    return x * np.repeat(unit, 32, axis=-1)


def encode_block_ref(x):
    """(scale byte, 32 codes, distance of the nearest border between two codes in
    units) of one block of 32 values; ties go to the even code."""
    x = np.asarray(x, np.float64)
    with np.errstate(over="ignore"):
        as_f32 = x.astype(np.float32)
    if not np.isfinite(as_f32).all():
        return 255, [0] * 32, math.inf
    most = float(np.abs(x).max())
    e = -126
    while most / 2.0 ** e >= 7:
        e += 1
    codes, near = [], math.inf
    for v in np.abs(x) / 2.0 ** e:
        best = min(range(8), key=lambda c: (abs(VALUES[c] - v), c & 1))
        near = min(near, min(abs(v - (a + b) / 2) for a, b in zip(VALUES, VALUES[1:])))
        codes.append(best)
    codes = [c | 8 if math.copysign(1.0, v) < 0 else c for c, v in zip(codes, x)]
    return e + 127, codes, near


def encode_ref(x):
    """Packed codes, scale bytes and border distances [.., D / 32] of rows of values."""
    x = np.asarray(x, np.float64)
    flat = x.reshape(-1, 32)
    codes, scales, near = np.zeros((len(flat), 16), np.uint8), np.zeros(len(flat), np.uint8), np.zeros(len(flat))
    for i, block in enumerate(flat):
        scales[i], c, near[i] = encode_block_ref(block)
        codes[i] = [c[2 * j] | c[2 * j + 1] << 4 for j in range(16)]
    lead = x.shape[:-1]
    return codes.reshape(*lead, -1), scales.reshape(*lead, -1), near.reshape(*lead, -1)


def where_ref(b: int, row: int, rows: int, table=None):
    """(slab or page, row there) of row ``row`` of sequence b; ``rows``: of a slab or page."""
    if table is None:
        return b, row
    return int(table[b][row // rows]), row % rows


def cache_append_ref(q, k, v, cache, q_out, ctx_lens, chunk_lens, inv_freq=None, rope="halves", q_weight=None,
                     k_weight=None, eps=1e-6, words=None, table=None):
    """(q_out float64, [k_codes, k_scales, v_codes, v_scales], distances of the keys' blocks to a
    border) after the append, as copies; distances [B, C, Hkv, D / 32]."""
    q_out, cache = np.array(q_out, np.float64), [np.array(x) for x in cache]
    B, C, Hkv, D = k.shape
    near = np.full((B, C, Hkv, D // 32), np.inf)
    for b, (l, c) in enumerate(zip(ctx_lens, chunk_lens)):
        for i, pos in enumerate(positions_ref(int(l), int(c), None if words is None else words[b])):
            for h in range(q.shape[2]):
                q_out[b, i, h] = head_ref(q[b, i, h], pos, inv_freq, rope, q_weight, eps)
            at, row = where_ref(b, int(l) + i, cache[0].shape[2], table)
            for h in range(Hkv):
                key = head_ref(k[b, i, h], pos, inv_freq, rope, k_weight, eps)
                cache[0][at, h, row], cache[1][at, h, row], near[b, i, h] = encode_ref(key)
                cache[2][at, h, row], cache[3][at, h, row], _ = encode_ref(v[b, i, h])
    return q_out, cache, near


def cache_rows_ref(cache, b: int, first: int, n: int, table=None):
    """Keys and values [n, Hkv, D] that rows first .. first + n - 1 of sequence b stand for."""
    Hkv, D = cache[0].shape[1], 2 * cache[0].shape[3]
    k, v = np.zeros((n, Hkv, D)), np.zeros((n, Hkv, D))
    for i in range(n):
        at, row = where_ref(b, first + i, cache[0].shape[2], table)
        k[i], v[i] = decode_ref(cache[0][at, :, row], cache[1][at, :, row]), decode_ref(cache[2][at, :, row],
                                                                                       cache[3][at, :, row])
    return k, v


def cache_move_ref(cache, ctx_lens, path, S_max: int, table=None):
    """The cache after each sequence's path rows moved right behind its context."""
    old, cache = cache, [np.array(x) for x in cache]
    for b, l in enumerate(ctx_lens):
        nodes = [n for n in range(64) if int(path[b]) >> n & 1]
        for j, node in enumerate(nodes):
            if int(l) + node >= S_max:
                continue
            src = where_ref(b, int(l) + node, old[0].shape[2], table)
            dst = where_ref(b, int(l) + j, old[0].shape[2], table)
            for x, y in zip(cache, old):
                x[dst[0], :, dst[1]] = y[src[0], :, src[1]]
    return cache


def assign_pages_ref(ctx_lens, chunk_lens, table, held, free_pages, free_count, page_size: int, C_max: int):
    """Dict of table, held, free_pages, free_count, missing and slots after the step."""
    table, held, free = np.array(table), np.array(held), np.array(free_pages)
    B, per = table.shape
    stack = [int(x) for x in free[:free_count]]
    l = np.minimum(np.maximum(ctx_lens, 0), per * page_size)
    c = np.minimum(np.clip(chunk_lens, 0, C_max), per * page_size - l)
    need = -(-(l + c) // page_size)
    for b in range(B):
        for j in range(int(need[b]), int(held[b])):
            free[len(stack)] = table[b, j]
            stack.append(int(table[b, j]))
        held[b] = min(held[b], need[b])
    missing = np.zeros(B, np.int32)
    short = False
    for b in range(B):
        want = int(need[b] - held[b])
        short = short or want > len(stack)
        if short:
            missing[b] = want
            continue
        for _ in range(want):
            table[b, held[b]] = stack.pop()
            held[b] += 1
    slots = np.full((B, C_max), -1, np.int64)
    for b in range(B):
        for i in range(int(c[b])):
            pos = int(l[b]) + i
            if pos // page_size < held[b]:
                slots[b, i] = int(table[b, pos // page_size]) * page_size + pos % page_size
    return dict(table=table, held=held, free_pages=free, free_count=len(stack), missing=missing, slots=slots)
