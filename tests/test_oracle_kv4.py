"""The oracle of the 4-bit cache and of pages from lengths, pinned to worked
examples and closed forms."""
import numpy as np
import pytest

from oracle.kv4 import (VALUES, assign_pages_ref, cache_append_ref, cache_move_ref, cache_rows_ref, decode_ref,
                        encode_block_ref, encode_ref)


def block(*head):
    return np.array(list(head) + [0.0] * (32 - len(head)))


def test_every_code_and_scale_decodes():
    codes = np.array([[0x10, 0x32, 0x54, 0x76, 0x98, 0xba, 0xdc, 0xfe] * 2], np.uint8)
    for byte, unit in ((127, 1.0), (128, 2.0), (120, 2.0 ** -7), (1, 2.0 ** -126), (0, 2.0 ** -127), (254, 2.0 ** 127)):
        got = decode_ref(codes, np.array([[byte]], np.uint8))[0]
        want = np.array((VALUES + [-v for v in VALUES]) * 2) * unit
        assert np.array_equal(got, want)
    assert np.isnan(decode_ref(codes, np.array([[255]], np.uint8))).all()


@pytest.mark.parametrize("most,unit", [(6.0, 1.0), (6.99, 1.0), (7.0, 2.0), (3.5, 1.0), (3.49, 0.5), (0.875, 0.25),
                                       (0.87, 0.125), (2.0 ** 100, 2.0 ** 98), (2.0 ** -126, 2.0 ** -126)])
def test_the_unit_is_the_smallest_that_leaves_the_largest_below_7(most, unit):
    byte, codes, _ = encode_block_ref(block(0.1 * most, -most))
    assert 2.0 ** (byte - 127.0) == unit
    assert codes[1] & 8 and VALUES[codes[1] & 7] <= 6


def test_ties_go_to_the_even_code():
    x = block(6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, 0.2500001, 4.9999)
    byte, codes, near = encode_block_ref(x)
    assert byte == 127 and near == 0
    assert codes[:12] == [7, 0, 2, 2, 4, 4, 6, 6, 8, 14, 1, 6]


def test_a_block_of_zeros_and_blocks_without_a_value():
    assert encode_block_ref(block())[:2] == (1, [0] * 32)
    for bad in (np.inf, -np.inf, np.nan, 4e38):
        assert encode_block_ref(block(1.0, bad))[:2] == (255, [0] * 32)


def test_values_of_the_grid_come_back():
    rng = np.random.default_rng(1)
    unit = 2.0 ** rng.integers(-20, 20, size=(5, 4, 1))
    x = rng.choice(VALUES, size=(5, 4, 32)) * rng.choice([-1, 1], size=(5, 4, 32))
    x[:, :, 0] = 6.0
    x = (x * unit).reshape(5, 128)
    codes, scales, _ = encode_ref(x)
    assert np.array_equal(decode_ref(codes, scales), x)


def test_rounding_is_to_nearest():
    x = np.random.default_rng(2).standard_normal((50, 64))
    codes, scales, _ = encode_ref(x)
    unit = np.repeat(2.0 ** (scales - 127.0), 32, axis=-1)
    a = np.abs(x) / unit
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))   # (above 6 the values up to 7 round to 6)
    assert (np.abs(decode_ref(codes, scales) - x) <= step / 2 * unit + 1e-15).all()


def test_append_read_and_move_agree():
    rng = np.random.default_rng(3)
    B, C, Hkv, D, page = 2, 5, 2, 64, 8
    cache = [rng.integers(0, 256, size=(7, Hkv, page, n)).astype(np.uint8) for n in (32, 2, 32, 2)]
    table = np.array([[3, 0, 5], [1, 6, 2]])
    k, v, q = (rng.standard_normal((B, C, Hkv, D)) for _ in range(3))
    got_q, new, near = cache_append_ref(q, k, v, cache, q * 0, [6, 0], [5, 3], table=table)
    assert np.array_equal(got_q[0], q[0]) and np.array_equal(got_q[1, 3:], 0 * q[1, 3:])
    assert np.isfinite(near[0]).all() and np.isinf(near[1, 3:]).all()
    rk, rv = cache_rows_ref(new, 0, 6, 5, table)
    assert np.array_equal(rk, decode_ref(*encode_ref(k[0])[:2])) and np.array_equal(rv, decode_ref(*encode_ref(v[0])[:2]))
    assert np.array_equal(new[0][3, :, :6], cache[0][3, :, :6])          # rows before the chunk
    moved = cache_move_ref(new, [6, 0], [0b10101, 0b11], 24, table)
    mk, _ = cache_rows_ref(moved, 0, 6, 3, table)
    assert np.array_equal(mk, rk[[0, 2, 4]])
    assert np.array_equal(moved[0][table[1]], new[0][table[1]])


def test_pages_worked_example():
    """Pages of 8.  Request 0 shrinks from 3 pages to 1, request 1 grows from 1 to 2,
    request 2 ends, request 3 begins with 2, request 4 asks for 5 when 1 is left."""
    table = np.array([[10, 11, 12, 0, 0], [13, 0, 0, 0, 0], [14, 0, 0, 0, 0], [0] * 5, [0] * 5])
    free = np.array([20, 0, 0, 0, 0, 0])
    r = assign_pages_ref(np.array([5, 8, 0, 0, 33]), np.array([3, 2, 0, 9, 3]), table, np.array([3, 1, 1, 0, 0]), free, 1,
                         8, 4)
    # the stack after the returns: 20 11 12 14; request 1 takes 14, request 3 (chunk clamped to 4) takes 12
    assert r["held"].tolist() == [1, 2, 0, 1, 0] and r["missing"].tolist() == [0, 0, 0, 0, 5]
    assert r["table"][1, :2].tolist() == [13, 14] and r["table"][3, 0] == 12
    assert r["free_count"] == 2 and r["free_pages"].tolist() == [20, 11, 12, 14, 0, 0]
    assert r["slots"].tolist() == [[85, 86, 87, -1], [112, 113, -1, -1], [-1] * 4, [96, 97, 98, 99], [-1] * 4]


def test_pages_nothing_is_lost_or_doubled():
    rng = np.random.default_rng(4)
    B, per, n = 40, 12, 150
    table, held, free, count = np.zeros((B, per), int), np.zeros(B, int), np.arange(n), n
    for step in range(60):
        ctx = np.where(rng.random(B) < 0.1, 0, rng.integers(0, 90, size=B))
        chunk = np.where(ctx == 0, 0, rng.integers(0, 7, size=B))
        r = assign_pages_ref(ctx, chunk, table, held, free, count, 8, 6)
        table, held, free, count = r["table"], r["held"], r["free_pages"], r["free_count"]
        everything = [p for b in range(B) for p in table[b, :held[b]]] + list(free[:count])
        assert sorted(everything) == list(range(n))
        need = -(-(ctx + chunk) // 8)
        assert (held + r["missing"] == need).all()
