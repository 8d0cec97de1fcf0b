"""Lengths out of range in the calls that read, append and move rows of a 4-bit cache:
clamped before anything is subtracted from them, so nothing around the outputs and the
cache changes.  Every buffer is the inner part of a larger one."""
import numpy as np
import pytest
import torch

import paper_2508_21706_amd as pkg
from test_gpu_kv4 import i32, make, make_cache
from test_gpu_parity import dev, note

pytestmark = pytest.mark.gpu

LEAST, MOST = -(1 << 31), (1 << 31) - 1


def inside(*shape, dtype, guard=4096):
    """(a tensor of the shape, the flat one around it), filled with 7."""
    n = int(np.prod(shape))
    flat = torch.full((n + 2 * guard,), 7, dtype=dtype, device=dev())
    return flat[guard:guard + n].view(shape), flat


@pytest.mark.parametrize("N", [5, 4, 1, 30])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_to_read(N, dtype):
    """No rows for any negative number, as many as the output holds for a large one."""
    cache, table = make_cache(90, 3, 2, 64, 64, 8)
    for rows in ([LEAST, LEAST + 3, -1], [0, LEAST, LEAST + 1], [MOST, LEAST, 2]):
        note(f"case rows {rows} of {N}")
        pair = [inside(3, N, 2, 64, dtype=dtype) for _ in range(2)]
        pkg.read_kv4(cache, i32([3, 7, 20]), i32(rows), out=(pair[0][0], pair[1][0]), block_table=table)
        ref = pkg.read_kv4(cache, i32([3, 7, 20]), i32([min(max(r, 0), N) for r in rows]), N, dtype=dtype, block_table=table)
        torch.cuda.synchronize()
        for (got, flat), want in zip(pair, ref):
            assert (flat[:4096] == 7).all() and (flat[-4096:] == 7).all()
            for b, r in enumerate(rows):
                r = min(max(r, 0), N)
                assert torch.equal(got[b, :r].nan_to_num(9.0), want[b, :r].nan_to_num(9.0)) and (got[b, r:] == 7).all()


def test_first_rows_out_of_range():
    """Negative ones count as 0; what would lie past the cache stays."""
    cache, _ = make_cache(91, 3, 2, 64, 32)
    (k, k_flat), (v, v_flat) = (inside(3, 6, 2, 64, dtype=torch.float32) for _ in range(2))
    pkg.read_kv4(cache, i32([LEAST, MOST, 30]), i32([6, 6, 6]), out=(k, v))
    ref = pkg.read_kv4(cache, i32([0, 0, 30]), i32([6, 0, 2]), 6, dtype=torch.float32)
    torch.cuda.synchronize()
    for got, flat, want in ((k, k_flat, ref[0]), (v, v_flat, ref[1])):
        assert torch.equal(got[0].nan_to_num(9.0), want[0].nan_to_num(9.0)) and (got[1] == 7).all()
        assert torch.equal(got[2, :2].nan_to_num(9.0), want[2, :2].nan_to_num(9.0)) and (got[2, 2:] == 7).all()
        assert (flat[:4096] == 7).all() and (flat[-4096:] == 7).all()


def test_lengths_of_appends_and_moves():
    """Chunks of a negative length write nothing, contexts of one begin at row 0, and rows
    past the cache are dropped."""
    x = make(92, "bf16", 4, 2, 2, 64, 3)
    shapes = [(4, 2, 16, 32), (4, 2, 16, 2)] * 2
    buffers = [inside(*s, dtype=torch.uint8) for s in shapes]
    cache = pkg.KV4Cache(*(t for t, _ in buffers))
    pkg.append_kv4(x["q"], x["k"], x["v"], cache, i32([LEAST, 5, MOST, 14]), i32([2, LEAST, 3, MOST]), q_out=x["q_out"])
    pkg.compact_accepted_kv4(cache, i32([LEAST, 5, MOST, 14]), torch.tensor([2, 0, -2, -4], device=dev()))
    ref = pkg.KV4Cache(*(torch.full(s, 7, dtype=torch.uint8, device=dev()) for s in shapes))
    pkg.append_kv4(x["q"], x["k"], x["v"], ref, i32([0, 5, 16, 14]), i32([2, 0, 0, 2]))
    pkg.compact_accepted_kv4(ref, i32([0, 5, 15, 14]), torch.tensor([2, 0, 0, 0], device=dev()))
    torch.cuda.synchronize()
    for (got, flat), want in zip(buffers, ref):
        assert torch.equal(got, want) and (flat[:4096] == 7).all() and (flat[-4096:] == 7).all()
