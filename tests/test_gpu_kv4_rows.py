"""verify_attn_kv4 where a wave has two row blocks (units of more than 16 rows in 16-bit
types, of more than 64 in float32): every type, head dim and placement of the cache,
with chains, trees and units that ranges cut, against the float64 oracle with the
tolerances of test_gpu_kv4_attn; and calls repeated give the same bits."""
import numpy as np
import pytest
import torch

from test_gpu_kv4_attn import call, check, make, on_gpu
from test_gpu_parity import note

pytestmark = pytest.mark.gpu

# (query heads, KV heads, chunk): rows of the longest chunk, past one wave's block up to all eight blocks
LAYOUTS = {"bf16": [(8, 2, 5), (7, 1, 9), (8, 1, 16)], "f16": [(8, 2, 5), (7, 1, 9), (8, 1, 16)],
           "f32": [(10, 2, 14), (7, 1, 13), (8, 1, 16)]}
ALL = [(dtype, D, page) for dtype in ("bf16", "f16", "f32") for D in (64, 128) for page in (0, 8, 16)]


def twice(x, label, **kw):
    note(f"case {label}")
    cache, table = on_gpu(x)
    first = call(x, cache, table, **kw)
    check(x, *first, label=label)
    again = call(x, cache, table, **kw)
    assert all(torch.equal(a, b) for a, b in zip(first, again)), f"{label}: another result the second time"


@pytest.mark.parametrize("layout", [0, 1, 2])
@pytest.mark.parametrize("dtype,D,page", ALL)
def test_chains(dtype, D, page, layout):
    Hq, Hkv, C = LAYOUTS[dtype][layout]
    x = make(40 + layout, dtype, [70, 5, 200, 0, 131], [C, C // 2, 1, C - 1, 0], Hq=Hq, Hkv=Hkv, D=D, C=C, page=page)
    twice(x, f"{dtype} {D} page {page} {Hq}/{Hkv} chunk {C}")


@pytest.mark.parametrize("dtype,D,page", ALL)
def test_trees(dtype, D, page):
    x = make(50, dtype, [0, 100, 17, 250, 64], [16, 16, 9, 1, 0], Hq=6, Hkv=1, D=D, C=16, page=page, tree=True)
    twice(x, f"tree {dtype} {D} page {page}")


@pytest.mark.parametrize("grid", [1, 3, 40])
@pytest.mark.parametrize("dtype,D,page", ALL)
def test_cut_units(dtype, D, page, grid):
    """Ranges end inside units, in their first and last tiles and at their ends."""
    Hq, Hkv, C = LAYOUTS[dtype][0]
    x = make(60, dtype, [900, 3, 640, 127], [C, C, 2, C - 1], Hq=Hq, Hkv=Hkv, D=D, C=C, page=page)
    twice(x, f"cut {dtype} {D} page {page} grid {grid}", grid_blocks=grid)


@pytest.mark.parametrize("dtype,D", [(dtype, D) for dtype in ("bf16", "f16", "f32") for D in (64, 128)])
def test_repeated_calls_agree(dtype, D):
    """Many steps in which nothing is masked, by all workgroups."""
    Hq, Hkv, C = LAYOUTS[dtype][0]
    ctx = np.random.default_rng(70).integers(300, 3000, size=24).tolist()
    x = make(70, dtype, ctx, [C] * 24, Hq=Hq, Hkv=Hkv, D=D, C=C, page=16)
    cache, table = on_gpu(x)
    first = call(x, cache, table)
    check(x, *first, label=f"repeated {dtype} {D}", rows=[0, 23])
    for _ in range(8):
        assert all(torch.equal(a, b) for a, b in zip(first, call(x, cache, table)))
