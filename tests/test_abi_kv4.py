"""Host-only checks of the 4-bit cache's and the pages' entry points: arguments are
refused before any HIP call (so these run without a GPU), and the binding's structs
mirror the headers'."""
import ctypes
import os
import re

import pytest
import torch

import paper_2508_21706_amd as pkg
from paper_2508_21706_amd import binding as bd

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
FAKE = 0x10000          # 16-byte aligned, never dereferenced by these tests
MEMBERS = ("k_codes", "k_scales", "v_codes", "v_scales")


@pytest.fixture(scope="module")
def lib():
    return bd.load_library()


@pytest.mark.parametrize("header,struct,mirror", [
    ("specmoe_kv4.h", "specmoe_kv4", bd.KV4),
    ("specmoe_kv4.h", "specmoe_kv4_desc", bd.KV4Desc),
    ("specmoe_pages.h", "specmoe_pages_desc", bd.PagesDesc),
])
def test_structs_match_the_headers(header, struct, mirror):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, header)).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (struct, struct), text, re.S).group(1)
    fields = [(n, ctypes.c_void_p if star else ctypes.c_int32)
              for _, star, n in re.findall(r"(\w+)\s*(\*?)\s*(\w+)\s*;", body)]
    assert fields == list(mirror._fields_)


def test_headers_are_plain_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "specmoe_kv4.h"\n#include "specmoe_pages.h"\nint main(void) { return 0; }\n')
    assert os.system(f"gcc -std=c99 -Wall -Werror -I{INCLUDE} -c {src} -o {tmp_path / 'use.o'}") == 0


def ref(s):
    return None if s is None else ctypes.byref(s)


def kv4(**kw):
    return bd.KV4(**dict(dict.fromkeys(MEMBERS, FAKE), **kw))


APPEND = ["q", "k", "v", "q_weight", "k_weight", "inv_freq", "ctx_lens", "chunk_lens", "draft_mask", "block_table",
          "q_out", "cache", "stream"]


def append_desc(**kw):
    return bd.AppendDesc(**dict(dict(B=2, Hq=32, Hkv=8, D=128, C_max=5, S_max=256, dtype=bd.SPECMOE_BF16, rot_dim=128,
                                     rope_style=0, norm_eps=1e-6, q_stride=0, k_stride=0, v_stride=0), **kw))


def append(lib, desc, paged=None, **kw):
    args = dict.fromkeys(APPEND, FAKE)
    args.update(cache=kv4(), draft_mask=None, block_table=None if paged is None else FAKE, stream=None)
    args.update(kw)
    args["cache"] = ref(args["cache"])
    return lib.specmoe_append_kv4(*(args[n] for n in APPEND), ref(desc), ref(paged))


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), -5), (dict(D=96), -4), (dict(D=0), -4), (dict(B=-1), -2), (dict(Hq=-1), -2), (dict(Hkv=0), -2),
    (dict(C_max=0), -2), (dict(S_max=0), -2), (dict(B=1 << 20, C_max=8), -2), (dict(Hq=1 << 21), -2),
    (dict(Hkv=1 << 21), -2), (dict(q_stride=4095), -2), (dict(q_stride=4100), -2), (dict(k_stride=1000), -2),
    (dict(v_stride=-1024), -2), (dict(v_stride=1 << 28), -2), (dict(rot_dim=144), -16), (dict(rot_dim=-16), -16),
    (dict(rot_dim=24), -16), (dict(rope_style=2), -16), (dict(norm_eps=-1.0), -16), (dict(norm_eps=float("nan")), -16),
])
def test_append_refuses_bad_descriptors(lib, kw, code):
    assert append(lib, append_desc(**kw)) == code
    assert append(lib, append_desc(**dict(dict(B=0), **kw)), q=None) == code or kw.get("B")


def test_append_refuses_bad_pointers_and_pages(lib):
    d = append_desc()
    assert append(lib, None) == -1
    for n in ("q", "k", "v", "inv_freq", "ctx_lens", "chunk_lens", "q_out", "cache"):
        assert append(lib, d, **{n: None}) == -1, n
    for n in MEMBERS:
        assert append(lib, d, cache=kv4(**{n: None})) == -1, n
        assert append(lib, d, cache=kv4(**{n: FAKE + 8})) == -9, n
    for n in ("q", "k", "v", "q_weight", "k_weight", "q_out"):
        assert append(lib, d, **{n: FAKE + 8}) == -9, n
    assert append(lib, d, inv_freq=FAKE + 4) == -9
    assert append(lib, d, draft_mask=FAKE + 4) == -9
    assert append(lib, append_desc(C_max=65), draft_mask=FAKE) == -13
    assert append(lib, append_desc(B=0), q=None, k=None, cache=None) == 0
    for bad in ((4, 64, 9), (24, 8, 9), (16, 15, 9), (16, 16, 0), (1 << 17, 1, 9), (16, 0, 9)):
        assert append(lib, d, bd.PagedKV(*bad)) == -14
    assert append(lib, d, bd.PagedKV(16, 16, 9), block_table=None) == -1
    assert append(lib, d, block_table=FAKE) == -1          # a table without its geometry


ATTN = ["q", "cache", "table", "ctx", "chunk", "mask", "scale", "out", "lse"]


def attn(lib, desc, paged=None, **kw):
    args = dict.fromkeys(ATTN, FAKE)
    args.update(cache=kv4(), mask=None, table=None if paged is None else FAKE, scale=0.088)
    args.update(kw)
    args["cache"] = ref(args["cache"])
    return lib.specmoe_verify_attn_kv4(*(args[n] for n in ATTN), None, ref(desc), ref(paged))


def attn_desc(**kw):
    d = bd.make_desc(**dict(dict(B=2, Hq=32, Hkv=8, D=128, C_max=5, S_max=2304, dtype=1), **kw))
    d.workspace, d.workspace_bytes = FAKE, 1 << 30
    return d


def test_attn_refusals(lib):
    assert attn(lib, None) == -1
    for kw, code in ((dict(dtype=7), -5), (dict(D=96), -4), (dict(B=-1), -2), (dict(Hq=30), -3), (dict(C_max=33), -6),
                     (dict(S_max=3), -2), (dict(S_max=1 << 24), -2), (dict(grid_blocks=4000), -7),
                     (dict(grid_blocks=-1), -7), (dict(flags=1), -12), (dict(flags=2), -12)):
        assert attn(lib, attn_desc(**kw)) == code, kw
    for n in ("q", "cache", "ctx", "chunk", "out", "lse"):
        assert attn(lib, attn_desc(), **{n: None}) == -1, n
    for n in MEMBERS:
        assert attn(lib, attn_desc(), cache=kv4(**{n: None})) == -1, n
        assert attn(lib, attn_desc(), cache=kv4(**{n: FAKE + 8})) == -9, n
    for n in ("q", "out"):
        assert attn(lib, attn_desc(), **{n: FAKE + 8}) == -9, n
    assert attn(lib, attn_desc(), mask=FAKE + 4) == -9
    assert attn(lib, attn_desc(Hq=8, C_max=65), mask=FAKE) == -13
    for scale in (-1.0, 0.0, float("nan"), float("inf")):
        assert attn(lib, attn_desc(), scale=scale) == -10
    assert attn(lib, attn_desc(), table=FAKE) == -1
    assert attn(lib, attn_desc(), bd.PagedKV(16, 144, 9), table=None) == -1
    assert attn(lib, attn_desc(), bd.PagedKV(16, 143, 9)) == -14
    d = attn_desc()
    d.workspace = None
    assert attn(lib, d) == -1
    d.workspace = FAKE + 8
    assert attn(lib, d) == -9
    d.workspace, d.workspace_bytes = FAKE, lib.specmoe_verify_attn_kv4_workspace_bytes(ref(d)) - 1
    assert attn(lib, d) == -8
    assert attn(lib, attn_desc(B=0), q=None, cache=None, out=None) == 0


def test_attn_workspace_holds_that_of_the_other_calls(lib):
    for kw in ({}, dict(C_max=32), dict(dtype=0, D=64), dict(grid_blocks=7), dict(Hkv=4, Hq=28)):
        d = attn_desc(**kw)
        assert lib.specmoe_verify_attn_kv4_workspace_bytes(ref(d)) >= lib.specmoe_verify_attn_workspace_bytes(ref(d)) > 0
    assert lib.specmoe_verify_attn_kv4_workspace_bytes(ref(attn_desc(D=96))) == 0


def rows_desc(**kw):
    return bd.KV4Desc(**dict(dict(B=2, Hkv=8, D=128, N_max=64, S_max=256, dtype=1), **kw))


def read(lib, desc, paged=None, cache=kv4(), table=False, **kw):
    a = dict(dict(first=FAKE, rows=FAKE, k=FAKE, v=FAKE), **kw)
    table = (None if paged is None else FAKE) if table is False else table
    return lib.specmoe_read_kv4(ref(cache), table, a["first"], a["rows"], a["k"], a["v"], None, ref(desc), ref(paged))


def move(lib, desc, paged=None, cache=kv4(), table=False, **kw):
    a = dict(dict(ctx=FAKE, path=FAKE), **kw)
    table = (None if paged is None else FAKE) if table is False else table
    return lib.specmoe_compact_accepted_kv4(ref(cache), table, a["ctx"], a["path"], None, ref(desc), ref(paged))


def test_read_and_move_refusals(lib):
    for call, pointers, wide in ((read, ("first", "rows", "k", "v"), ("k", "v")), (move, ("ctx", "path"), ())):
        assert call(lib, None) == -1
        for kw, code in ((dict(D=96), -4), (dict(B=-1), -2), (dict(Hkv=0), -2), (dict(Hkv=1 << 21), -2),
                         (dict(S_max=0), -2)):
            assert call(lib, rows_desc(**kw)) == code, kw
        for n in pointers:
            assert call(lib, rows_desc(), **{n: None}) == -1, n
        for n in wide:
            assert call(lib, rows_desc(), **{n: FAKE + 8}) == -9, n
        assert call(lib, rows_desc(), cache=None) == -1
        for n in MEMBERS:
            assert call(lib, rows_desc(), cache=kv4(**{n: None})) == -1, n
            assert call(lib, rows_desc(), cache=kv4(**{n: FAKE + 4})) == -9, n
        assert call(lib, rows_desc(), bd.PagedKV(16, 15, 9)) == -14
        assert call(lib, rows_desc(), bd.PagedKV(16, 16, 9), table=None) == -1
        assert call(lib, rows_desc(), table=FAKE) == -1
        assert call(lib, rows_desc(B=0), cache=None, **dict.fromkeys(pointers)) == 0
    for kw, code in ((dict(dtype=3), -5), (dict(N_max=0), -2), (dict(B=1 << 16, N_max=1 << 15), -2),
                     (dict(B=(1 << 24) - 1, N_max=1), -2)):
        assert read(lib, rows_desc(**kw)) == code, kw
    assert move(lib, rows_desc(dtype=3, N_max=0, B=0)) == 0
    assert move(lib, rows_desc(B=1 << 20)) == -2
    assert move(lib, rows_desc(), path=FAKE + 4) == -9


PAGES = ["ctx", "chunk", "table", "held", "free", "count", "missing", "slots"]


def pages(lib, desc, **kw):
    args = dict(dict.fromkeys(PAGES, FAKE), **kw)
    return lib.specmoe_assign_pages(*(args[n] for n in PAGES), None, ref(desc))


def test_pages_refusals(lib):
    def desc(**kw):
        return bd.PagesDesc(**dict(dict(B=4, C_max=5, page_size=16, pages_per_seq=10, num_pages=50), **kw))
    assert pages(lib, None) == -1
    for kw, code in ((dict(B=-1), -2), (dict(B=65536), -2), (dict(C_max=0), -2), (dict(B=65535, C_max=1 << 16), -2),
                     (dict(page_size=4), -14), (dict(page_size=24), -14), (dict(page_size=1 << 17), -14),
                     (dict(pages_per_seq=0), -14), (dict(num_pages=0), -14), (dict(pages_per_seq=1 << 27), -14),
                     (dict(B=65535, pages_per_seq=1 << 16), -14)):
        assert pages(lib, desc(**kw)) == code, kw
    for n in ("ctx", "chunk", "table", "held", "free", "count"):
        assert pages(lib, desc(), **{n: None}) == -1, n
    for n in ("ctx", "chunk", "table", "held", "free", "count", "missing"):
        assert pages(lib, desc(), **{n: FAKE + 2}) == -9, n
    assert pages(lib, desc(), slots=FAKE + 4) == -9
    assert pages(lib, desc(B=0), ctx=None, table=None) == 0
    assert pages(lib, desc(B=0, C_max=0)) == -2


def test_binding_refuses_host_tensors_and_wrong_shapes():
    k = torch.zeros((1, 2, 2, 64))
    lens = torch.zeros((1,), dtype=torch.int32)
    cache = pkg.alloc_kv4_cache(1, 2, 8, 64, "cpu")
    assert [tuple(x.shape) for x in cache] == [(1, 2, 8, 32), (1, 2, 8, 2)] * 2
    for call in (lambda: pkg.append_kv4(None, k, k, cache, lens, lens), lambda: pkg.read_kv4(cache, lens, lens, 4),
                 lambda: pkg.compact_accepted_kv4(cache, lens, lens.long()),
                 lambda: pkg.verify_attn_kv4(k, cache, lens, lens, 1.0),
                 lambda: pkg.assign_pages(lens, lens, pkg.alloc_page_state(1, 2, 3, "cpu"), 16)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="rope"):
        pkg.append_kv4(None, k, k, cache, lens, lens, rope="thirds")
    with pytest.raises(ValueError, match="four dimensions"):
        pkg.append_kv4(None, k[0], k, cache, lens, lens)
    with pytest.raises(ValueError, match="C_max, Hq, D"):
        pkg.verify_attn_kv4(k[0], cache, lens, lens, 1.0)
