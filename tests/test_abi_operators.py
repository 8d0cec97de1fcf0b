"""Host-only checks of the entry points around the verification attention:
arguments are refused before any HIP call (so these run without a GPU), and
the binding's structs mirror the headers'."""
import ctypes
import os
import re

import pytest
import torch

import paper_2508_21706_amd as pkg
from paper_2508_21706_amd import binding as bd

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
FAKE = 0x10000          # 16-byte aligned, never dereferenced by these tests


@pytest.fixture(scope="module")
def lib():
    return bd.load_library()


@pytest.mark.parametrize("header,struct,mirror", [
    ("specmoe_append.h", "specmoe_append_desc", bd.AppendDesc),
    ("specmoe_verify.h", "specmoe_score", bd.Score),
    ("specmoe_sample.h", "specmoe_sample_desc", bd.SampleDesc),
    ("specmoe_sample.h", "specmoe_sampling", bd.Sampling),
])
def test_structs_match_the_headers(header, struct, mirror):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, header)).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (struct, struct), text, re.S).group(1)
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}
    fields = [(n, ctypes.c_void_p if star else kinds[t])
              for t, star, n in re.findall(r"(?:const\s+)?(\w+)\s*(\*?)\s*(\w+)\s*;", body)]
    assert fields == list(mirror._fields_)


def append_desc(**kw):
    base = dict(B=2, Hq=32, Hkv=8, D=128, C_max=5, S_max=256, dtype=bd.SPECMOE_BF16, rot_dim=128, rope_style=0,
                norm_eps=1e-6, q_stride=0, k_stride=0, v_stride=0)
    base.update(kw)
    return bd.AppendDesc(**base)


APPEND = ["q", "k", "v", "q_weight", "k_weight", "inv_freq", "ctx_lens", "chunk_lens", "draft_mask", "block_table",
          "q_out", "k_cache", "v_cache", "stream"]


def append(lib, desc, paged=None, **kw):
    args = dict.fromkeys(APPEND, FAKE)
    args.update(draft_mask=None, block_table=None if paged is None else FAKE, stream=None)
    args.update(kw)
    return lib.specmoe_append_kv(*(args[n] for n in APPEND), None if desc is None else ctypes.byref(desc),
                                 None if paged is None else ctypes.byref(paged))


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), -5), (dict(D=96), -4), (dict(D=0), -4), (dict(B=-1), -2), (dict(Hq=-1), -2), (dict(Hkv=0), -2),
    (dict(C_max=0), -2), (dict(S_max=0), -2), (dict(B=1 << 20, C_max=8), -2), (dict(Hq=1 << 21), -2),
    (dict(q_stride=4095), -2), (dict(q_stride=4100), -2), (dict(k_stride=1000), -2), (dict(v_stride=-1024), -2),
    (dict(v_stride=1 << 28), -2), (dict(rot_dim=144), -16), (dict(rot_dim=-16), -16), (dict(rot_dim=24), -16),
    (dict(rope_style=2), -16), (dict(norm_eps=-1.0), -16), (dict(norm_eps=float("nan")), -16),
    (dict(norm_eps=float("inf")), -16),
])
def test_append_refuses_bad_descriptors(lib, kw, code):
    assert append(lib, append_desc(**kw)) == code
    assert append(lib, append_desc(**dict(dict(B=0), **kw)), q=None) == code or kw.get("B")


def test_append_refuses_bad_pointers(lib):
    d = append_desc()
    assert append(lib, None) == -1
    for n in ("q", "k", "v", "inv_freq", "ctx_lens", "chunk_lens", "q_out", "k_cache", "v_cache"):
        assert append(lib, d, **{n: None}) == -1, n
    for n in ("q", "k", "v", "q_weight", "k_weight", "q_out", "k_cache", "v_cache"):
        assert append(lib, d, **{n: FAKE + 8}) == -9, n
    assert append(lib, d, inv_freq=FAKE + 4) == -9
    assert append(lib, d, draft_mask=FAKE + 4) == -9
    assert append(lib, append_desc(C_max=65), draft_mask=FAKE) == -13
    assert append(lib, append_desc(B=0), q=None, k=None, k_cache=None) == 0
    assert append(lib, append_desc(B=0, C_max=65), draft_mask=FAKE) == -13


def test_append_refuses_bad_pages(lib):
    page = lambda *a: bd.PagedKV(*a)   # noqa: E731
    d = append_desc(S_max=256)
    for bad in (page(4, 64, 9), page(24, 8, 9), page(16, 15, 9), page(16, 16, 0), page(1 << 17, 1, 9), page(16, 0, 9)):
        assert append(lib, d, bad) == -14
    assert append(lib, d, page(16, 16, 9), block_table=None) == -1
    assert append(lib, d, block_table=FAKE) == -1          # a table without its geometry


def sample(lib, desc, logits=FAKE, u=FAKE, settings=None, tokens=FAKE, logprobs=FAKE):
    return lib.specmoe_sample(logits, u, settings, tokens, logprobs, None, None if desc is None else ctypes.byref(desc))


def test_sample_refusals(lib):
    D = bd.SampleDesc
    assert sample(lib, None) == -1
    for desc, code in ((D(4, 100, 2, 0, 0), -5), (D(4, 100, 1, 1, 0), -12), (D(-1, 100, 1, 0, 0), -2),
                       (D(1 << 22, 100, 1, 0, 0), -2), (D(4, 0, 1, 0, 0), -2), (D(4, (1 << 20) + 1, 1, 0, 0), -2),
                       (D(4, 100, 1, 0, 99), -2), (D(4, 100, 1, 0, -100), -2), (D(4, 100, 1, 0, 1 << 36), -2)):
        assert sample(lib, desc) == code
    d = D(4, 100, 1, 0, 0)
    for n in ("logits", "u", "tokens"):
        assert sample(lib, d, **{n: None}) == -1, n
    assert sample(lib, d, logits=FAKE + 1) == -9
    assert sample(lib, D(4, 100, 0, 0, 0), logits=FAKE + 2) == -9
    assert sample(lib, D(0, 100, 1, 0, 0), logits=None, u=None, tokens=None) == 0


ACCEPT = ["logits", "tokens", "ctx", "chunk", "u", "settings", "sampled", "logprobs", "accepted", "next", "new_ctx"]


def accept(lib, desc, mask=False, path=FAKE, **kw):
    args = dict.fromkeys(ACCEPT, FAKE)
    args.update(settings=None)
    args.update(kw)
    ref = None if desc is None else ctypes.byref(desc)
    v = [args[n] for n in ACCEPT]
    if mask is False:
        return lib.specmoe_accept_sample(*v, None, ref)
    return lib.specmoe_accept_sample_tree(v[0], v[1], mask, *v[2:], path, None, ref)


def test_accept_sample_refusals(lib):
    def desc(**kw):
        d = bd.AcceptDesc(**dict(dict(B=4, C_max=5, V=32000, dtype=1, split=0, flags=0), **kw))
        d.workspace, d.workspace_bytes = FAKE, 1 << 30
        return d
    for mask in (False, FAKE):
        assert accept(lib, None, mask) == -1
        for kw, code in ((dict(dtype=2), -5), (dict(flags=1), -12), (dict(B=-1), -2), (dict(C_max=0), -2),
                         (dict(V=31999), -2), (dict(V=(1 << 20) + 8), -2), (dict(B=65536, C_max=64, V=8), -2)):
            assert accept(lib, desc(**kw), mask) == code, kw
        for n in set(ACCEPT) - {"settings", "logprobs"}:
            assert accept(lib, desc(), mask, **{n: None}) == -1, n
        assert accept(lib, desc(), mask, logits=FAKE + 8) == -9
        d = desc()
        d.workspace = None
        assert accept(lib, d, mask) == -1
        d.workspace = FAKE + 8
        assert accept(lib, d, mask) == -9
        d.workspace, d.workspace_bytes = FAKE, 100
        assert accept(lib, d, mask) == -8
        assert accept(lib, desc(B=0), mask, logits=None) == 0
    assert accept(lib, desc(C_max=65), FAKE) == -13
    assert accept(lib, desc(), None) == -1
    assert accept(lib, desc(), FAKE, path=None) == -1
    assert accept(lib, desc(), FAKE + 4) == -9
    assert accept(lib, desc(), FAKE, path=FAKE + 4) == -9


SCORED = ["q", "k", "v", "table", "ctx", "chunk", "mask", "scale", "out", "lse"]


def scored(lib, desc, score=bd.Score(30.0, 0, None, None), paged=None, **kw):
    args = dict.fromkeys(SCORED, FAKE)
    args.update(mask=None, table=None if paged is None else FAKE, scale=0.088)
    args.update(kw)
    ref = lambda s: None if s is None else ctypes.byref(s)   # noqa: E731
    return lib.specmoe_verify_attn_scored(*(args[n] for n in SCORED), None, ref(desc), ref(paged), ref(score))


def test_scored_refusals(lib):
    def desc(**kw):
        d = bd.make_desc(**dict(dict(B=2, Hq=32, Hkv=8, D=128, C_max=5, S_max=2304, dtype=1), **kw))
        d.workspace, d.workspace_bytes = FAKE, 1 << 30
        return d
    assert scored(lib, None) == -1
    assert scored(lib, desc(), None) == -1
    for kw, code in ((dict(dtype=7), -5), (dict(D=96), -4), (dict(B=-1), -2), (dict(Hq=30), -3),
                     (dict(C_max=33), -6), (dict(grid_blocks=4000), -7), (dict(flags=2), -12)):
        assert scored(lib, desc(**kw)) == code, kw
    for n in ("q", "k", "v", "ctx", "chunk", "out", "lse"):
        assert scored(lib, desc(), **{n: None}) == -1, n
    for n in ("q", "k", "v", "out"):
        assert scored(lib, desc(), **{n: FAKE + 8}) == -9, n
    assert scored(lib, desc(), mask=FAKE + 4) == -9
    assert scored(lib, desc(Hq=8, C_max=65), mask=FAKE) == -13
    assert scored(lib, desc(), scale=-1.0) == -10
    for cap, window in ((-1.0, 0), (float("nan"), 0), (float("inf"), 0), (1.0, -1)):
        assert scored(lib, desc(), bd.Score(cap, window, None, None)) == -17
        assert scored(lib, desc(B=0), bd.Score(cap, window, None, None)) == -17
    assert scored(lib, desc(), bd.Score(0.0, 0, FAKE + 2, None)) == -9
    assert scored(lib, desc(), bd.Score(0.0, 0, None, FAKE + 1)) == -9
    assert scored(lib, desc(), table=FAKE) == -1
    assert scored(lib, desc(), paged=bd.PagedKV(16, 144, 9), table=None) == -1
    assert scored(lib, desc(), paged=bd.PagedKV(16, 143, 9)) == -14
    d = desc()
    d.workspace_bytes = 64
    assert scored(lib, d) == -8
    assert scored(lib, desc(B=0), q=None, out=None) == 0


def test_scored_refuses_a_cap_too_small_for_its_scale(lib):
    d = bd.make_desc(2, 32, 8, 128, 5, 2304, 1)
    d.workspace, d.workspace_bytes = FAKE, 1 << 30
    assert scored(lib, d, bd.Score(1e-40, 0, None, None), scale=1.0) == -17     # (scale / softcap is infinite)


def test_binding_refuses_host_tensors_and_wrong_shapes():
    k = torch.zeros((1, 2, 2, 64))
    lens = torch.zeros((1,), dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        pkg.append_kv(None, k, k, torch.zeros((1, 2, 8, 64)), torch.zeros((1, 2, 8, 64)), lens, lens)
    with pytest.raises(ValueError, match="rope"):
        pkg.append_kv(None, k, k, k, k, lens, lens, rope="thirds")
    with pytest.raises(ValueError, match="four dimensions"):
        pkg.append_kv(None, k[0], k, k, k, lens, lens)
    with pytest.raises(ValueError, match="GPU"):
        pkg.sample(torch.zeros((2, 8)), torch.zeros((2,)))
    with pytest.raises(ValueError, match=r"\[N, V\]"):
        pkg.sample(torch.zeros((8,)), torch.zeros((2,)))
    with pytest.raises(ValueError, match="GPU"):
        pkg.accept_sample(torch.zeros((1, 2, 8)), torch.zeros((1, 2), dtype=torch.int32), lens, lens, torch.zeros((1, 2)))


def test_binding_refuses_rows_without_memory_of_their_own():
    """(expand() gives such rows a stride of 0, which the descriptors take for
    side-by-side rows)"""
    for B, C, row in ((1, 3, (1, 1, 2, 64)), (2, 1, (1, 1, 2, 64)), (2, 3, (1, 1, 2, 64)), (2, 3, (2, 1, 2, 64)),
                      (2, 3, (1, 3, 2, 64))):
        with pytest.raises(ValueError, match="one distance"):
            bd._token_stride(torch.zeros(row).expand(B, C, 2, 64), "k", (B, C, 2, 64), torch.float32, -1)
    for V in (1, 8):
        with pytest.raises(ValueError, match="memory of its own"):
            pkg.sample(torch.zeros((1, V)).expand(3, V), torch.zeros((3,)))
