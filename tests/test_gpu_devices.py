"""Every library call that launches or waits is made with the tensors' GPU current,
also from a program whose current GPU is another one: a stream's handle may be
that of the current GPU's null stream, whichever that is.  (The binding is told
that GPU 1 is current; on a machine with one GPU nothing else changes.)"""
import pytest
import torch

import paper_2508_21706_amd as pkg
from paper_2508_21706_amd import binding as bd
from test_gpu_parity import dev

pytestmark = pytest.mark.gpu

HOST_ONLY = {"specmoe_verify_attn_workspace_bytes", "specmoe_accept_workspace_bytes", "specmoe_verify_attn_key_tile",
             "specmoe_status_str"}


@pytest.fixture
def calls(monkeypatch):
    """The names of the library's functions called, each with GPU 0 current."""
    real, now, made = bd.load_library(), [1], []

    class Device:
        def __init__(self, gpu):
            # (None: the current one, as torch.cuda.synchronize() asks for)
            self.gpu = now[-1] if gpu is None else gpu if isinstance(gpu, int) else torch.device(gpu).index

        def __enter__(self):
            now.append(self.gpu)

        def __exit__(self, *_):
            now.pop()

    class Library:
        def __getattr__(self, name):
            call = getattr(real, name)

            def checked(*args):
                assert name in HOST_ONLY or now[-1] == 0, f"{name} with GPU {now[-1]} current"
                made.append(name)
                return call(*args)
            return checked

    monkeypatch.setattr(bd, "_current_gpu", lambda: now[-1])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(bd, "_lib", Library())
    return made


def inputs():
    d = dev()
    B, C, Hq, Hkv, D, S, V = 2, 3, 4, 2, 64, 32, 64
    z = lambda *shape, dt=torch.bfloat16: torch.zeros(shape, dtype=dt, device=d)   # noqa: E731
    n = lambda *a: torch.tensor(a, dtype=torch.int32, device=d)   # noqa: E731
    mask = torch.tensor([[1, 3, 5]] * B, device=d)
    return dict(q=z(B, C, Hq, D), k=z(B, Hkv, S, D), v=z(B, Hkv, S, D), ctx=n(5, 0), chunk=n(3, 2), mask=mask,
                logits=z(B, C, V), tokens=z(B, C, dt=torch.int32), u=z(B, C, dt=torch.float32), new=z(B, C, Hkv, D),
                pages=z(4, Hkv, 16, D), table=torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device=d))


def test_attention_calls(calls):
    x = inputs()
    head = (x["q"], x["k"], x["v"], x["ctx"], x["chunk"])
    out, lse = pkg.verify_attn(*head, 0.125)
    pkg.verify_attn_noalloc(*head, 0.125, out, lse)
    pkg.verify_attn_tree(*head, x["mask"], 0.125)
    pkg.verify_attn_paged(x["q"], x["pages"], x["pages"], x["table"], x["ctx"], x["chunk"], 0.125)
    pkg.verify_attn_scored(*head, 0.125, softcap=5.0)
    ws = pkg.alloc_scored_workspace(x["q"], x["k"])
    assert pkg.workspace_status(ws) == 0
    torch.cuda.synchronize()
    assert {"specmoe_verify_attn", "specmoe_verify_attn_noalloc", "specmoe_verify_attn_tree", "specmoe_verify_attn_paged",
            "specmoe_verify_attn_scored", "specmoe_verify_attn_workspace_init", "specmoe_verify_attn_status"} <= set(calls)


def test_append_sampling_and_acceptance_calls(calls):
    x = inputs()
    pkg.append_kv(None, x["new"], x["new"], x["k"], x["v"], x["ctx"], x["chunk"])
    pkg.sample(x["logits"][:, 0], x["u"][:, 0].contiguous())
    chain = (x["logits"], x["tokens"], x["ctx"], x["chunk"])
    tree = (x["logits"], x["tokens"], x["mask"], x["ctx"], x["chunk"])
    pkg.accept_sample(*chain, x["u"])
    pkg.accept_sample_tree(*tree, x["u"])
    pkg.accept_greedy(*chain)
    path = pkg.accept_greedy_tree(*tree)["path"]
    pkg.compact_accepted_kv(x["k"], x["v"], x["ctx"], path)
    torch.cuda.synchronize()
    assert {"specmoe_append_kv", "specmoe_sample", "specmoe_accept_sample", "specmoe_accept_sample_tree",
            "specmoe_accept_greedy", "specmoe_accept_greedy_tree", "specmoe_compact_accepted_kv",
            "specmoe_accept_workspace_init"} <= set(calls)
