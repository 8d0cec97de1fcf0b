"""A workspace that the kernels cannot write is refused before any launch."""
import pytest
import torch

import paper_2508_21706_amd as pkg
from paper_2508_21706_amd import binding as bd


class Elsewhere:
    """Stands in for a tensor on GPU ``gpu``; nothing but its place is asked for."""

    def __init__(self, gpu, contiguous=True):
        self.gpu, self.contiguous, self.device, self.nbytes = gpu, contiguous, f"cuda:{gpu}", 64

    def get_device(self):
        return self.gpu

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 256


def test_memory_of_the_host_or_another_gpu():
    for make in (bd.Desc, bd.AcceptDesc):
        desc = make()
        with pytest.raises(ValueError, match="workspace is on cpu, expected cuda:0"):
            bd._use_workspace(desc, torch.zeros(1 << 10, dtype=torch.uint8), 0)
        with pytest.raises(ValueError, match="workspace is on cuda:1, expected cuda:0"):
            bd._use_workspace(desc, Elsewhere(1), 0)
        with pytest.raises(ValueError, match="contiguous"):
            bd._use_workspace(desc, Elsewhere(0, contiguous=False), 0)
        assert desc.workspace is None and desc.workspace_bytes == 0
        bd._use_workspace(desc, Elsewhere(0), 0)
        assert desc.workspace == 256 and desc.workspace_bytes == 64
    with pytest.raises(ValueError, match="workspace is on cpu"):
        pkg.workspace_status(torch.zeros(1 << 10, dtype=torch.uint8))


@pytest.mark.gpu
def test_every_call_with_a_workspace_refuses_host_memory():
    from test_gpu_devices import inputs

    x = inputs()
    host = torch.zeros(1 << 20, dtype=torch.uint8)
    head = (x["q"], x["k"], x["v"], x["ctx"], x["chunk"])
    chain = (x["logits"], x["tokens"], x["ctx"], x["chunk"])
    tree = (x["logits"], x["tokens"], x["mask"], x["ctx"], x["chunk"])
    for call in (lambda **kw: pkg.verify_attn(*head, 0.125, **kw),
                 lambda **kw: pkg.verify_attn_tree(*head, x["mask"], 0.125, **kw),
                 lambda **kw: pkg.verify_attn_paged(x["q"], x["pages"], x["pages"], x["table"], x["ctx"], x["chunk"],
                                                    0.125, **kw),
                 lambda **kw: pkg.verify_attn_scored(*head, 0.125, softcap=5.0, **kw),
                 lambda **kw: pkg.accept_greedy(*chain, **kw),
                 lambda **kw: pkg.accept_greedy_tree(*tree, **kw),
                 lambda **kw: pkg.accept_sample(*chain, x["u"], **kw),
                 lambda **kw: pkg.accept_sample_tree(*tree, x["u"], **kw)):
        with pytest.raises(ValueError, match="workspace is on cpu"):
            call(workspace=host)
