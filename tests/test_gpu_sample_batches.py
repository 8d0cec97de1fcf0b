"""Rows of large batches, which share their CU with another row and are drawn by
half as many threads, give what they give alone."""
import pytest
import torch

import paper_2508_21706_amd as pkg
from test_gpu_parity import dev, note

pytestmark = pytest.mark.gpu

# One token of logit 12 and n of another, and a u at which the mass passed lies
# next to a token's end: temperature, the other's bf16 bits, 2^24 u, n.  (One
# unit of 2^-42 more in the weight of the n moves the place of the token drawn.)
BORDERS = [(0.699999988, 0x4121, 5875205, 18194), (0.699999988, 0x4121, 8732259, 9429),
           (0.703700006, 0x4120, 11056677, 9840), (0.703700006, 0x4133, 1218151, 9282),
           (0.707399964, 0x413b, 12914719, 28245), (0.711099982, 0x4128, 652191, 12320),
           (0.711099982, 0x4128, 10296431, 14173), (0.733299971, 0x4129, 8465595, 2728),
           (0.736999989, 0x4139, 5346779, 21181), (0.762899995, 0x4139, 9927615, 30875),
           (0.818399966, 0x4122, 6323159, 746), (0.851700008, 0x4122, 8838141, 6299)]


@pytest.mark.parametrize("T,bits,u24,n", BORDERS)
def test_draws_next_to_a_border_do_not_depend_on_the_batch(T, bits, u24, n):
    d, N = dev(), 300
    row = torch.full((n + 1,), bits, dtype=torch.int16).view(torch.bfloat16)
    row[0] = 12.0
    logits = row.to(d).repeat(N, 1)
    u = torch.full((N,), u24 / 2.0 ** 24, device=d)
    t = torch.full((N,), T, device=d)
    token, logp = pkg.sample(logits, u, temperature=t)
    alone, alone_p = pkg.sample(logits[:1], u[:1], temperature=t[:1])
    torch.cuda.synchronize()
    note(f"[border {T} {bits:#x}] {int(alone)} alone, {int(token[0])} in a batch of {N}")
    assert (token == alone).all() and (logp == alone_p).all()
