"""The layer that examples/quantized_experts.py wires from the calls on 4-bit weights, against 64 bits."""
import os
import sys

import pytest
import torch

from paper_2503_09716_amd import Moe
from test_gpu_mx import held

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("T,k,shared", [(300, 3, 2), (40, 4, 1), (17, 1, 0)])
def test_the_long_batch(T, k, shared):
    """Against the definition on x and h as MXFP4 holds them.  Apart from the order of sums the two differ where the kernels' h rounds to another bf16: sums of 320 products
    are off by some 2^-20, a bf16 is 2^-8 wide, so that is one value in 2^11.  Of those one in 2^5 at most passes a border between two values of MXFP4, or its block one
    between two scales, and changes by half of itself at most: 2^-11 2^-5 / 4 = 2^-18 of the square of h, and so of the output's, 2^-9 of the output.  With the
    output's own rounding, 2^-9 at most: 2^-8, and the bound is twice that.  A wrong matrix, expert, row or weight is a difference of the size of the output."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    from quantized_experts import QuantizedLayer
    H, F, E = 320, 192, 12
    gen = torch.Generator().manual_seed(T)

    def normal(shape, std):
        return (torch.randn(shape, generator=gen) * std).bfloat16().to(DEV)
    moe = Moe(0)
    w = [[normal(s, 0.06) for _ in range(E + shared)] for s in ((H, F), (H, F), (F, H))]
    wg, x = normal((H, E), 0.1), normal((T, H), 1.0)
    layer = QuantizedLayer(moe, wg, *w, k, shared)
    out = layer.long_batch(x)
    logits = x.double() @ wg.double()
    top, idx = logits.topk(k + 1, dim=1)
    assert (top[:, k - 1] - top[:, k] > 1e-5).all(), "a near tie: take another seed"
    weight = torch.softmax(top[:, :k], dim=1)      # renormalised
    xv, want = held(x).to(DEV), torch.zeros((T, H), dtype=torch.float64, device=DEV)
    for e in range(E + shared):
        v1, v3, v2 = (held(ws[e].t()).t().to(DEV) for ws in w)
        y = held((torch.nn.functional.silu(xv @ v1) * (xv @ v3)).bfloat16()).to(DEV) @ v2
        want += y * ((idx[:, :k] == e) * weight).sum(dim=1)[:, None] if e < E else y
    moe.close()
    assert ((out.double() - want).square().mean() / want.square().mean()).sqrt().item() < 2.0 ** -7
