"""The activation on more values than its workgroups take at once (8192 x 256 pieces of 8): the rest is walked."""
import numpy as np
import pytest
import torch

from oracle import block_fp8 as O
from paper_2410_09615_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,k", [(1700, 13001), (33000, 1000)])
def test_activation_walks(m, k, dtype):
    """As it is: bit for bit the oracle's.  Gated: each row as in a call of a few rows."""
    assert m * O.blocks(k) * 16 > 8192 * 256
    g = torch.Generator(device=DEV)
    g.manual_seed(m)
    G, V = (torch.randn(m, k, generator=g, device=DEV).mul_(3).to(dtype) for _ in range(2))
    codes, scales = B.slim_block_fp8_act(G, act="none")
    want, top = O.quantize_rows(G.float().cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), (top / O.FMAX).astype(np.float32))
    codes, scales = B.slim_block_fp8_act(G, V)
    for at in range(0, m, 500):
        c, s = B.slim_block_fp8_act(G[at:at + 500], V[at:at + 500])
        assert torch.equal(codes[at:at + 500], c) and torch.equal(scales[at:at + 500], s)
