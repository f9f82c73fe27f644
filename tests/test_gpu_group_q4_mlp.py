"""The feed-forward block on 4-bit group weights (mlp.GroupMlp) as a training program calls it."""
import pytest
import torch

from paper_2410_09615_amd import binding as B
from paper_2410_09615_amd.mlp import GroupMlp
from tests.test_gpu_group_q4 import DEV, _matrix

pytestmark = pytest.mark.gpu
F16 = torch.float16


def test_a_second_backward_on_what_was_kept():
    k, f, m = 256, 300, 20
    g = torch.Generator().manual_seed(m)
    mlp = GroupMlp(*(B.compress_group_q4((torch.randn(*s, generator=g) * 0.03).to(DEV), 64) for s in ((f, k), (f, k), (k, f))), max_tokens=m)
    X, dY = _matrix(m, k, F16, 1), _matrix(m, k, F16, 2, 0.1)
    _, saved = mlp.forward(X, keep=True)
    first = [t.clone() for t in mlp.backward(dY, saved)]
    for a, b in zip(first, mlp.backward(dY, saved)):
        assert torch.equal(a, b)
