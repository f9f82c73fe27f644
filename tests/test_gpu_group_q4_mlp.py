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


def test_calls_in_an_autograd_function():
    """What the calls' documentation says: no graph of their own, and the gradient as a Function's backward; against autograd on the values, whose product is in 32 bits."""
    n, k, m = 300, 256, 20
    layer = B.compress_group_q4((torch.randn(n, k, generator=torch.Generator().manual_seed(1)) * 0.03).to(DEV), 64)

    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, X):
            return B.slim_group_q4_gemm(layer, X)

        @staticmethod
        def backward(ctx, dY):
            return B.slim_group_q4_gemm_t(layer, dY.contiguous())

    X, dY = _matrix(m, k, F16, 1).clone().requires_grad_(), _matrix(m, n, F16, 2, 0.1)
    assert not B.slim_group_q4_gemm(layer, X).requires_grad
    Linear.apply(X).backward(dY)
    assert torch.equal(X.grad, B.slim_group_q4_gemm_t(layer, dY))
    V = B.slim_group_q4_values(layer, torch.float32)
    Z = X.detach().float().requires_grad_()
    (Z @ V.t()).backward(dY.float())
    mag = dY.float().abs() @ V.abs()                                  # weights rounded by half a step, sums in 32 bits on both sides, the result rounded once
    bound = (2.0 ** -11 + 2 * (n + 24) * 2.0 ** -24) * mag + 2.0 ** -25 * dY.float().abs().sum(1, keepdim=True)
    assert bool(((X.grad.float() - Z.grad).abs() <= bound + 2.0 ** -11 * (Z.grad.abs() + bound) + 2.0 ** -25).all())
