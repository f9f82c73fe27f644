"""The operators on 4-bit weights with group scales at the ends of what their types hold: tokens, scales and activations so large or so small that a step on the way could leave the range.

Bounds as in test_gpu_group_q4.py.
"""
import pytest
import torch

from oracle import group_q4 as O
from paper_2410_09615_amd import binding as B
from tests.test_gpu_group_q4 import _check, _matrix, _np, _sum_bound, _weights

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("power", [121, -110, -120])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("m", [1, 5, 40, 200])
def test_tokens_near_the_ends_of_bf16(m, group, zeros, power):
    """Tokens of 2^121 and of 2^-120 in bf16: results are in range, and so is everything before the scales.  Products with whole weights that fall below 2^-126 are in steps of 2^-149, of
    which half is lost per term, times the scale's power of two that the whole weights lack (2^15)."""
    n, k = 100, 515
    (gate, Vg), (up, Vu) = _weights(n, k, group, zeros, 1), _weights(n, k, group, zeros, 2)
    X = _matrix(m, k, BF16, 3, 2.0 ** power)
    x = _np(X)
    lost = (k + 24) * 2.0 ** -150 * 2 ** 15 * 0.02
    for got, V in zip((B.slim_group_q4_gemm(gate, X), *B.slim_group_q4_gated(gate, up, X, G=True, U=True)[1:]), (Vg, Vg, Vu)):
        ref, mag = O.gemm(x, V)
        _check(got, ref, _sum_bound(mag, k, x, BF16) + lost, BF16)
