"""The operators on 4-bit weights with group scales at the ends of what their types hold: tokens, scales and activations so large or so small that a step on the way could leave the range.

Bounds as in test_gpu_group_q4.py.
"""
import numpy as np
import pytest
import torch

from oracle import group_q4 as O
from paper_2410_09615_amd import binding as B
from tests.test_gpu_group_q4 import DEV, _check, _matrix, _np, _sum_bound, _weights

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


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", [(5, 70, 130), (200, 200, 130), (200, 300, 515), (513, 1100, 300), (130, 2050, 8201)])
def test_inputs_that_do_not_exist_have_no_part(m, n, k, group):
    """Weights near fp16's largest and rows that end inside a block: a code of 0 past their end would stand for -8 scales (symmetric) or as many as the zero point, beyond fp16, and is no
    weight."""
    W = (torch.rand(n, k, generator=torch.Generator().manual_seed(1)) * 2 - 1) * 60000
    W[:, ::17] = 60000
    codes = np.random.default_rng(2).integers(10, 16, (n, k), dtype=np.uint8)
    scales = np.full((n, O.groups(k, group)), 5000, np.float16)
    fifteen = B.SlimGroupQ4Weight(n, k, group, B.slim_group_q4_tile(torch.from_numpy(codes).to(DEV)), torch.from_numpy(scales).to(DEV),
                                  torch.full(scales.shape, 15, dtype=torch.uint8, device=DEV))
    X = _matrix(m, k, F16, 3, 2.0 ** -12)
    x = _np(X)
    for layer, V in ((B.slim_group_q4_weight(W.to(F16).to(DEV), group), None), (fifteen, O.values(codes, scales, np.full(scales.shape, 15, np.uint8), group))):
        V = _np(B.slim_group_q4_values(layer, torch.float32)) if V is None else V
        assert np.abs(V).max() <= 65504
        ref, mag = O.gemm(x, V)
        _check(B.slim_group_q4_gemm(layer, X), ref, _sum_bound(mag, k, x, F16), F16)
        _, G, U = B.slim_group_q4_gated(layer, layer, X, G=True, U=True)
        _check(G, ref, _sum_bound(mag, k, x, F16), F16)
        assert torch.equal(G, U)
