"""The operators on 4-bit weights with group scales at the ends of what their types hold: tokens, scales and activations so large or so small that a step on the way could leave the range.

Bounds as in test_gpu_group_q4.py.
"""
import numpy as np
import pytest
import torch

from oracle import group_q4 as O
from paper_2410_09615_amd import binding as B
from tests.test_gpu_group_q4 import DEV, _check, _check_backward, _check_gated, _matrix, _np, _sum_bound, _weights

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


def _wide(n, k, group, seed, most):
    """Scales of all sizes, each with one of 256 or more among small ones, and zero points of any byte."""
    g = np.random.default_rng(seed)
    codes = g.integers(0, 16, (n, k), dtype=np.uint8)
    shape = (n, O.groups(k, group))
    scales = (2.0 ** g.uniform(-12, np.log2(most), shape)).astype(np.float16)
    scales[::3] = (2.0 ** g.uniform(-12, -6, scales[::3].shape)).astype(np.float16)      # (rows without a large one)
    scales *= np.where(g.random(shape) < 0.3, -1, 1).astype(np.float16)
    points = g.integers(0, 256, shape, dtype=np.uint8)
    layer = B.SlimGroupQ4Weight(n, k, group, B.slim_group_q4_tile(torch.from_numpy(codes).to(DEV)), torch.from_numpy(scales).to(DEV), torch.from_numpy(points).to(DEV))
    return layer, O.values(codes, scales, points, group)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", [(5, 300, 700), (200, 200, 700), (200, 200, 2600), (130, 4099, 1000), (513, 8200, 200), (70, 2050, 4100), (400, 200, 8200), (600, 700, 2600)])
def test_weights_beyond_fp16(m, n, k, group, dtype):
    """(c - z) s to 255 x 2000, far beyond 65504: finite, and within half a step of it, in every kernel."""
    (one, Va), (two, Vb) = _wide(n, k, group, 1, 2000), _wide(n, k, group, 2, 2000)
    assert np.abs(Va).max() > 4e5
    X, dY = _matrix(m, k, dtype, 3, 2.0 ** -19), _matrix(m, n, dtype, 4, 2.0 ** -14)
    x, y = _np(X), _np(dY)
    ref, mag = O.gemm(x, Va)
    _check(B.slim_group_q4_gemm(one, X), ref, _sum_bound(mag, k, x, dtype), dtype)
    _check_gated(*B.slim_group_q4_gated(one, two, X, G=True, U=True), x, Va, Vb, k, dtype)
    ref, mag = O.gemm(y, Va.T)
    _check(B.slim_group_q4_gemm_t(one, dY), ref, _sum_bound(mag, n, y, dtype), dtype)
    G, U = _matrix(m, n, dtype, 5), _matrix(m, n, dtype, 6)
    _check_backward(*B.slim_group_q4_gated_backward(one, two, dY, G, U), dY, G, U, Va, Vb, dtype)


@pytest.mark.parametrize("m", [70, 300])
def test_what_is_not_finite_beside_weights_beyond_fp16(m):
    """An infinite input: rows without large scales have what the definition has, the others are not finite, other tokens' results are as without it.  A scale of NaN: its row's results and its group's
    gradients, no others."""
    n, k = 300, 640
    layer, V = _wide(n, k, 64, 1, 2000)
    X, dY = _matrix(m, k, F16, 2, 2.0 ** -13), _matrix(m, n, F16, 3, 2.0 ** -14)
    y, x = B.slim_group_q4_gemm(layer, X).clone(), B.slim_group_q4_gemm_t(layer, dY).clone()
    bad = X.clone()
    bad[3, 100] = float("inf")
    got, others = B.slim_group_q4_gemm(layer, bad), torch.arange(m, device=DEV) != 3
    assert torch.equal(got[others], y[others]) and not bool(torch.isfinite(got[3]).any())
    small = torch.arange(n) % 3 == 0                                  # (rows of _wide without a large scale)
    want = torch.where(torch.from_numpy(V[:, 100]) > 0, float("inf"), -float("inf"))
    want[torch.from_numpy(V[:, 100]) == 0] = float("nan")
    assert torch.equal(got[3].float().cpu()[small].nan_to_num(nan=7.0), want[small].nan_to_num(nan=7.0))
    bad = dY.clone()
    bad[3, 0] = -float("inf")
    got = B.slim_group_q4_gemm_t(layer, bad)
    assert torch.equal(got[others], x[others]) and not bool(torch.isfinite(got[3]).any())
    layer.scales[n - 1, 4] = float("nan")
    got = B.slim_group_q4_gemm(layer, X)
    assert bool(torch.isnan(got[:, n - 1]).all()) and torch.equal(got[:, :n - 1], y[:, :n - 1])
    got = B.slim_group_q4_gemm_t(layer, dY)
    assert bool(torch.isnan(got[:, 256:320]).all()) and torch.equal(got[:, :256], x[:, :256]) and torch.equal(got[:, 320:], x[:, 320:])
