"""The operators on 4-bit weights with group scales against their definition in 64 bits.

Bounds, for a sum of `len` terms of magnitudes adding up to mag, h half a step of the type (2^-11 fp16, 2^-8 bf16), u = 2^-24:
  sum       (len + 24) u mag: every addition in binary32, whatever their order, and the few multiplications by scales;
  values    h mag where weights are rounded to the inputs' type before they are multiplied (and 2^-25 per weight where fp16 has no smaller step);
  result    h (|exact| + the above), one rounding (2^-25 where fp16 has no smaller step).
silu and its gradient: exp's argument -g log2(e) is rounded (|g| u relative to the result), and there are at most eight more operations of error u: (2 |g| + 16) u.
"""
import numpy as np
import pytest
import torch

from oracle import group_q4 as O
from paper_2410_09615_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U24 = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}


def _np(t):
    return t.detach().double().cpu().numpy()


def _weights(n, k, group, zeros, seed, spread=0.02):
    """(layer, its exact values): codes of every value, scales over a factor of 8."""
    g = np.random.default_rng(seed)
    codes = g.integers(0, 16, (n, k), dtype=np.uint8)
    scales = (spread * 2.0 ** g.uniform(-3, 0, (n, O.groups(k, group)))).astype(np.float16)
    points = g.integers(0, 16, scales.shape, dtype=np.uint8) if zeros else None
    layer = B.SlimGroupQ4Weight(n, k, group, B.slim_group_q4_tile(torch.from_numpy(codes).to(DEV)), torch.from_numpy(scales).to(DEV),
                                None if points is None else torch.from_numpy(points).to(DEV))
    return layer, O.values(codes, scales, points, group)


def _matrix(m, k, dtype, seed, scale=1.0, gap=0, offset=0):
    """[m][k] of a larger buffer: rows `gap` elements apart, the first `offset` elements from an aligned address."""
    g = torch.Generator()
    g.manual_seed(seed)
    whole = torch.full((m * (k + gap) + offset,), float("nan"), dtype=dtype, device=DEV)
    t = whole[offset:].view(m, k + gap)[:, :k]
    t.copy_((torch.randn(m, k, generator=g) * scale).to(dtype))
    return t


def _sum_bound(mag, length, inputs, dtype):
    """Of a product whose weights are rounded to the type (which the precise kernels' are not)."""
    return (length + 24) * U24 * mag + HALF[dtype] * mag + TINY[dtype] * np.abs(inputs).sum(axis=1, keepdims=True)


def _check(got, ref, bound, dtype):
    got = _np(got)
    assert np.isfinite(got).all()
    err = np.abs(got - ref) - (bound + HALF[dtype] * (np.abs(ref) + bound) + TINY[dtype])
    assert err.max() <= 0, (np.unravel_index(err.argmax(), err.shape), err.max())


SIZES = [(1, 1, 1), (1, 16, 128), (1, 4096, 4096), (2, 17, 129), (5, 300, 1000), (16, 512, 2048), (16, 1000, 4100), (17, 333, 515), (33, 130, 640), (48, 700, 1152),
         (64, 256, 256), (65, 129, 1000), (77, 1003, 515), (130, 300, 1100), (257, 515, 333), (300, 1000, 640), (513, 260, 4100)]


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (128, False)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_gemm(m, n, k, dtype, group, zeros):
    layer, V = _weights(n, k, group, zeros, n + k)
    X = _matrix(m, k, dtype, m)
    x = _np(X)
    ref, mag = O.gemm(x, V)
    _check(B.slim_group_q4_gemm(layer, X), ref, _sum_bound(mag, k, x, dtype), dtype)


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_gemm_t(m, n, k, dtype, group, zeros):
    layer, V = _weights(n, k, group, zeros, n + k + 1)
    dY = _matrix(m, n, dtype, m)
    y = _np(dY)
    ref, mag = O.gemm(y, V.T)
    _check(B.slim_group_q4_gemm_t(layer, dY), ref, _sum_bound(mag, n, y, dtype), dtype)


def _check_gated(H, G, U, x, Vg, Vu, k, dtype):
    g, gm = O.gemm(x, Vg)
    u, um = O.gemm(x, Vu)
    bg, bu = _sum_bound(gm, k, x, dtype), _sum_bound(um, k, x, dtype)
    if G is not None:
        _check(G, g, bg, dtype)
    if U is not None:
        _check(U, u, bu, dtype)
    h = O.gated(g, u)
    silu = np.abs(g * O.sigma(g))
    bound = 1.1 * bg * (np.abs(u) + bu) + silu * bu                   # |silu'| <= 1.1
    bound = bound + (2 * (np.abs(g) + bg) + 16) * U24 * (np.abs(h) + bound)
    _check(H, h, bound, dtype)


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_gated(m, n, k, keep, dtype, group, zeros):
    (gate, Vg), (up, Vu) = _weights(n, k, group, zeros, n + k, 0.004), _weights(n, k, group, not zeros, n + k + 7, 0.004)
    X = _matrix(m, k, dtype, m)
    H, G, U = B.slim_group_q4_gated(gate, up, X, G=True if keep else None, U=True if keep else None)
    assert (G is None) == (not keep) and (U is None) == (not keep)
    _check_gated(H, G, U, _np(X), Vg, Vu, k, dtype)


def _check_backward(dX, dG, dU, dH, G, U, Vg, Vu, dtype):
    h, g, u = _np(dH), _np(G), _np(U)
    rg, ru = O.gated_backward(h, g, u)
    rel = (2 * np.abs(g) + 16) * U24
    _check(dG, rg, np.abs(h * u) * O.sigma(g) * (1 + np.abs(g)) * rel, dtype)
    _check(dU, ru, np.abs(ru) * rel, dtype)
    g, u = _np(dG), _np(dU)                                           # dX is the product of the rounded ones
    (a, am), (b, bm) = O.gemm(g, Vg.T), O.gemm(u, Vu.T)
    _check(dX, a + b, _sum_bound(am + bm, 2 * Vg.shape[0], np.concatenate([g, u], axis=1), dtype), dtype)


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_gated_backward(m, n, k, dtype, group, zeros):
    (gate, Vg), (up, Vu) = _weights(n, k, group, zeros, n + k), _weights(n, k, group, not zeros, n + k + 7)
    dH, G, U = (_matrix(m, n, dtype, m + i, 2.0) for i in range(3))
    dX, dG, dU = B.slim_group_q4_gated_backward(gate, up, dH, G, U)
    _check_backward(dX, dG, dU, dH, G, U, Vg, Vu, dtype)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,k", [(1, 1), (16, 128), (17, 129), (100, 1000), (333, 4100), (5, 31)])
def test_weight(n, k, dtype, group, zeros):
    """Codes, scales and zero points bit for bit, in a matrix with gaps that starts anywhere; what they stand for, read back in every type."""
    W = _matrix(n, k, dtype, n + k, 0.02, gap=3, offset=1)
    W[0, 0] = 0.5
    if n > 10:
        W[3] = 0
        W[4, :40] = 1e-7 if dtype != torch.float16 else 6e-8
        W[5] = W[5].abs()
        W[6] = -W[6].abs()
    layer = B.slim_group_q4_weight(W, group, zeros)
    codes, scales, points = O.quantize(W.float().cpu().numpy(), group, zeros)
    assert np.array_equal(layer.codes.cpu().numpy(), O.tile(codes))
    assert np.array_equal(layer.scales.cpu().numpy().view(np.uint16), scales.view(np.uint16))
    assert (layer.zeros is None) == (points is None) and (points is None or np.array_equal(layer.zeros.cpu().numpy(), points))
    assert np.array_equal(B.slim_group_q4_untile(layer.codes, n, k).cpu().numpy(), codes)
    assert torch.equal(B.slim_group_q4_tile(torch.from_numpy(codes).to(DEV)), layer.codes)
    V = torch.from_numpy(O.values(codes, scales, points, group)).float().to(DEV)       # (a code, a zero point and a scale: 16 bits, exact in 32)
    for t in (torch.float32, torch.float16, torch.bfloat16):
        assert torch.equal(B.slim_group_q4_values(layer, t), V.to(t))


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan"), 3e38, -3e38])
def test_weight_of_groups_that_have_no_scale(value, zeros):
    W = torch.randn(20, 256, generator=torch.Generator().manual_seed(0)) * 0.02
    W[3, 70] = value
    layer = B.slim_group_q4_weight(W.to(DEV), 64, zeros)
    codes, scales, points = O.quantize(W.numpy(), 64, zeros)
    assert np.array_equal(layer.scales.cpu().numpy().view(np.uint16) & 0x7FFF, scales.view(np.uint16) & 0x7FFF)
    assert np.array_equal(layer.codes.cpu().numpy(), O.tile(codes)) and (not zeros or np.array_equal(layer.zeros.cpu().numpy(), points))
    V = B.slim_group_q4_values(layer, torch.float32)
    assert torch.isnan(V[3, 64:128]).all() == (not np.isfinite(value)) and int(torch.isnan(V).sum()) in (0, 64)
