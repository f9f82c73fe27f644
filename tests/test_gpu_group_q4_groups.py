"""Every kernel of the 4-bit group products in groups of 32, 64 and 128 (how windows of scales, steps and pieces follow one another depends on them), bit for bit, both products of a gated pair and
both terms of its gradient among them; and the streamed kernels as is documented of them: nothing is rounded before the result."""
import numpy as np
import pytest
import torch

from oracle import group_q4 as O
from paper_2410_09615_amd import binding as B
from tests.test_gpu_group_q4 import DEV
from tests.test_gpu_group_q4_plans import PLANS, _planned

pytestmark = pytest.mark.gpu
TILES = [p for p in PLANS if p[4] != "stream"]
STREAMS = [p for p in PLANS if p[4] == "stream"]


def _whole(n, k, group, zeros, seed):
    """A layer with scales of 2^-6 to 2^-4 and whole c - z, and its values: 7 bits each, multiples of 2^-6."""
    g = np.random.default_rng(seed)
    codes, shape = g.integers(0, 16, (n, k), dtype=np.uint8), (n, O.groups(k, group))
    scales = (2.0 ** g.integers(-6, -3, shape)).astype(np.float16)
    points = g.integers(0, 16, shape, dtype=np.uint8) if zeros else None
    layer = B.SlimGroupQ4Weight(n, k, group, B.slim_group_q4_tile(torch.from_numpy(codes).to(DEV)), torch.from_numpy(scales).to(DEV),
                                None if points is None else torch.from_numpy(points).to(DEV))
    return layer, O.values(codes, scales, points, group)


def _signs(m, k, dtype, seed):
    x = np.random.default_rng(seed).integers(-1, 2, (m, k)).astype(np.float64)
    return x, torch.from_numpy(x).to(dtype).to(DEV)


def _same(got, want, dtype):
    """(the exact sums are multiples of 2^-6 below 2^18 in magnitude: exact in 32 bits, and so are all sums on the way)"""
    assert np.abs(want).max() < 2 ** 17
    assert torch.equal(got.cpu(), torch.from_numpy(want).float().to(dtype))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("plan", PLANS, ids=lambda p: "-".join(map(str, p)))
def test_to_the_bit(plan, dtype, group):
    """Inputs of -1, 0 and 1.  Of the two-layer gradient G is 32, where sigma is 1 in binary32: dG = dH U and dU = 32 dH, which have few bits too."""
    call, m, n, k = plan[:4]
    _planned(*plan)
    (one, Va), (two, Vb) = _whole(n, k, group, True, m + n), _whole(n, k, group, False, m + k)
    x, X = _signs(m, k if call in ("gemm", "gated") else n, dtype, m)
    if call == "gemm":
        _same(B.slim_group_q4_gemm(one, X), x @ Va.T, dtype)
    elif call == "gemm_t":
        _same(B.slim_group_q4_gemm_t(one, X), x @ Va, dtype)
    elif call == "gated":
        _, G, U = B.slim_group_q4_gated(one, two, X, G=True, U=True)
        _same(G, x @ Va.T, dtype)
        _same(U, x @ Vb.T, dtype)
    else:
        u, U = _signs(m, n, dtype, m + 1)
        dX, dG, dU = B.slim_group_q4_gated_backward(one, two, X, torch.full_like(X, 32.0), U)
        _same(dG, x * u, dtype)
        _same(dU, 32 * x, dtype)
        _same(dX, (x * u) @ Va + (32 * x) @ Vb, dtype)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("plan", STREAMS, ids=lambda p: "-".join(map(str, p)))
def test_streamed_weights_are_not_rounded(plan, dtype, group):
    """Scales of 11 bits, whose weights have up to 15 and fit neither type, and one input of -1 or 1 in sixteen: sums are multiples of 2^-16 below 2^8, exact in binary32, and the result is the exact
    one rounded once.  With weights rounded to the type it would be another."""
    call, m, n, k = plan[:4]
    _planned(*plan)
    g = np.random.default_rng(m + n + k)
    x, _ = _signs(m, k, dtype, m)
    x *= (np.arange(k) % 16 == 3)[None, :]
    X = torch.from_numpy(x).to(dtype).to(DEV)
    layers = []
    for zeros in (True, False):
        codes, shape = g.integers(0, 16, (n, k), dtype=np.uint8), (n, O.groups(k, group))
        scales = (g.integers(1024, 2048, shape) * 2.0 ** -16).astype(np.float16)
        points = g.integers(0, 16, shape, dtype=np.uint8) if zeros else None
        layers.append((B.SlimGroupQ4Weight(n, k, group, B.slim_group_q4_tile(torch.from_numpy(codes).to(DEV)), torch.from_numpy(scales).to(DEV),
                                           None if points is None else torch.from_numpy(points).to(DEV)), O.values(codes, scales, points, group)))
    results = [B.slim_group_q4_gemm(layers[0][0], X)] if call == "gemm" else B.slim_group_q4_gated(layers[0][0], layers[1][0], X, G=True, U=True)[1:]
    for got, (_, V) in zip(results, layers):
        ref, mag = O.gemm(x, V)
        assert mag.max() < 2 ** 8
        want = torch.from_numpy(ref).float().to(dtype)
        assert torch.equal(got.cpu(), want)
        rounded = x @ torch.from_numpy(V).to(dtype).double().numpy().T
        assert not torch.equal(torch.from_numpy(rounded).float().to(dtype), want)
