"""Every kernel of the products with 4-bit group weights, reached by name (slim_group_q4_plan), on sizes that end inside tiles, blocks and groups: within the bounds of
test_gpu_group_q4.py, and bit for bit on numbers whose sums have no error, so that one term lost or taken twice shows."""
import numpy as np
import pytest
import torch

from oracle import group_q4 as O
from paper_2410_09615_amd import binding as B
from tests.test_gpu_group_q4 import DEV, _check, _check_backward, _check_gated, _matrix, _np, _sum_bound, _weights

pytestmark = pytest.mark.gpu

# call, tokens, n, k, the plan: kernel, outputs and tokens of a tile, whether it is shared (by how many wavefronts, where weights are streamed)
PLANS = [("gemm", 1, 64, 515, "stream", 16, 4, 4), ("gemm", 5, 64, 1300, "stream", 16, 16, 8), ("gemm", 17, 64, 64, "stream", 16, 32, 2), ("gemm", 33, 64, 1300, "stream", 16, 48, 8),
         ("gemm", 3, 4099, 1300, "stream", 32, 4, 8), ("gemm", 5, 4099, 515, "stream", 32, 16, 4), ("gemm", 17, 4099, 1300, "stream", 32, 32, 8), ("gemm", 33, 4099, 515, "stream", 32, 48, 4),
         ("gemm", 96, 64, 1300, "stream", 16, 48, 8), ("gemm", 150, 300, 1300, "stream", 16, 48, 8), ("gemm", 70, 300, 1300, "stream", 16, 48, 8),
         ("gated", 1, 64, 515, "stream", 32, 4, 4), ("gated", 5, 300, 1300, "stream", 32, 16, 8), ("gated", 17, 64, 64, "stream", 32, 32, 2), ("gated", 33, 64, 515, "stream", 32, 48, 4),
         ("gemm", 200, 200, 200, "tile", 128, 64, False), ("gemm", 200, 200, 2600, "tile", 128, 64, True), ("gemm", 200, 8200, 200, "tile", 256, 64, False),
         ("gemm", 130, 4099, 8200, "tile", 256, 64, True), ("gemm", 513, 8200, 200, "tile", 256, 128, False), ("gemm", 70, 5003, 8200, "tile", 256, 128, True),
         ("gated", 200, 200, 200, "tile", 128, 64, False), ("gated", 200, 200, 2600, "tile", 128, 64, True), ("gated", 200, 4099, 200, "tile", 256, 64, False),
         ("gated", 130, 2050, 8200, "tile", 256, 64, True), ("gated", 200, 8200, 200, "tile", 256, 128, False), ("gated", 70, 4099, 8200, "tile", 256, 128, True),
         ("gemm_t", 70, 200, 200, "back", 128, 64, False), ("gemm_t", 70, 2050, 200, "back", 128, 64, True), ("gemm_t", 200, 200, 8200, "back", 128, 128, False),
         ("gemm_t", 70, 2050, 4100, "back", 128, 128, True), ("gemm_t", 400, 200, 8200, "back", 256, 128, False), ("gemm_t", 70, 8200, 8200, "back", 256, 128, True),
         ("gemm_t", 3000, 200, 2600, "back", 256, 256, False), ("gemm_t", 130, 4099, 8200, "back", 256, 256, True),
         ("gated_backward", 70, 200, 200, "back", 128, 64, False), ("gated_backward", 70, 515, 200, "back", 128, 64, True), ("gated_backward", 200, 200, 8200, "back", 128, 128, False),
         ("gated_backward", 130, 2050, 1300, "back", 128, 128, True), ("gated_backward", 400, 200, 8200, "back", 256, 128, False), ("gated_backward", 70, 4099, 8200, "back", 256, 128, True),
         ("gated_backward", 3000, 200, 2600, "back", 256, 256, False), ("gated_backward", 130, 4099, 4100, "back", 256, 256, True)]


def _planned(call, m, n, k, kernel, outputs, tokens, shared):
    p = B.slim_group_q4_plan(n, k, m, call)
    assert (p["kernel"], p["outputs"], p["tokens"]) == (kernel, outputs, tokens), p
    assert p["shared"] == shared if kernel == "stream" else (p["shared"] > 1) == shared, p


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("plan", PLANS, ids=lambda p: "-".join(map(str, p)))
def test_within_bounds(plan, dtype):
    call, m, n, k = plan[:4]
    _planned(*plan)
    group = (32, 64, 128)[(m + n + k) % 3]
    (one, Vg), (two, Vu) = _weights(n, k, group, True, n, 0.002), _weights(n, k, group, False, k, 0.002)
    if call in ("gemm", "gated"):
        X = _matrix(m, k, dtype, m)
        x = _np(X)
        if call == "gemm":
            ref, mag = O.gemm(x, Vg)
            _check(B.slim_group_q4_gemm(one, X), ref, _sum_bound(mag, k, x, dtype), dtype)
        else:
            _check_gated(*B.slim_group_q4_gated(one, two, X, G=True, U=True), x, Vg, Vu, k, dtype)
        return
    dY = _matrix(m, n, dtype, m)
    if call == "gemm_t":
        y = _np(dY)
        ref, mag = O.gemm(y, Vg.T)
        _check(B.slim_group_q4_gemm_t(one, dY), ref, _sum_bound(mag, n, y, dtype), dtype)
    else:
        G, U = _matrix(m, n, dtype, m + 1, 2.0), _matrix(m, n, dtype, m + 2, 2.0)
        dX, dG, dU = B.slim_group_q4_gated_backward(one, two, dY, G, U)
        _check_backward(dX, dG, dU, dY, G, U, Vg, Vu, dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("plan", [p for p in PLANS if p[0] in ("gemm", "gemm_t")], ids=lambda p: "-".join(map(str, p)))
def test_to_the_bit(plan, dtype):
    """Scales that are powers of two, whole weights (no rounding of theirs), inputs of -1, 0 and 1: sums are whole numbers times the smallest scale, exact in binary32, and the
    result is the exact one rounded once."""
    call, m, n, k = plan[:4]
    _planned(*plan)
    g = np.random.default_rng(m + n + k)
    group = (32, 64, 128)[(m + n + k) % 3]
    codes, points = g.integers(0, 16, (n, k), dtype=np.uint8), g.integers(0, 16, (n, O.groups(k, group)), dtype=np.uint8)
    scales = (2.0 ** g.integers(-6, -3, points.shape)).astype(np.float16)
    layer = B.SlimGroupQ4Weight(n, k, group, B.slim_group_q4_tile(torch.from_numpy(codes).to(DEV)), torch.from_numpy(scales).to(DEV), torch.from_numpy(points).to(DEV))
    V = O.values(codes, scales, points, group)
    x = g.integers(-1, 2, (m, k if call == "gemm" else n)).astype(np.float64)
    X = torch.from_numpy(x).to(dtype).to(DEV)
    got = B.slim_group_q4_gemm(layer, X) if call == "gemm" else B.slim_group_q4_gemm_t(layer, X)
    want = torch.from_numpy(x @ (V.T if call == "gemm" else V)).float().to(dtype)      # (15 * 2^3 * 8200 and the like: exact in 32 bits)
    assert torch.equal(got.cpu(), want)
