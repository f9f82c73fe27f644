"""The product of 8-bit inputs and weights where its loads and its two groups of wavefronts end: what lies behind a row's last block.

Bounds as in test_gpu_block_fp8.py: (128 + kb + 18) 2^-24 of the sum of the terms' magnitudes, above 64 tokens and in 16 bits 2^-10 of it more
(the 8-bit instruction's cut), and one rounding to the result's type.
"""
import numpy as np
import pytest
import torch

from oracle import block_fp8 as O
from paper_2410_09615_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF_ULP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: U}
NAN = 0x7F


def _codes(rows, cols, g):
    c = g.integers(0, 256, (rows, cols), dtype=np.uint8)
    c[(c & 0x7F) == 0x7F] = 0x3A
    return c


def _run(xc, xs, wc, ws, dtype):
    layer = B.SlimBlockFp8Weight(*wc.shape, B.slim_block_fp8_tile(torch.from_numpy(wc).to(DEV)), torch.from_numpy(ws).to(DEV))
    return B.slim_block_fp8_gemm(layer, torch.from_numpy(xc).to(DEV), torch.from_numpy(xs).to(DEV), dtype).double().cpu().numpy()


def _check(got, xc, xs, wc, ws, dtype):
    """Finite results within the bound, the others as the definition has them."""
    with np.errstate(all="ignore"):
        ref, mag = O.gemm(xc, xs, wc, ws)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    endless = np.isinf(ref)
    assert np.array_equal(got[endless], ref[endless])
    fine = np.isfinite(ref)
    bound = (128 + xs.shape[1] + 18) * U * mag
    if dtype != torch.float32 and got.shape[0] > 64:
        bound = bound + 2.0 ** -10 * mag
    assert np.all(np.abs(got - ref)[fine] <= (bound + HALF_ULP[dtype] * (np.abs(ref) + bound))[fine])


# one block (the second group has none), odd numbers of blocks (it has one less), more than the scales of one fetch
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("kb", [1, 3, 5, 17, 33])
@pytest.mark.parametrize("m", [3, 70, 130, 257])
def test_nothing_of_the_next_token_or_row_tile(m, kb, dtype):
    """The first block of every other token and of every other 64 rows, which lies behind the last block of the one before, is all NaN."""
    n, k = 300, kb * 128
    g = np.random.default_rng(m + kb)
    wc, xc = _codes(n, k, g), _codes(m, k, g)
    for t in range(64, n, 128):
        wc[t:t + 64, :128] = NAN
    xc[1::2, :128] = NAN
    ws = (2.0 ** g.uniform(-9, -6, (O.blocks(n), kb))).astype(np.float32)
    xs = (2.0 ** g.uniform(-9, -6, (m, kb))).astype(np.float32)
    got = _run(xc, xs, wc, ws, dtype)
    assert np.isfinite(got[0::2, :64]).all() and np.isnan(got[1::2]).all()
    _check(got, xc, xs, wc, ws, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("kb", [1, 3, 5, 17])
@pytest.mark.parametrize("m", [3, 70, 130, 257])
def test_an_infinite_scale_of_the_last_block(m, kb, dtype):
    """sum_b xs ws (sum of the block): a block's sum is a number, so its infinite scale gives an infinity of the sum's sign and no NaN
    (where the sum is further from zero than its own error)."""
    n, k = 300, kb * 128
    g = np.random.default_rng(100 * m + kb)
    wc, xc = _codes(n, k, g), _codes(m, k, g)
    ws = (2.0 ** g.uniform(-9, -6, (O.blocks(n), kb))).astype(np.float32)
    xs = (2.0 ** g.uniform(-9, -6, (m, kb))).astype(np.float32)
    ws[1, kb - 1] = np.inf
    xs[m - 1, kb - 1] = np.inf
    X, W = O.values(xc), O.values(wc)
    last, size = X[:, -128:] @ W[:, -128:].T, np.abs(X[:, -128:]) @ np.abs(W[:, -128:]).T
    cut = 128 * U + (2.0 ** -10 if dtype != torch.float32 and m > 64 else 0)
    got = _run(xc, xs, wc, ws, dtype)
    endless = np.zeros((m, n), bool)
    endless[:, 128:256] = True
    endless[m - 1] = True
    sure = endless & (np.abs(last) > cut * size)
    assert sure.sum() > 0.9 * endless.sum()
    assert np.array_equal(got[sure], np.copysign(np.inf, last)[sure]) and np.isfinite(got[~endless]).all()
    ws[1, kb - 1] = xs[m - 1, kb - 1] = 0
    got[endless] = 0
    ref, mag = O.gemm(xc, xs, wc, ws)
    bound = (128 + kb + 18) * U * mag + (2.0 ** -10 * mag if dtype != torch.float32 and m > 64 else 0)
    assert np.all((np.abs(got - ref) <= bound + HALF_ULP[dtype] * (np.abs(ref) + bound))[~endless])


def test_a_layer_whose_buffers_were_exchanged():
    """`.data` of a layer's tensors exchanged between products (weights reloaded or moved): the next product is on what is there now."""
    g = np.random.default_rng(5)
    wc, xc = _codes(70, 200, g), _codes(5, 256, g)
    xc[:, 200:] = 0
    ws, xs = np.full((1, 2), 0.25, np.float32), np.full((5, 2), 0.5, np.float32)
    X, S = torch.from_numpy(xc).to(DEV), torch.from_numpy(xs).to(DEV)
    layer = B.SlimBlockFp8Weight(70, 200, B.slim_block_fp8_tile(torch.from_numpy(wc).to(DEV)), torch.from_numpy(ws).to(DEV))
    first = layer.codes.data, layer.scales.data                        # (still there while the second product runs)
    _check(B.slim_block_fp8_gemm(layer, X, S, torch.float32).double().cpu().numpy(), xc, xs, wc, ws, torch.float32)
    wc = wc[::-1].copy()
    layer.codes.data = B.slim_block_fp8_tile(torch.from_numpy(wc).to(DEV))
    _check(B.slim_block_fp8_gemm(layer, X, S, torch.float32).double().cpu().numpy(), xc, xs, wc, ws, torch.float32)
    ws = 2 * ws
    layer.scales.data = torch.from_numpy(ws).to(DEV)
    _check(B.slim_block_fp8_gemm(layer, X, S, torch.float32).double().cpu().numpy(), xc, xs, wc, ws, torch.float32)
    layer.scales.data = layer.scales.data[:, :1].contiguous()
    with pytest.raises(ValueError):
        B.slim_block_fp8_gemm(layer, X, S, torch.float32)
    del first


def test_a_product_without_a_workspace_enqueues_nothing_else():
    """The default workspace is an allocation and no more: nothing reads it, so nothing fills it."""
    from torch.utils._python_dispatch import TorchDispatchMode

    class Names(TorchDispatchMode):
        def __init__(self):
            super().__init__()
            self.seen = []

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            self.seen.append(func.overloadpacket.__name__)
            return func(*args, **(kwargs or {}))

    g = np.random.default_rng(7)
    wc, xc = _codes(70, 256, g), _codes(2, 256, g)
    ws, xs = np.full((1, 2), 0.25, np.float32), np.full((2, 2), 0.5, np.float32)
    X, S = torch.from_numpy(xc).to(DEV), torch.from_numpy(xs).to(DEV)
    layer = B.SlimBlockFp8Weight(70, 256, B.slim_block_fp8_tile(torch.from_numpy(wc).to(DEV)), torch.from_numpy(ws).to(DEV))
    with Names() as names:
        Y = B.slim_block_fp8_gemm(layer, X, S, torch.float32)
    _check(Y.double().cpu().numpy(), xc, xs, wc, ws, torch.float32)
    assert set(names.seen) <= {"empty"}, names.seen
    for fill in (0, 0xFF):                              # whatever is in one
        full = torch.full((B.slim_block_fp8_gemm_workspace(70, 256, 2),), fill, dtype=torch.uint8, device=DEV)
        assert torch.equal(B.slim_block_fp8_gemm(layer, X, S, torch.float32, workspace=full), Y)
        assert bool((full == fill).all())


def test_one_token_of_a_wider_matrix():
    """A single row of codes has no gaps, whatever its stride says (torch calls it contiguous too); two rows of one have."""
    g = np.random.default_rng(9)
    wc, xc = _codes(70, 200, g), _codes(2, 256, g)
    xc[:, 200:] = 0
    ws, xs = np.full((1, 2), 0.25, np.float32), np.full((2, 2), 0.5, np.float32)
    layer = B.SlimBlockFp8Weight(70, 200, B.slim_block_fp8_tile(torch.from_numpy(wc).to(DEV)), torch.from_numpy(ws).to(DEV))
    wide, S = torch.zeros(2, 512, dtype=torch.uint8, device=DEV), torch.from_numpy(xs).to(DEV)
    wide[:, 256:] = torch.from_numpy(xc).to(DEV)
    one = wide[1:, 256:]
    assert one.is_contiguous()
    Y = B.slim_block_fp8_gemm(layer, one, S[1:], torch.float32)
    _check(Y.double().cpu().numpy(), xc[1:], xs[1:], wc, ws, torch.float32)
    with pytest.raises(ValueError):
        B.slim_block_fp8_gemm(layer, wide[:, 256:], S, torch.float32)
