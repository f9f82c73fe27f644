"""The 8-bit operators with a scale for each block of 128, against the oracle through the C-ABI.

Codes, tops and H are defined in binary32 and compared bit for bit.  Bounds for the rest, u = 2^-24:
  a norm's scale   the sum of k squares, all positive, loses at most one rounding per addition a term goes through:
                   (8 pieces of 8 in a lane, six steps over a wavefront, 16 wavefronts: 86; longer rows 8 more per 8192 values),
                   halved by the root, and five roundings follow:  (48 + 4 k / 8192 + 5) u;
  Y of the norm    that, one rounding for z and one for the product, and one to its type;
  the product      a term goes through at most 128 additions in its block, kb blocks and 16 shares, and two products:
                   (128 + kb + 16 + 2) u of the sum of the terms' magnitudes, and one rounding to its type; above 64 tokens, with
                   results in 16 bits, the 8-bit matrix instruction cuts each product 13 bits below the largest of its eight:
                   seven of eight terms lose up to 2^-13 of the largest, less than 2^-10 of the magnitudes' sum;
  an activation    the exponential's argument is rounded (|g| 1.45 u of the result), it, the sum, the quotient and the product
                   take two units each at most: (1.45 |g| + 8) u, so a code is one of those of the interval's ends.
"""
import ctypes

import numpy as np
import pytest
import torch

from oracle import block_fp8 as O
from paper_2410_09615_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF_ULP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: U}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133, torch.float32: 2.0 ** -149}
TYPES = [torch.float16, torch.bfloat16]


def _np32(t):
    return None if t is None else t.float().cpu().numpy()


def _rand(m, k, seed, dtype, outliers=True, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn(m, k, generator=g) * spread
    if outliers:
        X[:, torch.randperm(k, generator=g)[:max(1, k // 100)]] *= 20.0
    return X.to(dtype)


def _bits_equal(a, b):
    return np.array_equal(np.ascontiguousarray(a).view(np.uint8), np.ascontiguousarray(b).view(np.uint8))


def _same_codes(got, want):
    """Bit for bit, but for the sign of a NaN."""
    got = got.cpu().numpy().reshape(want.shape)
    nan = (want & 0x7F) == 0x7F
    return np.array_equal(got[~nan], want[~nan]) and np.all((got[nan] & 0x7F) == 0x7F)


def _check_norm(out, ref, k, dtype, H=True, Y=True):
    codes, scales, h, y = out
    assert _same_codes(codes, ref["codes"])
    rel = (53 + 4 * k / 8192) * U
    got = scales.cpu().numpy().astype(np.float64)
    fine = np.isfinite(ref["scales"])
    assert np.array_equal(np.isnan(got), np.isnan(ref["scales"]))
    assert np.all(np.abs(got - ref["scales"])[fine] <= rel * ref["scales"][fine] + 2.0 ** -149)
    if H:
        assert torch.equal(h.cpu(), torch.from_numpy(ref["h"]).to(dtype))
    if Y:
        e = np.abs(y.double().cpu().numpy() - ref["y"])
        assert np.all(e <= (HALF_ULP[dtype] * (1 + 1e-6) + rel + 2 * U) * np.abs(ref["y"]) + TINY[dtype])


# one block, one value, odd lengths, a wavefront's width, one and several pieces per lane, rows that are read twice
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k", [(1, 1), (3, 7), (2, 128), (5, 129), (1, 512), (4, 520), (7, 1000), (3, 5003), (1, 8192), (2, 8193), (2, 16385),
                                 (1, 32768), (2, 32777)])
def test_norm(m, k, dtype):
    X, res = _rand(m, k, 1, dtype), _rand(m, k, 2, dtype, spread=4.0)
    gain = (1 + 0.1 * torch.randn(k, generator=torch.Generator().manual_seed(3))).to(dtype)
    for r, g in ((res, gain), (None, gain.float()), (res, None)):
        ref = O.norm(_np32(X), _np32(g), 1e-5, _np32(r))
        dev = lambda t: None if t is None else t.to(DEV)
        out = B.slim_block_fp8_norm(X.to(DEV), dev(g), 1e-5, residual=dev(r), H=True, Y=True)
        _check_norm(out, ref, k, dtype)
        plain = B.slim_block_fp8_norm(X.to(DEV), dev(g), 1e-5, residual=dev(r))
        assert torch.equal(plain[0], out[0]) and torch.equal(plain[1], out[1]) and plain[2] is None and plain[3] is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [1000, 33000])
def test_norm_strides_and_in_place(dtype, k):
    """Rows with gaps at odd offsets; H over the residual, Y over X; nothing outside the rows is written."""
    m = 6
    wide = lambda s: _rand(m, k + 29, s, dtype).to(DEV)
    bx, br, bh, by = wide(1), wide(2), wide(3), wide(4)
    X, res, H, Y = (t[:, 3:3 + k] for t in (bx, br, bh, by))
    gain = _rand(1, k + 1, 5, dtype)[0, 1:].to(DEV)
    if gain.data_ptr() % 16 == 0:
        gain = _rand(1, k + 2, 5, dtype)[0, 1:1 + k].to(DEV)
    ref = O.norm(_np32(X), _np32(gain), 1e-6, _np32(res))
    guard = [t.clone() for t in (bh, by)]
    out = B.slim_block_fp8_norm(X, gain, 1e-6, residual=res, H=H, Y=Y)
    _check_norm(out, ref, k, dtype)
    for t, g in ((bh, guard[0]), (by, guard[1])):
        assert torch.equal(t[:, :3], g[:, :3]) and torch.equal(t[:, 3 + k:], g[:, 3 + k:])
    out = B.slim_block_fp8_norm(X, gain, 1e-6, residual=res, H=res, Y=X)
    _check_norm(out, ref, k, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_edges(dtype):
    """Rows of zeros, of the type's largest and smallest values, with a NaN, with an infinity; a block of zeros."""
    k = 384
    big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    X = _rand(8, k, 7, dtype, outliers=False)
    X[0] = 0
    X[1] = big
    X[2] = tiny / 4
    X[3, 200] = float("nan")
    X[4, 5] = float("inf")
    X[5, 128:256] = 0
    X[6, :] = -0.0
    X[7, 383] = big
    gain = torch.ones(k)
    gain[130] = -3.0
    ref = O.norm(_np32(X), gain.numpy(), 1e-6)
    codes, scales, _, Y = B.slim_block_fp8_norm(X.to(DEV), gain.to(DEV), 1e-6, Y=True)
    rows = [0, 2, 5, 6] + ([1, 7] if dtype == torch.float16 else [])
    assert _same_codes(codes[rows], ref["codes"][rows])
    got, want = scales.cpu().numpy().astype(np.float64)[rows], ref["scales"][rows]
    assert np.all(np.abs(got - want) <= 60 * U * want + 2.0 ** -149)
    # a NaN reaches every scale of its row; an infinity its block's, the other blocks' are zero, as they are of x / sqrt(inf)
    assert bool(torch.isnan(scales[3]).all()) and bool(torch.isnan(Y[3]).all())
    assert bool(torch.isnan(scales[4, 0])) and float(scales[4, 1]) == 0.0 and float(scales[4, 2]) == 0.0
    assert bool(torch.isnan(Y[4, 5])) and float(Y[4, 200]) == 0.0
    if dtype == torch.bfloat16:                   # squares past the largest binary32; three times the type's largest value is past it too
        assert float(scales[1, 0]) == 0.0 and bool(torch.isnan(scales[1, 1])) and float(scales[1, 2]) == 0.0
        assert float(scales[7].abs().max()) == 0.0
    assert int((codes[0] & 0x7F).max()) == 0 and int((codes[6] & 0x7F).max()) == 0          # (the gain of -3 makes one of them -0)


def test_norm_many_rows():
    """More rows than workgroups are launched."""
    m, k = (1 << 20) + 3, 8
    X = _rand(m, k, 9, torch.float16, outliers=False).to(DEV)
    codes, scales, _, _ = B.slim_block_fp8_norm(X, None, 1e-5)
    for rows in (slice(0, 5), slice(m - 6, m)):
        ref = O.norm(_np32(X[rows]), None, 1e-5)
        assert _same_codes(codes[rows], ref["codes"])
        assert np.all(np.abs(scales[rows].cpu().numpy() - ref["scales"]) <= 53 * U * ref["scales"])


def _check_act(codes, scales, a, slack):
    """a in 64 bits, slack: how far a value may be off.  The top is one of its interval's; a code lies between those of the interval's ends."""
    m, k = a.shape
    kb = O.blocks(k)
    pad = lambda t: np.concatenate([t, np.zeros((m, kb * 128 - k))], axis=1).reshape(m, kb, 128)
    A, S = pad(np.abs(a)), pad(slack)
    got = scales.cpu().numpy().astype(np.float64)
    lo, hi = np.maximum((A - S).max(axis=2), 2.0 ** -100), np.maximum((A + S).max(axis=2), 2.0 ** -100)
    assert np.all(got * 448.0 >= lo * (1 - 2 * U)) and np.all(got * 448.0 <= hi * (1 + 2 * U))
    v = np.abs(O.values(codes.cpu().numpy().reshape(m, kb, 128)))
    sign = np.signbit(O.values(codes.cpu().numpy().reshape(m, kb, 128)))
    q_lo = np.maximum(A - S, 0) / got[:, :, None] * (1 - 4 * U)
    q_hi = (A + S) / got[:, :, None] * (1 + 4 * U)
    r = lambda t: O.fp8_round(t, "e4m3")
    assert np.all(v >= r(q_lo)) and np.all(v <= r(q_hi))
    neg = pad(np.where(a < 0, 1.0, 0.0)) > 0
    assert np.all(sign[(v > 0)] == neg[(v > 0)])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k", [(1, 1), (2, 127), (3, 128), (16, 1000), (5, 13824), (300, 261)])
def test_act(m, k, dtype):
    G, V = _rand(m, k, 11, dtype, spread=3.0), _rand(m, k, 12, dtype)
    for u, act in ((V, "silu"), (None, "silu"), (V, "none"), (None, "none")):
        codes, scales = B.slim_block_fp8_act(G.to(DEV), None if u is None else u.to(DEV), act)
        g32, u32 = _np32(G), _np32(u)
        a = O.act(g32, u32, act == "silu")
        slack = ((1.45 * np.abs(g32) + 8) if act == "silu" else 1.0) * U * np.abs(a) + 2.0 ** -126
        _check_act(codes, scales, a, slack)
        if act == "none":                          # one binary32 product at most: bit for bit
            want, top = O.quantize_rows(g32 if u is None else g32 * u32)
            assert _same_codes(codes, want) and _bits_equal(scales.cpu().numpy(), (top / O.FMAX).astype(np.float32))


@pytest.mark.parametrize("dtype", TYPES)
def test_act_halves_of_one_matrix_and_edges(dtype):
    m, k = 9, 333
    both = _rand(m, 2 * k, 13, dtype).to(DEV)
    both[0, 0] = float("nan")
    both[1, 0], both[2, 0] = float("inf"), float("-inf")
    both[3, :k] = -200.0                            # the exponential overflows: silu is -0
    both[4, k:] = 0.0
    codes, scales = B.slim_block_fp8_act(both[:, :k], both[:, k:])
    s = scales.cpu()
    assert bool(torch.isnan(s[0, 0])) and bool(torch.isfinite(s[0, 1:]).all())
    assert float(s[1, 0]) == float("inf") and bool(torch.isnan(s[2, 0]))
    assert float(s[3].max()) == float(np.float32(2.0 ** -100) / np.float32(448)) and int((codes[3] & 0x7F).max()) == 0
    assert int((codes[4] & 0x7F).max()) == 0
    assert int(codes[1, 0] & 0x7F) == 0x7F and int((codes[1, 1:128] & 0x7F).max()) == 0
    rows = slice(5, m)
    g, u = _np32(both[rows, :k]), _np32(both[rows, k:])
    a = O.act(g, u, True)
    _check_act(codes[rows], scales[rows], a, (1.45 * np.abs(g) + 8) * U * np.abs(a) + 2.0 ** -126)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,k", [(1, 1), (64, 128), (65, 129), (128, 256), (200, 300), (129, 1000), (700, 515)])
def test_weight(n, k, dtype):
    W = _rand(n, k, 17, dtype, spread=0.02)
    if n > 128:
        W[128:, :min(k, 128)] = 0                   # a block of zeros
    want, sc = O.weight(_np32(W))
    codes, scales = B.slim_block_fp8_weight(W.to(DEV))
    assert _bits_equal(codes.cpu().numpy(), O.tile(want)) and _bits_equal(scales.cpu().numpy(), sc)
    assert _bits_equal(B.slim_block_fp8_untile(codes, n, k).cpu().numpy(), want)
    assert torch.equal(B.slim_block_fp8_tile(torch.from_numpy(want).to(DEV)), codes)
    wide = torch.zeros(n, k + 13, dtype=dtype, device=DEV)
    wide[:, 5:5 + k] = W.to(DEV)
    c2, s2 = B.slim_block_fp8_weight(wide[:, 5:5 + k])
    assert torch.equal(c2, codes) and torch.equal(s2, scales)
    rows = torch.zeros(n, k + 3, dtype=torch.uint8, device=DEV)
    rows[:, 1:1 + k] = torch.from_numpy(want).to(DEV)
    assert torch.equal(B.slim_block_fp8_tile(rows[:, 1:1 + k]), codes)


def test_weight_not_finite():
    W = _rand(256, 256, 19, torch.float32)
    W[3, 5], W[200, 10] = float("nan"), float("inf")
    codes, scales = B.slim_block_fp8_weight(W.to(DEV))
    c = B.slim_block_fp8_untile(codes, 256, 256).cpu()
    assert bool(torch.isnan(scales[0, 0])) and float(scales[1, 0]) == float("inf") and bool(torch.isfinite(scales[:, 1]).all())
    assert bool(((c[:128, :128] & 0x7F) == 0x7F).all())
    assert int(c[200, 10] & 0x7F) == 0x7F and int((c[128:, :128] & 0x7F).sum()) == 0x7F


def _layer(n, k, seed):
    g = np.random.default_rng(seed)
    wc = g.integers(0, 256, (n, k), dtype=np.uint8)
    wc[(wc & 0x7F) == 0x7F] = 0x3A
    ws = (2.0 ** g.uniform(-12, -4, (O.blocks(n), O.blocks(k)))).astype(np.float32)
    layer = B.SlimBlockFp8Weight(n, k, B.slim_block_fp8_tile(torch.from_numpy(wc).to(DEV)), torch.from_numpy(ws).to(DEV))
    return wc, ws, layer


def _inputs(m, k, seed):
    g = np.random.default_rng(seed)
    kb = O.blocks(k)
    xc = g.integers(0, 256, (m, kb * 128), dtype=np.uint8)
    xc[(xc & 0x7F) == 0x7F] = 0xB5
    xc[:, k:] = 0
    return xc, (2.0 ** g.uniform(-10, 2, (m, kb))).astype(np.float32)


def _check_product(Y, xc, xs, wc, ws, dtype, rows=slice(None)):
    ref, mag = O.gemm(xc[rows], xs[rows], wc, ws)
    got = Y[rows].double().cpu().numpy()
    bound = (128 + xs.shape[1] + 18) * U * mag
    if dtype != torch.float32 and Y.shape[0] > 64:
        bound = bound + 2.0 ** -10 * mag
    over = np.abs(ref) + bound > float(torch.finfo(dtype).max)          # may round to an infinity
    assert np.all(np.abs(got - ref)[~over] <= (bound + HALF_ULP[dtype] * (np.abs(ref) + bound) + TINY[dtype])[~over])
    assert np.all(np.abs(got[over]) >= float(torch.finfo(dtype).max) * (1 - 2 ** -8))


# every kernel and their edges: tokens below and above each tile's, rows that end inside a fragment, one block and many, fewer blocks than wavefronts
@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 33, 48, 64, 65, 127, 129, 200, 257, 520])
@pytest.mark.parametrize("n,k", [(1, 1), (5, 128), (64, 200), (130, 1000), (400, 2176), (1025, 515)])
def test_product(m, n, k):
    wc, ws, layer = _layer(n, k, 23)
    xc, xs = _inputs(m, k, 29 + m)
    X, S = torch.from_numpy(xc).to(DEV), torch.from_numpy(xs).to(DEV)
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        _check_product(B.slim_block_fp8_gemm(layer, X, S, dtype), xc, xs, wc, ws, dtype)


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (1, 11008, 4096), (16, 8192, 8192), (3, 28672, 1024), (48, 5120, 5120), (100, 4096, 4096),
                                   (333, 10007, 4100), (512, 4096, 11008), (1000, 5120, 2560), (2100, 8200, 640), (4096, 4096, 256)])
def test_product_of_layers(m, n, k):
    """Sizes of whole layers: a few tokens of each result against the oracle, all of it against itself on another call."""
    wc, ws, layer = _layer(n, k, 31)
    xc, xs = _inputs(m, k, 37)
    X, S = torch.from_numpy(xc).to(DEV), torch.from_numpy(xs).to(DEV)
    ws_buf = B.alloc_block_fp8_workspace(layer, m)
    Y = B.slim_block_fp8_gemm(layer, X, S, torch.float32, workspace=ws_buf)
    rows = sorted({0, m // 2, m - 1, m // 3, min(m - 1, 255), min(m - 1, 256)})
    _check_product(Y, xc, xs, wc, ws, torch.float32, rows)
    for _ in range(3):
        assert torch.equal(B.slim_block_fp8_gemm(layer, X, S, torch.float32, workspace=ws_buf), Y)
    # a token's result is the same in any company that takes the same kernel, and near it in any other
    alone = B.slim_block_fp8_gemm(layer, X[m - 1:], S[m - 1:], torch.float32)
    _check_product(alone, xc[m - 1:], xs[m - 1:], wc, ws, torch.float32)


@pytest.mark.parametrize("m", [3, 40, 150, 600])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_product_strided_output(m, dtype):
    """Y inside a wider matrix at an odd offset: its rows and nothing else."""
    n, k = 259, 700
    wc, ws, layer = _layer(n, k, 41)
    xc, xs = _inputs(m, k, 43)
    wide = torch.full((m + 2, n + 7), 3.0, dtype=dtype, device=DEV)
    Y = wide[1:m + 1, 3:3 + n]
    B.slim_block_fp8_gemm(layer, torch.from_numpy(xc).to(DEV), torch.from_numpy(xs).to(DEV), Y=Y)
    _check_product(Y, xc, xs, wc, ws, dtype)
    wide[1:m + 1, 3:3 + n] = 3.0
    assert bool((wide == 3.0).all())


@pytest.mark.parametrize("m", [2, 33, 140, 300])
def test_product_not_finite(m):
    """A NaN code, a NaN scale and an infinite scale reach their row or token, and no other."""
    n, k = 200, 640
    wc, ws, layer = _layer(n, k, 47)
    xc, xs = _inputs(m, k, 53)
    xc[m - 1, 130] = 0x7F
    xs[0, 4] = np.inf
    Y = B.slim_block_fp8_gemm(layer, torch.from_numpy(xc).to(DEV), torch.from_numpy(xs).to(DEV), torch.float32)
    assert bool(torch.isnan(Y[m - 1]).all()) and not bool(torch.isfinite(Y[0]).any())
    assert bool(torch.isfinite(Y[1:m - 1]).all())
    wc[7, 639] = 0xFF
    layer.codes = B.slim_block_fp8_tile(torch.from_numpy(wc).to(DEV))
    xc, xs = _inputs(m, k, 59)
    Y = B.slim_block_fp8_gemm(layer, torch.from_numpy(xc).to(DEV), torch.from_numpy(xs).to(DEV), torch.float32)
    assert bool(torch.isnan(Y[:, 7]).all())
    Y[:, 7] = 0
    assert bool(torch.isfinite(Y).all())


def test_streams_and_graph():
    """Calls on two streams with a workspace each, and a recorded chain of the operators replayed between eager calls."""
    m, n, k = 24, 1000, 1024
    wc, ws, layer = _layer(n, k, 61)
    X = _rand(m, k, 67, torch.float16).to(DEV)
    res = _rand(m, k, 71, torch.float16).to(DEV)
    codes, scales, H, _ = B.slim_block_fp8_norm(X, None, residual=res, H=True)
    want = B.slim_block_fp8_gemm(layer, codes, scales)
    torch.cuda.synchronize()
    outs = []
    for _ in range(2):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            ws_buf = B.alloc_block_fp8_workspace(layer, m)
            outs.append([B.slim_block_fp8_gemm(layer, codes, scales, workspace=ws_buf) for _ in range(4)])
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for ys in outs for y in ys)
    ws_buf = B.alloc_block_fp8_workspace(layer, m)
    c2, s2, Y2 = torch.zeros_like(codes), torch.zeros_like(scales), torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.slim_block_fp8_norm(X, None, residual=res, codes=c2, scales=s2)
        B.slim_block_fp8_gemm(layer, c2, s2, Y=Y2, workspace=ws_buf)
    for i in range(4):
        X.copy_(_rand(m, k, 80 + i, torch.float16))
        Y2.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        e = B.slim_block_fp8_norm(X, None, residual=res)
        assert torch.equal(Y2, B.slim_block_fp8_gemm(layer, e[0], e[1]))
        torch.cuda.synchronize()


def test_binding_refuses():
    X = torch.zeros(4, 256, dtype=torch.float16, device=DEV)
    for bad in (lambda: B.slim_block_fp8_norm(X.float()), lambda: B.slim_block_fp8_norm(X.cpu()), lambda: B.slim_block_fp8_norm(X.t()),
                lambda: B.slim_block_fp8_norm(X, residual=X[:3]), lambda: B.slim_block_fp8_norm(X, residual=X.bfloat16()),
                lambda: B.slim_block_fp8_norm(X, gain=torch.ones(255, device=DEV)), lambda: B.slim_block_fp8_norm(X, Y=X[:, :128]),
                lambda: B.slim_block_fp8_norm(X, codes=torch.zeros(4, 255, dtype=torch.uint8, device=DEV)),
                lambda: B.slim_block_fp8_act(X, X[:, :255]), lambda: B.slim_block_fp8_act(X, act="relu"),
                lambda: B.slim_block_fp8_weight(X.double()), lambda: B.slim_block_fp8_untile(torch.zeros(9, dtype=torch.uint8, device=DEV), 4, 4)):
        with pytest.raises(ValueError):
            bad()
    layer = B.compress_block_fp8(torch.ones(100, 256, device=DEV))
    codes, scales = B.slim_block_fp8_act(X, act="none")
    for bad in (lambda: B.slim_block_fp8_gemm(layer, codes[:, :128], scales), lambda: B.slim_block_fp8_gemm(layer, codes, scales[:3]),
                lambda: B.slim_block_fp8_gemm(layer, codes, scales, torch.float64),
                lambda: B.slim_block_fp8_gemm(layer, codes, scales, Y=torch.zeros(4, 99, dtype=torch.float16, device=DEV)),
                lambda: B.slim_block_fp8_gemm(B.SlimBlockFp8Weight(101, 257, layer.codes, layer.scales), codes, scales)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.SlimError) as e:
        B.slim_block_fp8_gemm(layer, codes, scales, workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == B.SLIM_ERR_WORKSPACE
    with pytest.raises(B.SlimError) as e:
        B.slim_block_fp8_norm(X, eps=-1.0)
    assert e.value.status == B.SLIM_ERR_SHAPE
