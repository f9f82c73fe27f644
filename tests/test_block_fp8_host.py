"""The 8-bit operators with a scale for each block of 128: sizes and refusals (host logic, nothing is launched), and the oracle's own pins."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import block_fp8 as O
from paper_2410_09615_amd import binding as B

A = ctypes.c_void_p(0x1000)              # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1001)
FOUR = ctypes.c_void_p(0x1004)           # for 32-bit elements
HALF = ctypes.c_void_p(0x1002)           # aligned for 16-bit elements, not for codes


def test_sizes():
    c, s = ctypes.c_size_t(), ctypes.c_size_t()
    assert B.lib().slim_block_fp8_sizes(5, 129, c, s) == 0 and (c.value, s.value) == (5 * 256, 5 * 2 * 4)
    assert B.lib().slim_block_fp8_sizes(5, 129, None, None) == 0
    assert B.slim_block_fp8_weight_sizes(65, 129) == {"codes": 2 * 2 * 8192, "scales": 1 * 2 * 4}
    assert B.slim_block_fp8_weight_sizes(1, 1) == {"codes": 8192, "scales": 4}
    assert B.slim_block_fp8_weight_sizes(28672, 8192) == {"codes": 28672 * 8192, "scales": 224 * 64 * 4}
    for bad in ((0, 5), (5, 0), (-1, 5), (5, (1 << 22) + 1)):
        assert B.lib().slim_block_fp8_sizes(*bad, c, s) == B.SLIM_ERR_SHAPE
        assert B.lib().slim_block_fp8_weight_sizes(*bad, c, s) == B.SLIM_ERR_SHAPE
        assert B.lib().slim_block_fp8_gemm_workspace(*bad, 1, c) == B.SLIM_ERR_SHAPE
    assert B.lib().slim_block_fp8_gemm_workspace(5, 5, 0, c) == B.SLIM_ERR_SHAPE
    assert B.lib().slim_block_fp8_gemm_workspace(5, 5, 1, None) == B.SLIM_ERR_NULL


def test_the_workspace_of_more_tokens_covers_fewer():
    for n, k in ((1, 1), (1000, 1000), (4096, 4096), (5120, 5120), (28672, 8192)):
        sizes = [B.slim_block_fp8_gemm_workspace(n, k, m) for m in range(1, 1100)]
        assert sizes == sorted(sizes)


def test_norm_refuses():
    f = B.lib().slim_block_fp8_norm
    ok = dict(X=A, x_ld=256, res=A, res_ld=256, gain=A, gain_dtype=0, dtype=0, m=4, k=256, eps=1e-5, H=A, h_ld=256, Y=A, y_ld=256, codes=A, scales=A)
    call = lambda **kw: f(*{**ok, **kw}.values(), None)
    for name in ("X", "codes", "scales"):
        assert call(**{name: None}) == B.SLIM_ERR_NULL
    for kw in ({"m": 0}, {"k": 0}, {"k": (1 << 22) + 1, "x_ld": 1 << 23, "res_ld": 1 << 23, "h_ld": 1 << 23, "y_ld": 1 << 23}, {"dtype": 2}, {"dtype": -1},
               {"gain_dtype": 1}, {"gain_dtype": 3}, {"x_ld": 255}, {"res_ld": 255}, {"h_ld": 0}, {"y_ld": 255}, {"eps": -1e-9}, {"eps": float("nan")}):
        assert call(**kw) == B.SLIM_ERR_SHAPE, kw
    for kw in ({"X": ODD}, {"res": ODD}, {"gain": ODD}, {"gain": HALF, "gain_dtype": 2}, {"H": ODD}, {"Y": ODD}, {"codes": FOUR}, {"scales": HALF}):
        assert call(**kw) == B.SLIM_ERR_ALIGN, kw


def test_act_refuses():
    f = B.lib().slim_block_fp8_act
    ok = dict(G=A, g_ld=256, U=A, u_ld=256, act=1, dtype=0, m=4, k=256, codes=A, scales=A)
    call = lambda **kw: f(*{**ok, **kw}.values(), None)
    for name in ("G", "codes", "scales"):
        assert call(**{name: None}) == B.SLIM_ERR_NULL
    for kw in ({"m": 0}, {"k": 0}, {"act": 2}, {"act": -1}, {"dtype": 2}, {"g_ld": 255}, {"u_ld": 255}):
        assert call(**kw) == B.SLIM_ERR_SHAPE, kw
    for kw in ({"G": ODD}, {"U": ODD}, {"codes": FOUR}, {"scales": HALF}):
        assert call(**kw) == B.SLIM_ERR_ALIGN, kw


def test_weight_and_tile_refuse():
    f = B.lib().slim_block_fp8_weight
    assert f(None, 256, 2, 64, 256, A, A, None) == B.SLIM_ERR_NULL
    assert f(A, 256, 2, 64, 256, None, A, None) == B.SLIM_ERR_NULL
    assert f(A, 255, 2, 64, 256, A, A, None) == B.SLIM_ERR_SHAPE
    assert f(A, 256, 3, 64, 256, A, A, None) == B.SLIM_ERR_SHAPE
    assert f(A, 256, 2, 0, 256, A, A, None) == B.SLIM_ERR_SHAPE
    assert f(HALF, 256, 2, 64, 256, A, A, None) == B.SLIM_ERR_ALIGN
    assert f(HALF, 256, 0, 64, 256, HALF, A, None) == B.SLIM_ERR_ALIGN
    t, u = B.lib().slim_block_fp8_tile, B.lib().slim_block_fp8_untile
    assert t(None, 256, 64, 256, A, None) == B.SLIM_ERR_NULL and u(A, 64, 256, None, 256, None) == B.SLIM_ERR_NULL
    assert t(A, 255, 64, 256, A, None) == B.SLIM_ERR_SHAPE and u(A, 64, 256, A, 255, None) == B.SLIM_ERR_SHAPE
    assert t(ODD, 256, 64, 256, HALF, None) == B.SLIM_ERR_ALIGN and u(HALF, 64, 256, ODD, 256, None) == B.SLIM_ERR_ALIGN


def test_gemm_refuses():
    f = B.lib().slim_block_fp8_gemm
    layer = lambda **kw: ctypes.byref(B.slim_block_fp8_layer(**{**dict(n=64, k=256, codes=0x1000, scales=0x1000), **kw}))
    ok = dict(layer=layer(), X=A, xs=A, m=4, Y=A, y_ld=64, dtype=0, ws=A, ws_bytes=1 << 30)
    call = lambda **kw: f(*{**ok, **kw}.values(), None)
    for kw in ({"layer": None}, {"layer": layer(codes=None)}, {"layer": layer(scales=None)}, {"X": None}, {"xs": None}, {"Y": None}, {"ws": None}):
        assert call(**kw) == B.SLIM_ERR_NULL, kw
    for kw in ({"layer": layer(n=0)}, {"layer": layer(k=0)}, {"m": 0}, {"y_ld": 63}, {"dtype": 3}, {"dtype": -1}):
        assert call(**kw) == B.SLIM_ERR_SHAPE, kw
    for kw in ({"layer": layer(codes=0x1008)}, {"layer": layer(scales=0x1002)}, {"X": FOUR}, {"xs": HALF}, {"Y": ODD}, {"Y": HALF, "dtype": 2}, {"ws": HALF}):
        assert call(**kw) == B.SLIM_ERR_ALIGN, kw
    assert call(ws_bytes=16) == B.SLIM_ERR_WORKSPACE


def test_oracle_by_hand():
    """One block worked out on paper: top 4.48, scale 0.01; 1.0 is 100 steps of it, between the codes 96 and 104 (step 8) and a tie goes to even."""
    z = np.zeros((1, 130), np.float32)
    z[0, :5] = [4.48, -1.0, 0.02, 1e-6, -4.48]
    z[0, 129] = 2.0 ** -101
    codes, top = O.quantize_rows(z)
    assert codes.shape == (1, 256) and float(top[0, 0]) == float(np.float32(4.48)) and float(top[0, 1]) == 2.0 ** -100
    assert list(O.values(codes[0, :5])) == [448.0, -96.0, 2.0, 0.0, -448.0]
    assert float(O.values(codes[0, 129])) == 224.0
    h = O.norm(np.array([[3.0, 4.0]], np.float32), None, 0.0)
    assert np.allclose(h["y"], np.array([[3.0, 4.0]]) / np.sqrt(12.5)) and np.allclose(h["scales"], 4.0 / 448.0 / np.sqrt(12.5))
    o, i = np.meshgrid(np.arange(64), np.arange(128), indexing="ij")
    rows, cols = O.tile(o.astype(np.uint8)), O.tile(i.astype(np.uint8))
    place = {0: (0, 0), 1: (0, 1), 16: (1, 0), 64: (16, 0), 256: (0, 16), 1024: (0, 64), 2048: (4, 0), 8191: (63, 127)}
    assert rows.size == 8192 and all((rows[p], cols[p]) == at for p, at in place.items())
    y, mag = O.gemm(np.full((1, 128), 0x38, np.uint8), np.array([[2.0]]), np.full((1, 3), 0xB8, np.uint8), np.array([[0.5]]))
    assert float(y[0, 0]) == -3.0 and float(mag[0, 0]) == 3.0


@pytest.mark.parametrize("seed", range(3))
def test_oracle_values_and_codes_agree(seed):
    v = np.random.default_rng(seed).normal(0, 100, 1000)
    r = O.fp8_round(v, "e4m3")
    assert np.array_equal(O.values(O.fp8_encode(r, "e4m3")), r)


def test_binding_refuses_what_is_not_on_a_device():
    """The arguments are looked at in C, type and device first: nothing here reaches the library."""
    X = torch.zeros(4, 256, dtype=torch.float16)
    codes, scales = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 2)
    layer = B.SlimBlockFp8Weight(64, 256, torch.zeros(64 * 256, dtype=torch.uint8), torch.zeros(1, 2))
    for bad in (lambda: B.slim_block_fp8_norm(X), lambda: B.slim_block_fp8_norm(X.double(), codes=codes, scales=scales),
                lambda: B.slim_block_fp8_norm(X, codes=codes, scales=scales, H=X, Y=X), lambda: B.slim_block_fp8_act(X, codes=codes, scales=scales),
                lambda: B.slim_block_fp8_act(X, act="gelu"), lambda: B.slim_block_fp8_weight(X), lambda: B.slim_block_fp8_tile(codes),
                lambda: B.slim_block_fp8_gemm(layer, codes, scales, workspace=codes)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.slim_block_fp8_norm(None, codes=codes, scales=scales), lambda: B.slim_block_fp8_act(3, codes=codes, scales=scales)):
        with pytest.raises((AttributeError, TypeError)):
            bad()
