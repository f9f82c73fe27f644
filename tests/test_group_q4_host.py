"""The operators on 4-bit weights with group scales: sizes and refusals (host logic, nothing is launched), and the oracle's own pins."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import group_q4 as O
from paper_2410_09615_amd import binding as B

A = ctypes.c_void_p(0x1000)              # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1001)
HALF = ctypes.c_void_p(0x1002)           # aligned for 16-bit elements, not for codes


def _layer(**kw):
    return ctypes.byref(B.slim_group_q4_layer(**{**dict(n=64, k=256, group=128, codes=0x1000, scales=0x1000, zeros=0x1001), **kw}))


def test_sizes():
    assert B.slim_group_q4_sizes(17, 129, 32) == {"codes": 2 * 2 * 1024, "scales": 17 * 5 * 2, "zeros": 17 * 5}
    assert B.slim_group_q4_sizes(1, 1, 128) == {"codes": 1024, "scales": 2, "zeros": 1}
    assert B.slim_group_q4_sizes(28672, 8192, 64) == {"codes": 28672 * 4096, "scales": 28672 * 128 * 2, "zeros": 28672 * 128}
    assert B.lib().slim_group_q4_sizes(5, 129, 64, None, None, None) == 0
    for bad in ((0, 5, 32), (5, 0, 32), (-1, 5, 32), (5, (1 << 22) + 1, 32), (5, 5, 16), (5, 5, 0), (5, 5, 256), (5, 5, -32), (1 << 30, 1 << 22, 128)):
        assert B.lib().slim_group_q4_sizes(*bad, None, None, None) == B.SLIM_ERR_SHAPE, bad


def test_weight_tile_and_values_refuse():
    f = B.lib().slim_group_q4_weight
    ok = dict(W=A, ld=256, dtype=2, n=64, k=256, group=64, codes=A, scales=A, zeros=ODD)
    call = lambda **kw: f(*{**ok, **kw}.values(), None)
    for name in ("W", "codes", "scales"):
        assert call(**{name: None}) == B.SLIM_ERR_NULL
    for kw in ({"ld": 255}, {"dtype": 3}, {"dtype": -1}, {"n": 0}, {"k": 0}, {"group": 48}):
        assert call(**kw) == B.SLIM_ERR_SHAPE, kw
    for kw in ({"W": HALF}, {"W": ODD, "dtype": 0}, {"codes": HALF}, {"scales": ODD}):
        assert call(**kw) == B.SLIM_ERR_ALIGN, kw
    t, u, v = B.lib().slim_group_q4_tile, B.lib().slim_group_q4_untile, B.lib().slim_group_q4_values
    assert t(None, 256, 64, 256, A, None) == B.SLIM_ERR_NULL and u(A, 64, 256, None, 256, None) == B.SLIM_ERR_NULL
    assert t(A, 255, 64, 256, A, None) == B.SLIM_ERR_SHAPE and u(A, 64, 256, A, 255, None) == B.SLIM_ERR_SHAPE
    assert t(ODD, 256, 64, 256, HALF, None) == B.SLIM_ERR_ALIGN and u(HALF, 64, 256, ODD, 256, None) == B.SLIM_ERR_ALIGN
    assert v(None, A, 256, 0, None) == B.SLIM_ERR_NULL and v(_layer(), None, 256, 0, None) == B.SLIM_ERR_NULL
    assert v(_layer(), A, 255, 0, None) == B.SLIM_ERR_SHAPE and v(_layer(), A, 256, 3, None) == B.SLIM_ERR_SHAPE
    assert v(_layer(group=100), A, 256, 0, None) == B.SLIM_ERR_SHAPE
    assert v(_layer(), ODD, 256, 0, None) == B.SLIM_ERR_ALIGN and v(_layer(codes=0x1008), A, 256, 0, None) == B.SLIM_ERR_ALIGN


@pytest.mark.parametrize("name", ["slim_group_q4_gemm", "slim_group_q4_gemm_t"])
def test_products_refuse(name):
    f, t = getattr(B.lib(), name), name.endswith("_t")
    ok = dict(layer=_layer(), x=A, x_ld=64 if t else 256, m=4, y=A, y_ld=256 if t else 64, dtype=0)
    call = lambda **kw: f(*{**ok, **kw}.values(), None, 0, None)
    for kw in ({"layer": None}, {"layer": _layer(codes=None)}, {"layer": _layer(scales=None)}, {"x": None}, {"y": None}):
        assert call(**kw) == B.SLIM_ERR_NULL, kw
    for kw in ({"layer": _layer(n=0)}, {"layer": _layer(k=0)}, {"layer": _layer(group=16)}, {"m": 0}, {"m": -1}, {"x_ld": ok["x_ld"] - 1},
               {"y_ld": ok["y_ld"] - 1}, {"dtype": 2}, {"dtype": -1}):
        assert call(**kw) == B.SLIM_ERR_SHAPE, kw
    for kw in ({"layer": _layer(codes=0x1008)}, {"layer": _layer(scales=0x1001)}, {"x": ODD}, {"y": ODD}):
        assert call(**kw) == B.SLIM_ERR_ALIGN, kw


def test_gated_refuses():
    f = B.lib().slim_group_q4_gated
    ok = dict(gate=_layer(), up=_layer(zeros=None), x=A, x_ld=256, m=4, h=A, h_ld=64, g=A, g_ld=64, u=A, u_ld=64, dtype=1)
    call = lambda **kw: f(*{**ok, **kw}.values(), None, 0, None)
    for kw in ({"gate": None}, {"up": None}, {"up": _layer(codes=None)}, {"x": None}, {"h": None}):
        assert call(**kw) == B.SLIM_ERR_NULL, kw
    for kw in ({"up": _layer(n=65)}, {"up": _layer(k=255)}, {"gate": _layer(group=64)}, {"m": 0}, {"x_ld": 255}, {"h_ld": 63}, {"g_ld": 63}, {"u_ld": 0},
               {"dtype": 2}):
        assert call(**kw) == B.SLIM_ERR_SHAPE, kw
    for kw in ({"up": _layer(codes=0x1004)}, {"x": ODD}, {"h": ODD}, {"g": ODD}, {"u": ODD}):
        assert call(**kw) == B.SLIM_ERR_ALIGN, kw


def test_gated_backward_refuses():
    f = B.lib().slim_group_q4_gated_backward
    C, D, E, F, G = (ctypes.c_void_p(0x100000 * i) for i in range(1, 6))
    ok = dict(gate=_layer(), up=_layer(), dh=A, dh_ld=64, g=C, g_ld=64, u=D, u_ld=64, m=4, dg=E, dg_ld=64, du=F, du_ld=64, dx=G, dx_ld=256, dtype=0)
    call = lambda **kw: f(*{**ok, **kw}.values(), None, 0, None)
    for name in ("gate", "up", "dh", "g", "u", "dg", "du", "dx"):
        assert call(**{name: None}) == B.SLIM_ERR_NULL, name
    for kw in ({"up": _layer(n=65)}, {"up": _layer(group=32)}, {"m": 0}, {"dh_ld": 63}, {"g_ld": 63}, {"u_ld": 63}, {"dg_ld": 63}, {"du_ld": 63}, {"dx_ld": 255},
               {"dtype": 2}):
        assert call(**kw) == B.SLIM_ERR_SHAPE, kw
    for name in ("dh", "g", "u", "dg", "du", "dx"):
        assert call(**{name: ODD}) == B.SLIM_ERR_ALIGN, name
    assert call(dg=E, du=E) == B.SLIM_ERR_SHAPE                       # one would overwrite the other


def test_binding_refuses_what_is_not_on_a_device():
    X = torch.zeros(4, 256, dtype=torch.float16)
    layer = B.SlimGroupQ4Weight(64, 256, 128, torch.zeros(8192, dtype=torch.uint8), torch.zeros(64, 2, dtype=torch.float16))
    for bad in (lambda: B.slim_group_q4_weight(X), lambda: B.slim_group_q4_weight(X.double()), lambda: B.slim_group_q4_tile(X.to(torch.uint8)),
                lambda: B.slim_group_q4_gemm(layer, X), lambda: B.slim_group_q4_gemm_t(layer, X), lambda: B.slim_group_q4_gated(layer, layer, X),
                lambda: B.slim_group_q4_gated_backward(layer, layer, X, X, X), lambda: B.slim_group_q4_values(layer)):
        with pytest.raises(ValueError):
            bad()


def test_oracle_by_hand():
    """Two groups of 32 worked out on paper.  Symmetric: largest 7, scale 1; 2.5 is a tie and goes to 2.  With zero points: from -3 to 12, scale 1, zero 3."""
    W = np.zeros((1, 40), np.float32)
    W[0, :4] = [7.0, -7.0, 2.5, -0.5]
    W[0, 32:36] = [14.0, -14.0, 1.0, 3.0]
    codes, scales, _ = O.quantize(W, 32, False)
    assert list(codes[0, :5]) == [15, 1, 10, 8, 8] and list(codes[0, 32:37]) == [15, 1, 8, 10, 8] and list(scales[0]) == [1.0, 2.0]
    assert list(O.values(codes, scales, None, 32)[0, 32:36]) == [14.0, -14.0, 0.0, 4.0]         # 0.5 is a tie (to 0), 1.5 another (to 2)
    W[0, :4] = [12.0, -3.0, 2.5, 0.0]
    codes, scales, points = O.quantize(W, 32, True)
    assert float(scales[0, 0]) == 1.0 and points[0, 0] == 3 and list(codes[0, :4]) == [15, 0, 5, 3]
    assert list(O.values(codes, scales, points, 32)[0, :4]) == [12.0, -3.0, 2.0, 0.0]
    for zeros in (False, True):
        codes, scales, _ = O.quantize(np.zeros((1, 3), np.float32), 32, zeros)
        assert float(scales[0, 0]) == 1.0
        assert np.isnan(O.quantize(np.array([[1.0, np.inf]], np.float32), 32, zeros)[1]).all()
        assert float(O.quantize(np.array([[3e38, -3e38]], np.float32), 32, zeros)[1][0, 0]) == 65504.0
        assert float(O.quantize(np.array([[1e-30]], np.float32), 32, zeros)[1][0, 0]) == 2.0 ** -24


def test_oracle_layout():
    """Places that the header names: the dword of row r and inputs 32 j + 8 q .., nibble i + 4 h."""
    for r, c, byte, shift in ((0, 0, 0, 0), (0, 1, 2, 0), (0, 2, 0, 4), (0, 7, 3, 4), (1, 0, 16, 0), (0, 8, 256, 0), (0, 32, 4, 0), (15, 127, (16 * 3 + 15) * 16 + 15, 4)):
        codes = np.zeros((16, 128), np.uint8)
        codes[r, c] = 9
        t = O.tile(codes)
        assert t.size == 1024 and t[byte] == 9 << shift and np.count_nonzero(t) == 1
    codes = np.zeros((17, 130), np.uint8)
    codes[16, 129] = 5
    t = O.tile(codes)
    assert t.size == 4096 and t[3 * 1024 + 2] == 5


def test_oracle_gradients_by_differences():
    g = np.random.default_rng(0)
    G, U, dH = (g.normal(0, 2, (5, 7)) for _ in range(3))
    dG, dU = O.gated_backward(dH, G, U)
    step = 1e-6                                           # error of a central difference: step^2 |f'''| / 6 and 2^-53 |f| / step, below 1e-8 here
    for at in np.ndindex(5, 7):
        e = np.zeros((5, 7))
        e[at] = step
        assert abs(((O.gated(G + e, U) - O.gated(G - e, U)) * dH).sum() / (2 * step) - dG[at]) < 1e-7
        assert abs(((O.gated(G, U + e) - O.gated(G, U - e)) * dH).sum() / (2 * step) - dU[at]) < 1e-7


def test_workspaces():
    """Few tokens forward need none; where tiles are shared a call without room is refused before anything is launched."""
    for n, k in ((1, 1), (4096, 4096), (28672, 8192)):
        for call in ("gemm", "gated"):
            assert all(B.slim_group_q4_workspace(n, k, m, call) == 0 for m in (1, 2, 16, 17, 48))
    need = B.slim_group_q4_workspace(4096, 4096, 200, "gemm_t")
    assert need > 0 and need % (200 * 4096 * 4) == 0
    f = B.lib().slim_group_q4_gemm_t
    big = _layer(n=4096, k=4096)
    assert f(big, A, 4096, 200, A, 4096, 0, None, 0, None) == B.SLIM_ERR_WORKSPACE
    assert f(big, A, 4096, 200, A, 4096, 0, A, need - 1, None) == B.SLIM_ERR_WORKSPACE
    assert f(big, A, 4096, 200, A, 4096, 0, HALF, need, None) == B.SLIM_ERR_ALIGN
    out = ctypes.c_size_t()
    assert B.lib().slim_group_q4_workspace(5, 5, 1, 0, None) == B.SLIM_ERR_NULL
    for bad in ((0, 5, 1, 0), (5, 0, 1, 0), (5, 5, 0, 0), (5, 5, 1, 4), (5, 5, 1, -1)):
        assert B.lib().slim_group_q4_workspace(*bad, out) == B.SLIM_ERR_SHAPE, bad


def test_another_device_is_made_current_for_the_call(monkeypatch):
    """What the binding does where the tensors' device is not the current one (status 2), and where a layer's data has moved (1) or room is wanted."""
    seen = []
    monkeypatch.setattr(B.torch.cuda, "device", lambda d: __import__("contextlib").nullcontext(seen.append(d)))
    monkeypatch.setattr(B, "alloc_group_q4_workspace", lambda layer, m, call: ("room", m, call))
    calls = []

    def call(again, ws):
        calls.append((again, ws))
        return {1: 2, 2: B.SLIM_ERR_WORKSPACE, 3: 0}[len(calls)]
    B._q4_call("slim_group_q4_gemm_t", None, 5, 7, None, 1, call)
    assert seen == [5] and calls == [(True, None), (False, None), (False, ("room", 7, "gemm_t"))]
    with pytest.raises(B.SlimError):
        B._q4_call("slim_group_q4_gemm", None, 0, 1, "small", B.SLIM_ERR_WORKSPACE, call)


def test_sizes_beyond_32_bits_are_refused():
    """Not taken modulo 2^32: a matrix of 2^32 + 5 rows is not one of 5."""
    big = (1 << 32) + 5
    for bad in (lambda: B.slim_group_q4_sizes(big, 64), lambda: B.slim_group_q4_sizes(64, big), lambda: B.slim_group_q4_sizes(64, 64, big), lambda: B.alloc_group_q4(big, 1, device="cpu"),
                lambda: B.slim_group_q4_workspace(64, 64, big), lambda: B.slim_group_q4_workspace(big, 64, 1), lambda: B.slim_group_q4_plan(64, 64, big),
                lambda: B.SlimGroupQ4Weight(big, 64, 128, torch.zeros(4096, dtype=torch.uint8), torch.zeros(5, 1, dtype=torch.float16)).c_ref()):
        with pytest.raises(ValueError):
            bad()


def test_layers_that_no_launch_has_threads_for_are_refused():
    """Fewer than 2^32 threads: 64 to a block of codes that is made or read back, 128 to two blocks of rows that are streamed, or to one of a gated pair.  (Nothing is launched: the first refusal
    of what would have been is that of an odd address.)"""
    L = B.lib()
    rows = ((1 << 26) - 4) // 4 * 16                                  # of 512 inputs: 2^26 - 4 blocks
    weight = lambda n, k: L.slim_group_q4_weight(ODD, k, 0, n, k, 128, A, A, None, None)
    values = lambda n, k: L.slim_group_q4_values(_layer(n=n, k=k), ODD, k, 0, None)
    gemm = lambda n, k: L.slim_group_q4_gemm(_layer(n=n, k=k), ODD, k, 1, A, n, 0, None, 0, None)
    gated = lambda n, k: L.slim_group_q4_gated(_layer(n=n, k=k), _layer(n=n, k=k), ODD, k, 1, A, n, None, 0, None, 0, 0, None, 0, None)
    for f in (weight, values):
        assert f(rows, 512) == f(1 << 29, 128) == f(16, 1 << 22) == B.SLIM_ERR_ALIGN
        assert f(rows + 1, 512) == f(1 << 30, 1) == f(1 << 21, 1 << 16) == B.SLIM_ERR_SHAPE
    assert gemm((1 << 30) - 32, 1) == gemm(1 << 21, 1 << 16) == gated((1 << 29) - 16, 1) == gated(1 << 21, 1 << 16) == B.SLIM_ERR_ALIGN
    assert gemm((1 << 30) - 31, 1) == gated((1 << 29) - 15, 1) == B.SLIM_ERR_SHAPE


def test_scales_that_are_not_by_rows_are_refused(monkeypatch):
    """[groups][n], as some checkpoints hold them, has a layer's number of elements too."""
    monkeypatch.setattr(B, "_dev", lambda *a, **kw: None)             # (CPU tensors here; nothing is launched)
    make = lambda scales, zeros=None: B.SlimGroupQ4Weight(64, 256, 128, torch.zeros(8192, dtype=torch.uint8), scales, zeros).c_ref()
    s, z = torch.zeros(64, 2, dtype=torch.float16), torch.zeros(64, 2, dtype=torch.uint8)
    for good in ((s, None), (s, z), (s.flatten(), z.flatten()), (s[:, :, None], None)):
        make(*good)
    for bad in ((s.t().contiguous(), None), (s, z.t().contiguous())):
        with pytest.raises(ValueError, match="row-major"):
            make(*bad)
