"""The operators on 4-bit weights with group scales in the calls that their documentation allows: strides, odd addresses, what lies behind rows, infinities, streams, graphs, shared tiles.

Bounds as in test_gpu_group_q4.py.
"""
import copy
import pickle

import numpy as np
import pytest
import torch

from oracle import group_q4 as O
from paper_2410_09615_amd import binding as B
from paper_2410_09615_amd.mlp import GroupMlp
from tests.test_gpu_group_q4 import DEV, HALF, _check, _check_backward, _check_gated, _matrix, _np, _sum_bound, _weights

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def _untouched(t, gap):
    """What lies between and behind the rows of a matrix that _matrix made: still NaN."""
    whole = t.as_strided((t.shape[0], t.shape[1] + gap), (t.stride(0), 1))
    return bool(torch.isnan(whole[:, t.shape[1]:]).all())


# streamed, on tiles, tiles shared by workgroups
@pytest.mark.parametrize("m,n,k", [(1, 100, 300), (7, 515, 1003), (50, 4200, 515), (100, 700, 4100), (300, 4099, 1003)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_rows_with_gaps_at_odd_addresses(m, n, k, dtype):
    """Every matrix starts one element past an aligned address and has gaps of NaN, which are not read into results and not written."""
    (gate, Vg), (up, Vu) = _weights(n, k, 64, True, 1, 0.004), _weights(n, k, 64, False, 2, 0.004)
    X = _matrix(m, k, dtype, 3, gap=5, offset=1)
    Y, H, G, U = (_matrix(m, n, dtype, 9, gap=3, offset=1) for _ in range(4))
    x = _np(X)
    assert B.slim_group_q4_gemm(gate, X, Y=Y) is Y
    ref, mag = O.gemm(x, Vg)
    _check(Y, ref, _sum_bound(mag, k, x, dtype), dtype)
    B.slim_group_q4_gated(gate, up, X, H=H, G=G, U=U)
    _check_gated(H, G, U, x, Vg, Vu, k, dtype)
    dH, dG, dU, dX, dZ = _matrix(m, n, dtype, 4, gap=1, offset=1), *(_matrix(m, n, dtype, 8, gap=7, offset=1) for _ in range(2)), *(_matrix(m, k, dtype, 7, gap=9, offset=1) for _ in range(2))
    B.slim_group_q4_gated_backward(gate, up, dH, G, U, dG=dG, dU=dU, dX=dX)
    _check_backward(dX, dG, dU, dH, G, U, Vg, Vu, dtype)
    B.slim_group_q4_gemm_t(up, dH, dX=dZ)
    y = _np(dH)
    ref, mag = O.gemm(y, Vu.T)
    _check(dZ, ref, _sum_bound(mag, n, y, dtype), dtype)
    for t, gap in ((Y, 3), (H, 3), (G, 3), (U, 3), (dG, 7), (dU, 7), (dX, 9), (dZ, 9)):
        assert _untouched(t[:-1], gap)                                # (the last row's gap is past the buffer)


def test_halves_of_one_matrix():
    """G and U written into the halves of one matrix, and gradients over them: in place."""
    n, k, m = 260, 384, 70
    (gate, Vg), (up, Vu) = _weights(n, k, 32, False, 1, 0.004), _weights(n, k, 32, False, 2, 0.004)
    X, dH = _matrix(m, k, F16, 3), _matrix(m, n, F16, 4)
    both = torch.empty(m, 2 * n, dtype=F16, device=DEV)
    H, G, U = B.slim_group_q4_gated(gate, up, X, G=both[:, :n], U=both[:, n:])
    _check_gated(H, G, U, _np(X), Vg, Vu, k, F16)
    g, u = G.clone(), U.clone()
    dX, dG, dU = B.slim_group_q4_gated_backward(gate, up, dH, G, U, dG=G, dU=U)
    assert dG is G and dU is U
    _check_backward(dX, dG, dU, dH, g, u, Vg, Vu, F16)
    again = B.slim_group_q4_gated_backward(gate, up, dH, g, u, dG=g, dU=dH)          # dU over dH
    for a, b in zip(again, (dX, dG, dU)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("m", [1, 40, 70, 130, 300])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_tokens_that_are_not_finite_stay_their_own(m, dtype):
    """Infinities and NaN in some tokens: those tokens' results are what the definition has (an infinite product, or NaN), the others' are as without them."""
    n, k = 300, 1003
    layer, V = _weights(n, k, 64, True, 5)
    V[V == 0] = 1.0                                                   # (only the signs are used below, where the value is not 0)
    X = _matrix(m, k, dtype, 6)
    clean = B.slim_group_q4_gemm(layer, X).clone()
    dY = _matrix(m, n, dtype, 7)
    clean_t = B.slim_group_q4_gemm_t(layer, dY).clone()
    bad = X.clone()
    bad[m // 2, k - 1] = float("inf")
    got = B.slim_group_q4_gemm(layer, bad)
    w = B.slim_group_q4_values(layer, torch.float32)[:, k - 1]
    rows = torch.arange(m, device=DEV) != m // 2
    assert torch.equal(got[rows], clean[rows])
    hit = got[m // 2].float()
    assert bool(torch.isnan(hit[w == 0]).all()) and torch.equal(hit[w != 0], torch.where(w > 0, float("inf"), -float("inf"))[w != 0])
    bad = dY.clone()
    bad[m // 2, 0] = float("nan")
    got = B.slim_group_q4_gemm_t(layer, bad)
    assert torch.equal(got[rows], clean_t[rows]) and bool(torch.isnan(got[m // 2]).all())


@pytest.mark.parametrize("m", [3, 70, 300])
def test_scales_that_are_not_finite(m):
    """A scale of NaN: its row's results are NaN, and its group's inputs' gradients; no other's."""
    n, k = 300, 640
    layer, _ = _weights(n, k, 128, False, 5)
    X, dY = _matrix(m, k, F16, 6), _matrix(m, n, F16, 7)
    y, x = B.slim_group_q4_gemm(layer, X).clone(), B.slim_group_q4_gemm_t(layer, dY).clone()
    layer.scales[n - 1, 4] = float("nan")
    got = B.slim_group_q4_gemm(layer, X)
    assert bool(torch.isnan(got[:, n - 1]).all()) and torch.equal(got[:, :n - 1], y[:, :n - 1])
    got = B.slim_group_q4_gemm_t(layer, dY)
    assert bool(torch.isnan(got[:, 512:]).all()) and torch.equal(got[:, :512], x[:, :512])


def test_large_activations_saturate_as_the_definition():
    """silu far out on both sides, and its gradient: no NaN where the definition has none."""
    n = 64
    one = B.SlimGroupQ4Weight(n, 128, 128, B.slim_group_q4_tile(torch.full((n, 128), 9, dtype=torch.uint8, device=DEV)), torch.ones(n, 1, dtype=F16, device=DEV))
    X = torch.zeros(3, 128, dtype=BF16, device=DEV)
    X[0, 0], X[1, 0], X[2, 0] = 1e30, -1e30, -90.0
    H, G, U = B.slim_group_q4_gated(one, one, X, G=True, U=True)
    assert bool(torch.isinf(H[0]).all()) and bool((H[1] == 0).all()) and torch.equal(G, U)
    assert torch.allclose(H[2].double(), torch.full((n,), 90.0 ** 2 * np.exp(-90.0), dtype=torch.float64, device=DEV), rtol=2 ** -7)
    g = torch.tensor([[1e30, -1e30, -200.0, 200.0, 0.0]], dtype=BF16, device=DEV).repeat(1, 13)[:, :n].contiguous()
    dH = torch.ones(1, n, dtype=BF16, device=DEV)
    dX, dG, dU = B.slim_group_q4_gated_backward(one, one, dH, g, torch.ones_like(g))
    assert dG[0, :5].tolist() == [1.0, 0.0, 0.0, 1.0, 0.5] and dU[0, 1:5].tolist()[0:2] == [0.0, 0.0] and float(dU[0, 3]) == 200.0


@pytest.mark.parametrize("m,n,k", [(1, 1024, 4096), (16, 300, 700), (100, 512, 4096), (300, 4096, 1024)])
def test_captured_and_replayed(m, n, k):
    """The four calls recorded into one graph, replayed with other inputs and eager work between; a second graph with workspaces of its own replayed beside it."""
    (gate, Vg), (up, Vu) = _weights(n, k, 128, True, 1, 0.004), _weights(n, k, 128, False, 2, 0.004)
    rooms = lambda: {c: B.alloc_group_q4_workspace(gate, m, c) for c in B.Q4_CALLS}

    def step(X, dH, out, ws):
        B.slim_group_q4_gemm(gate, X, Y=out["Y"], workspace=ws["gemm"])
        B.slim_group_q4_gated(gate, up, X, H=out["H"], G=out["G"], U=out["U"], workspace=ws["gated"])
        B.slim_group_q4_gemm_t(gate, dH, dX=out["dZ"], workspace=ws["gemm_t"])
        B.slim_group_q4_gated_backward(gate, up, dH, out["G"], out["U"], dG=out["dG"], dU=out["dU"], dX=out["dX"], workspace=ws["gated_backward"])

    new = lambda: {name: torch.empty(m, k if name in ("dZ", "dX") else n, dtype=F16, device=DEV) for name in ("Y", "H", "G", "U", "dZ", "dG", "dU", "dX")}
    sets = []
    for i in range(2):
        X, dH, out = _matrix(m, k, F16, i), _matrix(m, n, F16, 10 + i), new()
        ws = rooms()
        step(X, dH, out, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(X, dH, out, ws)
        sets.append((graph, X, dH, out, ws))                       # (a recorded call's workspace has to live as long as its graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(3):
        eager = []
        for i, (graph, X, dH, out, _) in enumerate(sets):
            X.copy_(_matrix(m, k, F16, 100 * turn + i))
            dH.copy_(_matrix(m, n, F16, 100 * turn + 50 + i))
            want = new()
            step(X, dH, want, rooms())
            eager.append(want)
            for t in out.values():
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for stream, (graph, *_) in zip(streams, sets):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for want, (_, _, _, out, _) in zip(eager, sets):
            for name in out:
                assert torch.equal(out[name], want[name]), name
    _check_gated(sets[0][3]["H"], sets[0][3]["G"], sets[0][3]["U"], _np(sets[0][1]), Vg, Vu, k, F16)


@pytest.mark.parametrize("m", [1, 60, 333])
def test_repeats_and_streams_agree(m):
    """The same call twice, and on another stream, gives the same bits; a workspace that is too small is refused, one that is larger is taken."""
    n, k = 1100, 1500
    layer, _ = _weights(n, k, 32, True, 1)
    X, dY = _matrix(m, k, F16, 2), _matrix(m, n, F16, 3)
    Y, dX = B.slim_group_q4_gemm(layer, X), B.slim_group_q4_gemm_t(layer, dY)
    assert torch.equal(B.slim_group_q4_gemm(layer, X), Y)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a, b = B.slim_group_q4_gemm(layer, X), B.slim_group_q4_gemm_t(layer, dY)
    stream.synchronize()
    assert torch.equal(a, Y) and torch.equal(b, dX)
    need = B.slim_group_q4_workspace(n, k, m, "gemm_t")
    room = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    assert torch.equal(B.slim_group_q4_gemm_t(layer, dY, workspace=room), dX)
    if need:
        with pytest.raises(B.SlimError) as e:
            B.slim_group_q4_gemm_t(layer, dY, workspace=room[:need - 16])
        assert e.value.status == B.SLIM_ERR_WORKSPACE


@pytest.mark.parametrize("m", [5, 70])
def test_far_rows(m):
    """Rows so far apart that a call goes token by token (2^23 elements)."""
    n, k = 40, 200
    (gate, Vg), (up, Vu) = _weights(n, k, 64, True, 1, 0.004), _weights(n, k, 64, True, 2, 0.004)
    far = torch.empty(m * (1 << 23), dtype=F16, device=DEV)
    X = far.view(m, 1 << 23)[:, 3:3 + k]
    X.copy_(_matrix(m, k, F16, 5))
    assert torch.equal(B.slim_group_q4_gemm(gate, X), torch.cat([B.slim_group_q4_gemm(gate, X[t:t + 1].clone()) for t in range(m)]))
    H, G, U = B.slim_group_q4_gated(gate, up, X, G=True, U=True)
    _check_gated(H, G, U, _np(X), Vg, Vu, k, F16)
    dY = far.view(m, 1 << 23)[:, 1000:1000 + n]
    dY.copy_(_matrix(m, n, F16, 6))
    y = _np(dY)
    ref, mag = O.gemm(y, Vg.T)
    _check(B.slim_group_q4_gemm_t(gate, dY), ref, _sum_bound(mag, n, y, F16), F16)


def test_zero_points_of_any_byte():
    n, k, m = 64, 256, 70
    layer, _ = _weights(n, k, 64, True, 1)
    layer.zeros.random_(0, 256)
    codes = B.slim_group_q4_untile(layer.codes, n, k).cpu().numpy()
    V = O.values(codes, layer.scales.cpu().numpy(), layer.zeros.cpu().numpy(), 64)
    assert torch.equal(B.slim_group_q4_values(layer, torch.float32).double().cpu(), torch.from_numpy(V))
    for dtype in (F16, BF16):
        for tokens in (3, m):
            X, dY = _matrix(tokens, k, dtype, 2), _matrix(tokens, n, dtype, 3)
            x, y = _np(X), _np(dY)
            ref, mag = O.gemm(x, V)
            _check(B.slim_group_q4_gemm(layer, X), ref, _sum_bound(mag, k, x, dtype), dtype)
            ref, mag = O.gemm(y, V.T)
            _check(B.slim_group_q4_gemm_t(layer, dY), ref, _sum_bound(mag, n, y, dtype), dtype)


def test_layers_are_copied_stored_and_changed():
    layer, V = _weights(64, 256, 64, True, 1)
    X = _matrix(4, 256, F16, 2)
    Y = B.slim_group_q4_gemm(layer, X)
    for other in (copy.deepcopy(layer), pickle.loads(pickle.dumps(layer))):
        assert torch.equal(B.slim_group_q4_gemm(other, X), Y)
    layer.scales.data = layer.scales.data * 2                         # the tensor's data is elsewhere now
    assert torch.equal(B.slim_group_q4_gemm(layer, X), Y * 2)
    layer.zeros = None
    V = O.values(B.slim_group_q4_untile(layer.codes, 64, 256).cpu().numpy(), layer.scales.cpu().numpy(), None, 64)
    x = _np(X)
    ref, mag = O.gemm(x, V)
    _check(B.slim_group_q4_gemm(layer, X), ref, _sum_bound(mag, 256, x, F16), F16)


def test_binding_refuses():
    layer, _ = _weights(64, 256, 64, True, 1)
    other, _ = _weights(64, 256, 32, True, 1)
    X, H = _matrix(4, 256, F16, 2), _matrix(4, 64, F16, 3)
    for bad in (lambda: B.slim_group_q4_gemm(layer, X.float()), lambda: B.slim_group_q4_gemm(layer, X[:, :255]), lambda: B.slim_group_q4_gemm(layer, X, Y=H.to(BF16)),
                lambda: B.slim_group_q4_gemm(layer, X, Y=H[:3]), lambda: B.slim_group_q4_gemm(layer, X.t()), lambda: B.slim_group_q4_gemm(layer, X[0]),
                lambda: B.slim_group_q4_gemm_t(layer, X), lambda: B.slim_group_q4_gated(layer, layer, X, G=H[:, :63]), lambda: B.slim_group_q4_gemm(layer, X.cpu()),
                lambda: B.slim_group_q4_gated_backward(layer, layer, H, H, H.to(BF16)), lambda: B.slim_group_q4_gemm(layer, X, workspace=H),
                lambda: B.slim_group_q4_weight(X, layer=layer), lambda: B.slim_group_q4_values(layer, values=H)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.slim_group_q4_gated(layer, other, X), lambda: B.slim_group_q4_weight(X, group=48), lambda: B.slim_group_q4_gated_backward(layer, layer, H, H, H, dG=H, dU=H),
                lambda: B.slim_group_q4_gemm(layer, X[:1].expand(4, 256))):
        with pytest.raises(B.SlimError) as e:
            bad()
        assert e.value.status == B.SLIM_ERR_SHAPE
    with pytest.raises(B.SlimError):                                  # (no tokens: an empty tensor has no address either)
        B.slim_group_q4_gemm(layer, X[:0])


def test_product_and_gradient_by_differences():
    """<dY, Y(X + D) - Y(X - D)> = 2 <dX, D>: the product is linear, so the two sides differ by roundings alone."""
    n, k, m = 300, 515, 90
    layer, V = _weights(n, k, 64, True, 1)
    X, dY = _matrix(m, k, BF16, 2), _matrix(m, n, BF16, 3)
    D = (torch.randn(m, k, generator=torch.Generator().manual_seed(4)) * 0.5).to(BF16).to(DEV)
    p, q = (X.float() + D.float()).to(BF16), (X.float() - D.float()).to(BF16)
    left = (_np(dY) * (_np(B.slim_group_q4_gemm(layer, p)) - _np(B.slim_group_q4_gemm(layer, q)))).sum()
    right = (_np(B.slim_group_q4_gemm_t(layer, dY)) * (_np(p) - _np(q))).sum()
    bound = 0.0
    for x in (_np(p), _np(q)):
        ref, mag = O.gemm(x, V)
        e = _sum_bound(mag, k, x, BF16)
        bound += (np.abs(_np(dY)) * (e + HALF[BF16] * (np.abs(ref) + e))).sum()
    y = _np(dY)
    ref, mag = O.gemm(y, V.T)
    e = _sum_bound(mag, n, y, BF16)
    bound += (np.abs(_np(p) - _np(q)) * (e + HALF[BF16] * (np.abs(ref) + e))).sum()
    assert abs(left - right) <= bound and abs(right) > 0


@pytest.mark.parametrize("m", [1, 20, 130])
def test_a_run_of_them(m):
    """Weights quantized, the block forward with its products kept, the gradient back to its input: against the same on the values that the codes stand for."""
    k, f = 512, 1100
    g = torch.Generator().manual_seed(m)
    W = [torch.randn(*s, generator=g) * 0.03 for s in ((f, k), (f, k), (k, f))]
    mlp = GroupMlp(*(B.compress_group_q4(w.to(DEV), 64, zeros=True) for w in W), max_tokens=m)
    Vg, Vu, Vd = (_np(B.slim_group_q4_values(layer, torch.float32)) for layer in (mlp.gate, mlp.up, mlp.down))
    X, dY = _matrix(m, k, F16, 1), _matrix(m, k, F16, 2, 0.1)
    out, saved = mlp.forward(X, keep=True)
    assert torch.equal(mlp.forward(X)[0], out)
    H, G, U = saved
    _check_gated(H, G, U, _np(X), Vg, Vu, k, F16)
    h = _np(H)
    ref, mag = O.gemm(h, Vd)
    _check(out, ref, _sum_bound(mag, f, h, F16), F16)
    want_g, want_u = G.clone(), U.clone()
    dX, dH, dG, dU = mlp.backward(dY, saved)
    y = _np(dY)
    ref, mag = O.gemm(y, Vd.T)
    _check(dH, ref, _sum_bound(mag, k, y, F16), F16)
    _check_backward(dX, dG, dU, dH, want_g, want_u, Vg, Vu, F16)


def test_gradients_of_far_rows_in_place():
    """Rows 2^23 elements apart: dG over dH and dU over U, where a call goes token by token behind the activation's gradient."""
    n, k, m = 40, 200, 3
    (gate, Vg), (up, Vu) = _weights(n, k, 64, True, 1), _weights(n, k, 64, False, 2)
    far = torch.empty(m * (1 << 23), dtype=F16, device=DEV).view(m, 1 << 23)
    dH, G, U, dX = far[:, 1:1 + n], far[:, 100:100 + n], far[:, 201:201 + n], far[:, 300:300 + k]
    for i, t in enumerate((dH, G, U)):
        t.copy_(_matrix(m, n, F16, i, 2.0))
    h, g, u = dH.clone(), G.clone(), U.clone()
    out = B.slim_group_q4_gated_backward(gate, up, dH, G, U, dG=dH, dU=U, dX=dX)
    assert out[0] is dX and out[1] is dH and out[2] is U and torch.equal(G, g)
    _check_backward(dX, dH, U, h, g, u, Vg, Vu, F16)


@pytest.mark.parametrize("m", [1, 70])
def test_a_row_out_of_one_column_and_no_workspace_bytes(m):
    """Layers of one input or one output: a single row's stride says nothing, and a workspace without bytes is taken where none are needed."""
    (layer, V), (wide, Vw) = _weights(5, 1, 32, True, 1), _weights(1, 70, 32, False, 2)
    X = _matrix(m, 1, F16, 3)
    room = B.alloc_group_q4_workspace(layer, m)
    assert room.numel() == 0
    x = _np(X)
    ref, mag = O.gemm(x, V)
    _check(B.slim_group_q4_gemm(layer, X, workspace=room), ref, _sum_bound(mag, 1, x, F16), F16)
    X = _matrix(70, m, F16, 4).t() if m == 1 else _matrix(m, 70, F16, 4)              # (of one token: 1 x 70 with strides 1, 1)
    x = _np(X)
    ref, mag = O.gemm(x, Vw)
    _check(B.slim_group_q4_gemm(wide, X), ref, _sum_bound(mag, 70, x, F16), F16)
