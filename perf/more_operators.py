"""What is timed of the 4-bit layers with a scale for each group of inputs: their plain form and the framework's calls.

Weights are held as codes of 4 bits with a scale (fp16) and, where they are not symmetric, a zero point for each group
of 32, 64 or 128 inputs of a row: value = (code - zero point) * scale (`slim_group_q4_weight`; a checkpoint's codes are laid
out by `slim_group_q4_tile`).  `slim_group_q4_gemm` multiplies by them, `slim_group_q4_gated` is the first half of a
feed-forward block (both projections, the activation, their product), and the gradients that frozen weights pass on are
`slim_group_q4_gemm_t` and `slim_group_q4_gated_backward`.  Sizes are the layers of the package's workloads (4096 x 4096 to
28672 x 8192, 1 to 4096 tokens) and odd ones between.  Inputs are made on the device, with the distributions of those workloads.
"""
from __future__ import annotations

import math

import torch

DEV = "cuda:0"
own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
TINY = 2.0 ** -24      # smallest positive fp16
LARGE = 65504.0        # largest


def listed():
    return [
        # a layer is compressed where it is loaded, and read back to see what was lost: symmetric, as a checkpoint in fp16 holds it
        {"name": "weight_4096x4096_g128", "op": "weight", "n": 4096, "k": 4096, "group": 128, "zeros": False, "type": "f16"},
        # the same of a width that no group divides, from 32 bits, with zero points in small groups
        {"name": "weight_10007x5003_g32_f32", "op": "weight", "n": 10007, "k": 5003, "group": 32, "zeros": True, "type": "f32"},
        # one sequence being decoded, an attention projection: the smallest product, four per layer and token
        {"name": "gemm_1_4096x4096", "op": "gemm", "m": 1, "n": 4096, "k": 4096, "group": 128, "zeros": False, "type": "f16"},
        # 16 sequences decoded together on the widest projection of the widest model
        {"name": "gemm_16_28672x8192_bf16", "op": "gemm", "m": 16, "n": 28672, "k": 8192, "group": 128, "zeros": True, "type": "bf16"},
        # a prompt whose length is a multiple of nothing, on a layer whose sizes are not either, in small groups
        {"name": "gemm_333_10007x4100_g32", "op": "gemm", "m": 333, "n": 10007, "k": 4100, "group": 32, "zeros": True, "type": "f16"},
        # one sequence being decoded: the first half of the feed-forward part
        {"name": "gated_1_11008x4096", "op": "gated", "m": 1, "n": 11008, "k": 4096, "group": 128, "zeros": True, "type": "f16", "keep": False},
        # a few drafted tokens of each of several sequences, looked at together
        {"name": "gated_48_13824x5120_bf16", "op": "gated", "m": 48, "n": 13824, "k": 5120, "group": 64, "zeros": False, "type": "bf16", "keep": False},
        # a chunk of a long prompt on the widest model
        {"name": "gated_4096_28672x8192", "op": "gated", "m": 4096, "n": 28672, "k": 8192, "group": 128, "zeros": False, "type": "f16", "keep": False},
        # the gradient through a frozen attention projection: a training sequence
        {"name": "gemm_t_2048_4096x4096_bf16", "op": "gemm_t", "m": 2048, "n": 4096, "k": 4096, "group": 128, "zeros": True, "type": "bf16"},
        # the same of a short one with odd sizes
        {"name": "gemm_t_77_5003x4100", "op": "gemm_t", "m": 77, "n": 5003, "k": 4100, "group": 64, "zeros": False, "type": "f16"},
        # the gradient through a frozen feed-forward block's first half, a short sequence
        {"name": "backward_500_11008x4096", "op": "backward", "m": 500, "n": 11008, "k": 4096, "group": 32, "zeros": False, "type": "f16"},
        # the same of a training batch in bf16
        {"name": "backward_4096_11008x4096_bf16", "op": "backward", "m": 4096, "n": 11008, "k": 4096, "group": 128, "zeros": True, "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Any number, half of the time a multiple of 128 where it is large enough to be one."""
    v = _log_int(rng, lo, hi)
    return v // 128 * 128 if v >= 256 and rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["weight", "gemm", "gemm", "gated", "gated", "gemm_t", "backward"])
    case = {"op": op, "n": _size(rng, 128, 28672), "k": _size(rng, 128, 8192), "group": rng.choice([32, 64, 128]), "zeros": rng.random() < 0.5,
            "type": rng.choice(["f16", "bf16", "f32"] if op == "weight" else ["f16", "bf16"])}
    if op != "weight":
        case["m"] = _log_int(rng, 1, 4096)
    if op == "gated":
        case["keep"] = rng.random() < 0.4
    if op == "backward":                     # (no more work than the largest listed case)
        case["m"] = min(case["m"], 2048)
    return case


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _activations(m, k, g):
    X = torch.randn(m, k, generator=g, device=DEV)
    X[:, torch.randperm(k, generator=g, device=DEV)[:math.ceil(0.01 * k)]] *= 20.0      # outlier channels
    return X


def _groups(k, size):
    return (k + size - 1) // size


def _quantize(W, size, zeros):
    """W [n][k] fp32 -> (codes uint8 [n][k], scales fp16 [n][groups], zero points uint8 [n][groups] or None)."""
    n, k = W.shape
    kg = _groups(k, size)
    z = torch.nn.functional.pad(W, (0, kg * size - k)).view(n, kg, size)
    if zeros:
        lo, hi = z.amin(dim=2).clamp_max(0.0), z.amax(dim=2).clamp_min(0.0)
        span, steps = hi - lo, 15.0
    else:
        span, steps = z.abs().amax(dim=2), 7.0
    scale = (span / torch.full_like(span, steps)).to(torch.float16).float().clamp(TINY, LARGE)   # (a quotient by a plain number may be a product)
    scale = torch.where(span == 0, torch.ones_like(scale), scale)
    q = torch.round(z / scale[:, :, None])
    if zeros:
        zero = torch.round(-lo / scale).clamp(0, 15)
        codes = (q + zero[:, :, None]).clamp(0, 15)
        points = zero.to(torch.uint8)
    else:
        codes = q.clamp(-8, 7) + 8
        points = None
    return codes.view(n, kg * size)[:, :k].to(torch.uint8).contiguous(), scale.to(torch.float16), points


def _values(codes, scales, points, size):
    """What the codes stand for, fp32 [n][k]."""
    n, k = codes.shape
    kg = scales.shape[1]
    c = torch.nn.functional.pad(codes.float(), (0, kg * size - k)).view(n, kg, size)
    c = c - (8.0 if points is None else points.float()[:, :, None])
    return (c * scales.float()[:, :, None]).view(n, kg * size)[:, :k]


def _weights(case, g):
    """One layer's weights in fp32; where they have zero points, groups lie to one side as a checkpoint's do."""
    n, k = case["n"], case["k"]
    W = torch.randn(n, k, generator=g, device=DEV) * 0.02
    if case["zeros"]:
        W += (torch.randn(n, _groups(k, 32), generator=g, device=DEV) * 0.01).repeat_interleave(32, dim=1)[:, :k]
    return W


def _made(case, seed):
    """The inputs, from the seed alone."""
    g, op, n, k = _gen(1000 + seed), case["op"], case["n"], case["k"]
    dt = TYPES[case["type"]]
    if op == "weight":
        return {"W": _weights(case, g).to(dt)}
    m = case["m"]
    st = {}
    if op == "gemm" or op == "gated":
        st["X"] = _activations(m, k, g).to(dt)
    elif op == "gemm_t":
        st["dY"] = (torch.randn(m, n, generator=g, device=DEV) * 0.02).to(dt)
    else:
        st["dH"] = (torch.randn(m, n, generator=g, device=DEV) * 0.02).to(dt)
        st["G"], st["U"] = (torch.randn(m, n, generator=g, device=DEV) * 2.0).to(dt), (torch.randn(m, n, generator=g, device=DEV) * 2.0).to(dt)
    st["layers"] = [_quantize(_weights(case, g), case["group"], case["zeros"]) for _ in range(2 if op in ("gated", "backward") else 1)]
    return st


def prepare(case, seed):
    st = _made(case, seed)
    op, n, k, dt = case["op"], case["n"], case["k"], TYPES[case["type"]]
    if op == "weight":
        st["values"] = torch.empty(n, k, dtype=dt, device=DEV)
        if own:
            from paper_2410_09615_amd import binding as B
            st["layer"] = B.alloc_group_q4(n, k, case["group"], zeros=case["zeros"], device=DEV)
    else:
        m = case["m"]
        if op == "gemm":
            st["Y"] = torch.empty(m, n, dtype=dt, device=DEV)
        elif op == "gated":
            for name in ("H", "G", "U") if case["keep"] else ("H",):
                st[name] = torch.empty(m, n, dtype=dt, device=DEV)
        else:
            st["dX"] = torch.empty(m, k, dtype=dt, device=DEV)
            if op == "backward":
                st["dG"], st["dU"] = torch.empty(m, n, dtype=dt, device=DEV), torch.empty(m, n, dtype=dt, device=DEV)
        if own:
            from paper_2410_09615_amd import binding as B
            st["layers"] = [B.SlimGroupQ4Weight(n, k, case["group"], B.slim_group_q4_tile(codes), scales, zeros)
                            for codes, scales, zeros in st["layers"]]
    st["case"] = case
    return st


def _run_own(st):
    from paper_2410_09615_amd import binding as B
    op = st["case"]["op"]
    if op == "weight":
        layer = B.slim_group_q4_weight(st["W"], layer=st["layer"])
        values = B.slim_group_q4_values(layer, values=st["values"])
        out = {"values": values, "scales": layer.scales}
        return out if layer.zeros is None else {**out, "zeros": layer.zeros}
    if op == "gemm":
        return B.slim_group_q4_gemm(st["layers"][0], st["X"], Y=st["Y"])
    if op == "gated":
        H, G, U = B.slim_group_q4_gated(*st["layers"], st["X"], H=st["H"], G=st.get("G"), U=st.get("U"))
        return {"H": H, "G": G, "U": U} if st["case"]["keep"] else H
    if op == "gemm_t":
        return B.slim_group_q4_gemm_t(st["layers"][0], st["dY"], dX=st["dX"])
    dX, dG, dU = B.slim_group_q4_gated_backward(*st["layers"], st["dH"], st["G"], st["U"], dG=st["dG"], dU=st["dU"], dX=st["dX"])
    return {"dX": dX, "dG": dG, "dU": dU}


def run(st):
    if own:
        return _run_own(st)
    case = st["case"]
    op, size, dt = case["op"], case["group"], TYPES[case["type"]]
    if op == "weight":
        codes, scales, zeros = _quantize(st["W"].float(), size, case["zeros"])
        out = {"values": _values(codes, scales, zeros, size).to(dt), "scales": scales}
        return out if zeros is None else {**out, "zeros": zeros}
    W = [_values(*layer, size) for layer in st["layers"]]
    if op == "gemm":
        return (st["X"].float() @ W[0].t()).to(dt)
    if op == "gated":
        X = st["X"].float()
        G, U = X @ W[0].t(), X @ W[1].t()
        H = G / (1.0 + torch.exp(-G)) * U
        return {"H": H.to(dt), "G": G.to(dt), "U": U.to(dt)} if case["keep"] else H.to(dt)
    if op == "gemm_t":
        return (st["dY"].float() @ W[0]).to(dt)
    G, U, dH = st["G"].float(), st["U"].float(), st["dH"].float()
    sig = 1.0 / (1.0 + torch.exp(-G))
    dU = dH * (G * sig)
    dG = dH * U * (sig * (1.0 + G * (1.0 - sig)))
    return {"dX": (dG @ W[0] + dU @ W[1]).to(dt), "dG": dG.to(dt), "dU": dU.to(dt)}


def work(case):
    op, n, k = case["op"], case["n"], case["k"]
    size = {"f16": 2, "bf16": 2, "f32": 4}[case["type"]]
    held = n * ((k + 1) // 2) + n * _groups(k, case["group"]) * (3 if case["zeros"] else 2)
    if op == "weight":                       # quantized, and read back
        return {"bytes": 2 * (n * k * size + held), "flops": 6 * n * k}
    m = case["m"]
    if op == "gemm" or op == "gemm_t":
        return {"bytes": held + size * m * (n + k), "flops": 2 * m * n * k}
    if op == "gated":
        return {"bytes": 2 * held + size * m * (k + n * (3 if case["keep"] else 1)), "flops": 4 * m * n * k + 6 * m * n}
    return {"bytes": 2 * held + size * m * (5 * n + k), "flops": 4 * m * n * k + 12 * m * n}


def _near32(q):
    """A quotient in 64 bits as the nearest one of 32: the definition's."""
    return q.to(torch.float32).double()


def _exact_weight(W, size, zeros):
    n, k = W.shape
    col = torch.arange(k, device=W.device) // size
    kg = int(col[-1]) + 1
    top = torch.zeros(n, kg, dtype=torch.float64, device=W.device)
    low = torch.zeros(n, kg, dtype=torch.float64, device=W.device)
    for g in range(kg):
        part = W[:, g * size:(g + 1) * size]
        if zeros:
            top[:, g], low[:, g] = part.max(dim=1).values, part.min(dim=1).values
        else:
            top[:, g] = part.abs().max(dim=1).values
    if zeros:
        top, low = top.clamp(min=0), low.clamp(max=0)
    span = _near32(top - low)
    scale = _near32(span / (15 if zeros else 7)).to(torch.float16).double().clamp(TINY, LARGE)
    scale[span == 0] = 1.0
    zero = _near32(-low / scale).round().clamp(0, 15) if zeros else None
    q = _near32(W / scale[:, col]).round()
    q = torch.minimum(torch.maximum(q, -zero[:, col]), 15 - zero[:, col]) if zeros else q.clamp(-8, 7)
    return q * scale[:, col], scale, zero


def _exact_values(layer, size):
    codes, scales, zeros = layer
    col = torch.arange(codes.shape[1], device=codes.device) // size
    point = 8 if zeros is None else zeros[:, col].double()
    return (codes.double() - point) * scales[:, col].double()


def exact(case, seed):
    """The same from the definitions in 64 bits."""
    st, op, size = _made(case, seed), case["op"], case["group"]
    if op == "weight":
        values, scales, zeros = _exact_weight(st["W"].double(), size, case["zeros"])
        return {"values": values, "scales": scales} if zeros is None else {"values": values, "scales": scales, "zeros": zeros.to(torch.uint8)}
    first = _exact_values(st["layers"][0], size)
    if op == "gemm":
        return st["X"].double() @ first.t()
    if op == "gemm_t":
        return st["dY"].double() @ first
    if op == "gated":
        X = st["X"].double()
        G = X @ first.t()
        del first
        U = X @ _exact_values(st["layers"][1], size).t()
        H = G * torch.sigmoid(G) * U
        return {"H": H, "G": G, "U": U} if case["keep"] else H
    G, U, dH = st["G"].double(), st["U"].double(), st["dH"].double()
    sig = torch.sigmoid(G)
    dG, dU = dH * U * (sig + G * sig * (1 - sig)), dH * G * sig
    return {"dX": dG @ first + dU @ _exact_values(st["layers"][1], size), "dG": dG, "dU": dU}
