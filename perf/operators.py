"""What is timed of the 8-bit operators with a scale for each block of 128: their plain form and the framework's calls.

A layer that is not compressed to 4 bits runs in 8: its weights are quantized once,
128 x 128 weights to a scale (`slim_block_fp8_weight`, or codes that a checkpoint
brings are laid out by `slim_block_fp8_tile`), its inputs are quantized where they
are made, 128 inputs of a token to a scale -- by the norm that adds the residual
(`slim_block_fp8_norm`) or by the gated activation (`slim_block_fp8_act`) -- and
`slim_block_fp8_gemm` multiplies the two.  Sizes are the layers of the package's
workloads (4096 x 4096 to 28672 x 8192, 1 to 4096 tokens) and odd ones between.
Inputs are made on the device, with the distributions of those workloads.
"""
from __future__ import annotations

import math

import torch

DEV = "cuda:0"
own = False

BLK = 128            # values to a scale
FMAX = 448.0         # largest value of the 8-bit format (E4M3)
FLOOR = 2.0 ** -100  # a block's largest magnitude counts as this much at least
EPS = 1e-5
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one sequence being decoded on the widest model: the smallest call, two per layer and token
        {"name": "norm_1x8192", "op": "norm", "m": 1, "k": 8192, "type": "f16", "residual": True, "wide": False},
        # a prompt whose length and width are multiples of nothing; the values are wanted in 16 bits too (a 4-bit layer reads them)
        {"name": "norm_1777x5003_bf16", "op": "norm", "m": 1777, "k": 5003, "type": "bf16", "residual": True, "wide": True},
        # a chunk of a long prompt on the widest model
        {"name": "norm_4096x8192", "op": "norm", "m": 4096, "k": 8192, "type": "f16", "residual": True, "wide": False},
        # the inner activations of a decode step of 16 sequences: both halves of one product's output
        {"name": "act_16x13824", "op": "act", "m": 16, "k": 13824, "type": "f16", "gated": True},
        # those of an ordinary prompt
        {"name": "act_2048x11008_bf16", "op": "act", "m": 2048, "k": 11008, "type": "bf16", "gated": True},
        # quantizing one attention projection, and the largest layer as a checkpoint holds it
        {"name": "weight_4096x4096", "op": "weight", "n": 4096, "k": 4096, "type": "f32"},
        {"name": "weight_28672x8192_bf16", "op": "weight", "n": 28672, "k": 8192, "type": "bf16"},
        # one sequence being decoded, the smallest layer: one call per projection and token
        {"name": "product_1_4096x4096", "op": "product", "m": 1, "n": 4096, "k": 4096, "type": "f16"},
        # a few sequences decoded together on the largest layer
        {"name": "product_16_28672x8192", "op": "product", "m": 16, "n": 28672, "k": 8192, "type": "f16"},
        # a busy server's decode step
        {"name": "product_48_5120x5120_bf16", "op": "product", "m": 48, "n": 5120, "k": 5120, "type": "bf16"},
        # a short prompt, sizes that are multiples of nothing, the results in 32 bits (scores of a vocabulary)
        {"name": "product_333_10007x4100_f32", "op": "product", "m": 333, "n": 10007, "k": 4100, "type": "f32"},
        # a chunk of a long prompt on the largest layer
        {"name": "product_4096_28672x8192", "op": "product", "m": 4096, "n": 28672, "k": 8192, "type": "f16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Any number, half of the time a multiple of 128 where it is large enough to be one."""
    v = _log_int(rng, lo, hi)
    return v // 128 * 128 if v >= 256 and rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["norm", "act", "weight", "product", "product", "product"])
    wide = rng.choice(["f16", "bf16"])
    if op == "norm":
        return {"op": op, "m": _log_int(rng, 1, 4096), "k": _size(rng, 128, 8192), "type": wide,
                "residual": rng.random() < 0.7, "wide": rng.random() < 0.3}
    if op == "act":
        return {"op": op, "m": _log_int(rng, 1, 2048), "k": _size(rng, 128, 11008), "type": wide, "gated": rng.random() < 0.7}
    if op == "weight":
        return {"op": op, "n": _size(rng, 128, 28672), "k": _size(rng, 128, 8192), "type": rng.choice(["f32", "f16", "bf16"])}
    return {"op": op, "m": _log_int(rng, 1, 4096), "n": _size(rng, 128, 28672), "k": _size(rng, 128, 8192),
            "type": rng.choice(["f16", "f16", "bf16", "f32"])}


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _activations(m, k, g):
    X = torch.randn(m, k, generator=g, device=DEV)
    X[:, torch.randperm(k, generator=g, device=DEV)[:math.ceil(0.01 * k)]] *= 20.0      # outlier channels
    return X


def _blocks(k):
    return (k + BLK - 1) // BLK


def _padded(t, rows, cols):
    return torch.nn.functional.pad(t, (0, cols - t.shape[1], 0, rows - t.shape[0]))


def _quantize_rows(z):
    """z [m][k] fp32 -> (codes [m][128 blocks], largest magnitude of a block [m][blocks]); padded with zeros."""
    m, k = z.shape
    kb = _blocks(k)
    z = _padded(z, m, kb * BLK).view(m, kb, BLK)
    top = z.abs().amax(dim=2).clamp_min(FLOOR)
    codes = (z * (FMAX / top)[:, :, None]).to(torch.float8_e4m3fn)
    return codes.view(m, kb * BLK), top


def _quantize_weight(W):
    """W [n][k] fp32 -> (codes [n][k] row-major, padded to whole blocks; scales [n blocks][k blocks])."""
    n, k = W.shape
    nb, kb = _blocks(n), _blocks(k)
    W = _padded(W, nb * BLK, kb * BLK).view(nb, BLK, kb, BLK)
    top = W.abs().amax(dim=3).amax(dim=1).clamp_min(FLOOR)
    codes = (W * (FMAX / top)[:, None, :, None]).to(torch.float8_e4m3fn)
    return codes.view(nb * BLK, kb * BLK), top / FMAX


def _tiled(codes, n):
    """Row-major codes -> the order in which the matrix instructions hold them: tiles of 64 rows x 128 inputs; a row in
    a tile is 16 g + 4 t + r, an input 64 h + 16 q + b, and a byte's place is (t, h, q, g, r, b)."""
    rows, cols = -(-n // 64) * 64, codes.shape[1]
    c = codes.view(torch.uint8)[:rows].view(rows // 64, 4, 4, 4, cols // 128, 2, 4, 16)   # tile row, g, t, r, tile column, h, q, b
    return c.permute(0, 4, 2, 5, 6, 1, 3, 7).contiguous().view(-1)


def prepare(case, seed):
    g, op = _gen(1000 + seed), case["op"]
    dt = TYPES[case["type"]]
    st = {"case": case, "type": dt}
    if op == "norm":
        m, k = case["m"], case["k"]
        st["X"] = _activations(m, k, g).to(dt)
        st["gain"] = (1.0 + 0.1 * torch.randn(k, generator=g, device=DEV)).to(dt)
        if case["residual"]:
            st["residual"] = (4.0 * torch.randn(m, k, generator=g, device=DEV)).to(dt)
            st["H"] = torch.empty(m, k, dtype=dt, device=DEV)
        if case["wide"]:
            st["Y"] = torch.empty(m, k, dtype=dt, device=DEV)
    elif op == "act":
        m, k = case["m"], case["k"]
        both = torch.randn(m, 2 * k if case["gated"] else k, generator=g, device=DEV).to(dt)
        st["G"], st["U"] = (both[:, :k], both[:, k:]) if case["gated"] else (both, None)
    elif op == "weight":
        n, k = case["n"], case["k"]
        st["W"] = (torch.randn(n, k, generator=g, device=DEV) * 0.02).to(dt)
        rows, kb = -(-n // 64) * 64, _blocks(k)
        st["codes"] = torch.empty(rows * kb * BLK, dtype=torch.uint8, device=DEV)
        st["scales"] = torch.empty(_blocks(n), kb, device=DEV)
        return st
    else:
        m, n, k = case["m"], case["n"], case["k"]
        codes, top = _quantize_rows(_activations(m, k, g))
        st["codes"], st["scales"] = codes.view(torch.uint8), top / FMAX
        wcodes, wscales = _quantize_weight(torch.randn(n, k, generator=g, device=DEV) * 0.02)
        wcodes = wcodes.view(torch.uint8)[:n, :k].contiguous()          # as a checkpoint holds them
        st["Y"] = torch.empty(m, n, dtype=dt, device=DEV)
        if own:
            from paper_2410_09615_amd import binding as B
            st["layer"] = B.SlimBlockFp8Weight(n, k, B.slim_block_fp8_tile(wcodes), wscales)
            st["ws"] = B.alloc_block_fp8_workspace(st["layer"], m)
        else:
            st["wcodes"], st["wscales"] = wcodes, wscales
        return st
    kb = _blocks(case["k"])
    st["codes"] = torch.empty(case["m"], kb * BLK, dtype=torch.uint8, device=DEV)
    st["scales"] = torch.empty(case["m"], kb, device=DEV)
    return st


def _run_own(st):
    from paper_2410_09615_amd import binding as B
    op = st["case"]["op"]
    if op == "norm":
        codes, scales, H, Y = B.slim_block_fp8_norm(st["X"], st["gain"], EPS, residual=st.get("residual"), codes=st["codes"],
                                                    scales=st["scales"], H=st.get("H"), Y=st.get("Y"))
        return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales, "H": H, "Y": Y}
    if op == "act":
        codes, scales = B.slim_block_fp8_act(st["G"], st["U"], act="silu" if st["case"]["gated"] else "none", codes=st["codes"],
                                             scales=st["scales"])
        return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales}
    if op == "weight":
        codes, scales = B.slim_block_fp8_weight(st["W"], codes=st["codes"], scales=st["scales"])
        return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales}
    return B.slim_block_fp8_gemm(st["layer"], st["codes"], st["scales"], Y=st["Y"], workspace=st["ws"])


def run(st):
    if own:
        out = _run_own(st)
        return {k: v for k, v in out.items() if v is not None} if isinstance(out, dict) else out
    case, dt = st["case"], st["type"]
    op = case["op"]
    if op == "norm":
        h = st["X"].float()
        if case["residual"]:
            h = h + st["residual"].float()
        rstd = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
        z = h * st["gain"].float()
        # the row's factor is in the scale alone: a block's codes are z over the block's largest, whatever that factor is
        codes, top = _quantize_rows(z)
        out = {"codes": codes, "scales": top / FMAX * rstd}
        if case["residual"]:
            out["H"] = h.to(dt)
        if case["wide"]:
            out["Y"] = (z * rstd).to(dt)
        return out
    if op == "act":
        a = st["G"].float()
        if case["gated"]:
            a = a / (1.0 + torch.exp(-a)) * st["U"].float()
        codes, top = _quantize_rows(a)
        return {"codes": codes, "scales": top / FMAX}
    if op == "weight":
        codes, scales = _quantize_weight(st["W"].float())
        return {"codes": _tiled(codes, case["n"]).view(torch.float8_e4m3fn), "scales": scales}
    m, n, k = case["m"], case["n"], case["k"]
    X = st["codes"].view(torch.float8_e4m3fn)[:, :k].float() * st["scales"].repeat_interleave(BLK, dim=1)[:, :k]
    W = st["wcodes"].view(torch.float8_e4m3fn).float()
    W = W * st["wscales"].repeat_interleave(BLK, dim=0)[:n].repeat_interleave(BLK, dim=1)[:, :k]
    return (X @ W.t()).to(dt)


def work(case):
    size = {"f16": 2, "bf16": 2, "f32": 4}[case["type"]]
    op, k = case["op"], case["k"]
    kb = _blocks(k)
    if op == "norm":
        m = case["m"]
        streams = 1 + (2 if case["residual"] else 0) + (1 if case["wide"] else 0)
        return {"bytes": m * k * (size * streams + 1) + 4 * m * kb + size * k, "flops": 8 * m * k}
    if op == "act":
        m = case["m"]
        return {"bytes": m * k * (size * (2 if case["gated"] else 1) + 1) + 4 * m * kb, "flops": (8 if case["gated"] else 3) * m * k}
    if op == "weight":
        n = case["n"]
        return {"bytes": n * k * (size + 1) + 4 * _blocks(n) * kb, "flops": 3 * n * k}
    m, n = case["m"], case["n"]
    return {"bytes": (m + n) * k + 4 * (m + _blocks(n)) * kb + size * m * n, "flops": 2 * m * n * k}


def _nearest8(q):
    """The value of the 8-bit format (four exponent bits of bias 7, three of mantissa, subnormals) nearest to q, ties to even."""
    _, e = torch.frexp(q)                                      # |q| = f 2^e, f in [1/2, 1)
    step = torch.ldexp(torch.ones_like(q), e.clamp_min(-5) - 4)
    return (torch.round(q / step) * step).clamp(-FMAX, FMAX)


def _exact_rows(z):
    m, k = z.shape
    kb = -(-k // BLK)
    full = torch.zeros(m, kb * BLK, dtype=torch.float64, device=z.device)
    full[:, :k] = z
    top = torch.clamp(full.abs().unflatten(1, (kb, BLK)).max(dim=2).values, min=FLOOR)
    return _nearest8(full * FMAX / torch.repeat_interleave(top, BLK, 1)), top / FMAX


def exact(case, seed):
    """The same from the definitions in 64 bits."""
    st = prepare(case, seed)
    op, k = case["op"], case["k"]
    if op == "norm":
        h = st["X"].double()
        if case["residual"]:
            h = h + st["residual"].double()
        factor = 1.0 / torch.sqrt(torch.sum(h * h, dim=1) / k + EPS)
        z = h * st["gain"].double()[None, :]
        codes, scales = _exact_rows(z)
        out = {"codes": codes, "scales": scales * factor[:, None]}
        if case["residual"]:
            out["H"] = h
        if case["wide"]:
            out["Y"] = z * factor[:, None]
        return out
    if op == "act":
        a = st["G"].double()
        if case["gated"]:
            a = a * torch.sigmoid(a) * st["U"].double()
        codes, scales = _exact_rows(a)
        return {"codes": codes, "scales": scales}
    if op == "weight":
        W = st["W"].double()
        n = case["n"]
        rows, kb, nb = -(-n // 64) * 64, -(-k // BLK), -(-n // BLK)
        full = torch.zeros(nb * BLK, kb * BLK, dtype=torch.float64, device=DEV)
        full[:n, :k] = W
        del W
        top = torch.clamp(full.abs().unflatten(1, (kb, BLK)).amax(dim=2).unflatten(0, (nb, BLK)).amax(dim=1), min=FLOOR)
        place = torch.arange(rows * kb * BLK, device=DEV)
        tile, at = place // 8192, place % 8192
        t, h, q, g, r, b = at // 2048, at // 1024 % 2, at // 256 % 4, at // 64 % 4, at // 16 % 4, at % 16
        o = tile // kb * 64 + 16 * g + 4 * t + r
        i = tile % kb * BLK + 64 * h + 16 * q + b
        del tile, at, t, h, q, g, r, b, place
        return {"codes": _nearest8(full[o, i] * FMAX / top[o // BLK, i // BLK]), "scales": top / FMAX}
    m, n = case["m"], case["n"]
    g = _gen(1000 + seed)
    codes, top = _quantize_rows(_activations(m, k, g))
    wcodes, wscales = _quantize_weight(torch.randn(n, k, generator=g, device=DEV) * 0.02)
    col = torch.arange(k, device=DEV) // BLK
    X = codes[:, :k].double() * (top / FMAX).double()[:, col]
    W = wcodes[:n, :k].double() * wscales.double()[torch.arange(n, device=DEV) // BLK][:, col]
    return X @ W.t()
