"""The feed-forward part of a decoder layer on the library's kernels: an example of the 8-bit operators as a serving loop uses them.

    h = X + residual;  y = rmsnorm(h) gain;  out = (silu(y Wg^T) * (y Wu^T)) Wd^T

`Wg` and `Wu` are one layer of 2 f rows (gate first), in 8 bits (SlimBlockFp8Weight) or compressed to 4 (SlimLayer, whose
forward call reads the norm's output in fp16); `Wd` is in 8 bits.  Four launches with 8-bit layers, whatever the number of
tokens: the norm with the residual's addition writes 8-bit codes, the product reads them, the gated activation writes codes
of its output, the second product reads those.  Returned are out and h, the next part's X and residual.

    python -m paper_2410_09615_amd.mlp [tokens]        # 4096 x 11008: a prompt, and a decode step recorded into a HIP graph
"""
from __future__ import annotations

import sys
import time

import torch

from paper_2410_09615_amd import binding as slim


class DecoderMlp:
    """Weights of one layer and buffers for up to `max_tokens` tokens; calls follow one another on one stream."""

    def __init__(self, gain: torch.Tensor, gate_up: slim.SlimBlockFp8Weight | slim.SlimLayer, down: slim.SlimBlockFp8Weight, max_tokens: int,
                 eps: float = 1e-5):
        if gate_up.n != 2 * down.k or gate_up.k != down.n:
            raise ValueError("gate_up must be [2 f][k] and down [k][f]")
        self.gain, self.gate_up, self.down, self.eps, self.max_tokens = gain, gate_up, down, eps, max_tokens
        self.k, self.f = gate_up.k, down.k
        self.packed = isinstance(gate_up, slim.SlimLayer)
        dev = down.codes.device
        kb, fb = (self.k + 127) // 128, (self.f + 127) // 128
        byte = lambda *shape: torch.empty(*shape, dtype=torch.uint8, device=dev)
        real = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=dev)
        half = lambda *shape: torch.empty(*shape, dtype=torch.float16, device=dev)
        self._x, self._xs = byte(max_tokens, kb * 128), real(max_tokens, kb)
        self._a, self._as = byte(max_tokens, fb * 128), real(max_tokens, fb)
        self._gu = half(max_tokens, 2 * self.f)
        self._y = half(max_tokens, self.k) if self.packed else None
        if self.packed:        # what a call needs does not grow with its tokens throughout: the most that any number of them does
            room = max(slim.slim_workspace_bytes(gate_up, m) for m in range(1, max_tokens + 1))
            self._ws = torch.zeros(room, dtype=torch.uint8, device=dev)
        else:
            self._ws = slim.alloc_block_fp8_workspace(gate_up, max_tokens)
        self._wd = slim.alloc_block_fp8_workspace(down, max_tokens)

    def __call__(self, X: torch.Tensor, residual: torch.Tensor | None = None, out: torch.Tensor | None = None, h: torch.Tensor | None = None):
        """X, residual fp16 [m][k] -> (out, h), both fp16 [m][k]; h may be X or residual."""
        m = X.shape[0]
        if m > self.max_tokens:
            raise ValueError(f"{m} tokens, made for {self.max_tokens}")
        if X.dtype is not torch.float16:
            raise ValueError("X must be float16")
        gu = self._gu[:m]
        codes, scales, h, y = slim.slim_block_fp8_norm(X, self.gain, self.eps, residual=residual, codes=self._x[:m], scales=self._xs[:m],
                                                       H=True if h is None else h, Y=self._y[:m] if self.packed else None)
        if self.packed:
            forward = slim.slim_linear_gemv if m <= 16 else slim.slim_linear_gemm
            forward(self.gate_up, y, Y=gu, workspace=self._ws)
        else:
            slim.slim_block_fp8_gemm(self.gate_up, codes, scales, Y=gu, workspace=self._ws)
        a, a_scales = slim.slim_block_fp8_act(gu[:, :self.f], gu[:, self.f:], codes=self._a[:m], scales=self._as[:m])
        return slim.slim_block_fp8_gemm(self.down, a, a_scales, Y=out, workspace=self._wd), h


def _demo(tokens: int) -> None:
    dev, k, f = torch.device("cuda:0"), 4096, 11008
    g = torch.Generator(device=dev)
    g.manual_seed(0)
    gain = (1 + 0.1 * torch.randn(k, generator=g, device=dev)).half()
    gate_up = torch.randn(2 * f, k, generator=g, device=dev) * 0.02
    down = torch.randn(k, f, generator=g, device=dev) * 0.02
    mlp = DecoderMlp(gain, slim.compress_block_fp8(gate_up), slim.compress_block_fp8(down), max(tokens, 16))
    X, residual = (torch.randn(tokens, k, generator=g, device=dev).half() for _ in range(2))
    out, h = mlp(X, residual)
    y = h.float() * torch.rsqrt(h.float().pow(2).mean(1, keepdim=True) + mlp.eps) * gain.float()
    gu = y @ gate_up.t()
    want = (gu[:, :f] * torch.sigmoid(gu[:, :f]) * gu[:, f:]) @ down.t()
    print(f"{tokens} tokens: relative difference from fp32 weights and inputs {float((out.float() - want).norm() / want.norm()):.4f}")
    # a decode step: fixed buffers, recorded once
    x1, r1, o1 = X[:1].clone(), residual[:1].clone(), torch.empty(1, k, dtype=torch.float16, device=dev)
    mlp(x1, r1, out=o1, h=r1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mlp(x1, r1, out=o1, h=r1)
    for name, step in ((f"{tokens} tokens", lambda: mlp(X, residual, out=out, h=h)), ("1 token, recorded", graph.replay)):
        for _ in range(5):
            step()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(50):
            step()
        torch.cuda.synchronize()
        print(f"{name}: {(time.perf_counter() - t) / 50 * 1e6:.1f} us")


if __name__ == "__main__":
    _demo(int(sys.argv[1]) if len(sys.argv) > 1 else 512)
