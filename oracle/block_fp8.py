"""CPU oracle of the 8-bit operators with a scale for each block of 128 (test infrastructure only).

What include/slim.h defines in binary32 (codes, tops) is computed in binary32 here, one rounding
per operation, and compared bit for bit; sums, norms and products are in 64 bits.
"""
from __future__ import annotations

import numpy as np

from oracle.slim_oracle import fp8_encode, fp8_round

BLK = 128
FMAX = np.float32(448.0)
FLOOR = np.float32(2.0 ** -100)


def blocks(k: int) -> int:
    return -(-k // BLK)


def _codes(z: np.ndarray, top: np.ndarray) -> np.ndarray:
    """Codes of z (binary32) with `top` of each element's block."""
    with np.errstate(all="ignore"):
        q = (z * (FMAX / top).astype(np.float32)).astype(np.float32)
    nan = np.isnan(q)
    codes = fp8_encode(fp8_round(np.where(nan, 0.0, q), "e4m3"), "e4m3")
    return np.where(nan, np.uint8(0x7F), codes)


def quantize_rows(z: np.ndarray):
    """z [m][k] binary32 -> (codes uint8 [m][128 kb], top binary32 [m][kb]); the scale is top / 448."""
    m, k = z.shape
    kb = blocks(k)
    full = np.zeros((m, kb * BLK), np.float32)
    full[:, :k] = z
    b = full.reshape(m, kb, BLK)
    top = np.maximum(np.abs(b).max(axis=2), FLOOR)          # np.max and np.maximum hand a NaN on
    return _codes(b, top[:, :, None]).reshape(m, kb * BLK), top


def norm(X: np.ndarray, gain, eps: float, residual=None):
    """X, residual, gain as binary32 holding their type's values -> dict of codes, scales (64 bits), h (binary32), y (64 bits)."""
    with np.errstate(all="ignore"):
        h = X if residual is None else (X + residual).astype(np.float32)
        h64 = h.astype(np.float64)
        rstd = 1.0 / np.sqrt((h64 * h64).mean(axis=1) + eps)
        z = h if gain is None else (h * gain).astype(np.float32)
        codes, top = quantize_rows(z)
        zy = h64 if gain is None else h64 * gain.astype(np.float64)
        return {"codes": codes, "scales": top.astype(np.float64) / 448.0 * rstd[:, None], "h": h, "y": zy * rstd[:, None]}


def act(G: np.ndarray, U, silu: bool) -> np.ndarray:
    """act(G) * U in 64 bits."""
    g = G.astype(np.float64)
    with np.errstate(all="ignore"):
        a = g / (1.0 + np.exp(-g)) if silu else g
        return a if U is None else a * U.astype(np.float64)


def weight(W: np.ndarray):
    """W [n][k] binary32 -> (codes uint8 [n][k] row-major, scales binary32 [n blocks][k blocks])."""
    n, k = W.shape
    nb, kb = blocks(n), blocks(k)
    full = np.zeros((nb * BLK, kb * BLK), np.float32)
    full[:n, :k] = W
    b = full.reshape(nb, BLK, kb, BLK)
    top = np.maximum(np.abs(b).max(axis=3).max(axis=1), FLOOR)
    codes = _codes(b, top[:, None, :, None]).reshape(nb * BLK, kb * BLK)
    return np.ascontiguousarray(codes[:n, :k]), (top / FMAX).astype(np.float32)


def tile(codes: np.ndarray) -> np.ndarray:
    """Row-major codes [n][k] in the tiles of include/slim.h, written out byte by byte from the definition."""
    n, k = codes.shape
    rows, kb = -(-n // 64) * 64, blocks(k)
    out = np.zeros(rows * kb * BLK, np.uint8)
    o, i = np.meshgrid(np.arange(n), np.arange(k), indexing="ij")
    ol, il = o % 64, i % 128
    g, t, r = ol // 16, ol // 4 % 4, ol % 4
    h, q, b = il // 64, il // 16 % 4, il % 16
    out[(o // 64 * kb + i // 128) * 8192 + 2048 * t + 1024 * h + 256 * q + 64 * g + 16 * r + b] = codes
    return out


_VALUES = None


def values(codes: np.ndarray) -> np.ndarray:
    """What codes stand for, in 64 bits (0x7F and 0xFF: NaN)."""
    global _VALUES
    if _VALUES is None:
        c = np.arange(256)
        e, f = (c >> 3) & 15, c & 7
        v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * np.exp2(e - 10.0))
        v[(c & 0x7F) == 0x7F] = np.nan
        _VALUES = np.where(c & 0x80, -v, v)
    return _VALUES[codes]


def gemm(xc: np.ndarray, xs: np.ndarray, wc: np.ndarray, ws: np.ndarray):
    """(Y, sum of the magnitudes of its terms), both [m][n] in 64 bits; xc [m][128 kb], xs [m][kb], wc [n][k] row-major, ws [n blocks][kb]."""
    n, k = wc.shape
    X = values(xc)[:, :k] * np.repeat(xs.astype(np.float64), BLK, axis=1)[:, :k]
    W = values(wc) * np.repeat(np.repeat(ws.astype(np.float64), BLK, axis=0)[:n], BLK, axis=1)[:, :k]
    return X @ W.T, np.abs(X) @ np.abs(W).T
