"""4-bit weights with a scale for each group of inputs: definition in numpy, quotients in binary32 as the format says, everything else in binary64."""
import numpy as np

SYMMETRIC = 8


def groups(k, group):
    return -(-k // group)


def quantize(W, group, zeros):
    """W [n][k] float32 -> (codes uint8 [n][k], scales float16 [n][groups], zero points uint8 [n][groups] or None)."""
    W = np.asarray(W, np.float32)
    n, k = W.shape
    codes = np.zeros((n, k), np.uint8)
    scales = np.zeros((n, groups(k, group)), np.float16)
    points = np.zeros(scales.shape, np.uint8) if zeros else None
    with np.errstate(all="ignore"):
        for g in range(scales.shape[1]):
            w = W[:, g * group:(g + 1) * group]
            odd = ~np.isfinite(w).all(axis=1)
            lo, hi = np.minimum(w.min(axis=1), np.float32(0)), np.maximum(w.max(axis=1), np.float32(0))
            span = hi - lo if zeros else np.maximum(hi, -lo)
            s = (span / np.float32(15 if zeros else 7)).astype(np.float16)
            s[s == 0] = np.float16(2.0 ** -24)
            s[span == 0] = np.float16(1)
            s = np.minimum(s, np.float16(65504))
            sf = s.astype(np.float32)
            z = np.clip(np.rint(-lo / sf), 0, 15) if zeros else np.full(n, np.float32(SYMMETRIC))
            c = np.clip(np.rint(w / sf[:, None]) + z[:, None], 0, 15)
            c[odd], s[odd], z[odd] = 0, np.nan, 0
            codes[:, g * group:(g + 1) * group] = c.astype(np.uint8)
            scales[:, g] = s
            if zeros:
                points[:, g] = z.astype(np.uint8)
    return codes, scales, points


def values(codes, scales, points, group):
    """(c - z) s in binary64, [n][k]."""
    col = np.arange(codes.shape[1]) // group
    z = SYMMETRIC if points is None else points[:, col].astype(np.float64)
    return (codes.astype(np.float64) - z) * scales[:, col].astype(np.float64)


def tile(codes):
    """Row-major codes [n][k] -> the bytes of the blocks."""
    n, k = codes.shape
    rb, cb = -(-n // 16), -(-k // 128)
    full = np.zeros((rb * 16, cb * 128), np.uint8)
    full[:n, :k] = codes & 15
    c = full.reshape(rb, 16, cb, 4, 4, 4, 2)                         # row block, r, column block, j, q, i, h: input 32 j + 8 q + 2 i + h
    c = c.transpose(0, 2, 4, 1, 3, 6, 5).reshape(rb, cb, 4, 16, 4, 8).astype(np.uint32)     # ..., q, r, j, nibble i + 4 h
    words = (c << (4 * np.arange(8, dtype=np.uint32))).sum(axis=-1, dtype=np.uint32)
    return words.astype("<u4").reshape(-1).view(np.uint8)


def gemm(X, V):
    """(X V^T, sum of the terms' magnitudes)."""
    X = np.asarray(X, np.float64)
    return X @ V.T, np.abs(X) @ np.abs(V).T


def sigma(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-np.asarray(g, np.float64)))


def gated(G, U):
    return G * sigma(G) * U


def gated_backward(dH, G, U):
    """(dG, dU)."""
    s = sigma(G)
    return dH * U * s * (1.0 + G * (1.0 - s)), dH * G * s
